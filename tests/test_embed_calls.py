"""CPU-only: calls of include/tagore_embed.h that are refused, and what the workspaces cost."""
import ctypes

P, Q, R = (ctypes.c_void_p(256 * i) for i in (1, 2, 3))          # never followed: every call below is refused


def test_norms_in_place_of_rows_that_are_apart():
    """out_r has rows of d: written over x or the residual, it would meet rows still to be read if those are further apart."""
    from paper_2508_08744_amd import embed
    L = embed.lib()
    for x, ld_x, res, ld_res in ((R, 72, Q, 64), (Q, 64, R, 72), (R, 72, R, 64), (R, 72, R, 72)):
        assert L.tg_add_rms_norm(x, ld_x, res, ld_res, P, 1, 10, 64, 1e-6, P, R, P, None) == -1
        assert b"back to back" in L.tg_last_error()
        assert L.tg_add_rms_norm_q8(x, ld_x, res, ld_res, P, 1, 10, 64, 1e-6, P, P, R, None) == -1
        assert b"back to back" in L.tg_last_error()
