// Softmax cross entropy of n rows against all rows of a table, and its gradients, without the logits.
//
// Forward: a tile of logits stays in the registers of the workgroup that formed it and leaves a maximum and a sum of exponentials for
// every token; a second kernel joins them over the table.  2 n n_rows d operations on the matrix instructions bound it, or, for
// few tokens, the bytes of the table.  (8192 tokens, 131 072 rows of 1024 bf16: 1.9 ms, 1.14 PFLOP/s; 48 tokens: 41 us, 6.6 TB/s.)
//
// Gradient: the logits are formed again, a piece of the table at a time, and become P = scale dloss (softmax - [target]) in the
// inputs' type, which goes to memory once (a piece is small enough to be read again while the last-level cache holds it) and into two products:
// dh += P w over the piece's rows, dw = P^T h over the tokens.  The products read w, h and, for dw, P across their rows, through LDS
// reads that turn them; no transposed copy is made.  dh is kept in fp32 over the pieces.  (The same step: 8 pieces of 288 us for P and 435 for both
// products, 1.26 PFLOP/s.)  P in 16 bits is a choice for its bytes.  Its roundings are half a step of the type each; the one at a token's target,
// the entry that outweighs the others together, is given back to both gradients.  Of the other entries' roundings as much remains in a sum as the sum keeps of the
// entries themselves: a relative error like that of rounding the result, which comes on top.
//
// The gradient of log probabilities and entropy (include/tagore_learn.h) is the same with another P; without dw, where the table stays as it is, dh's parts alone fill the card.
// (4096 tokens, 131 072 rows of 1024 bf16: 4 pieces of 283 us for P and 422 for both products.)
#include "tg_embed.h"
#include "tg_softmax.h"
#include "tg_tiles.h"

#include <type_traits>

#define XENT_BELOW (-1000.0f)

// x: rows of the table from v0 on, y: tokens.  parts: for every tile along x (BM rows of the table), (maximum, sum) of every token.
template <class E, int BM, int BN, int WM, int WN, int NB>
__global__ __launch_bounds__(64 * WM * WN) void xent_part_kernel(TileRows X, TileRows Y, int bytes, const void* __restrict__ targets, int targets64,
                                                                 float scale, int64_t v0, int64_t n_rows, uint32_t nx, uint32_t ny, uint32_t group,
                                                                 float2* __restrict__ parts, int64_t parts_pitch, float* __restrict__ at_target)
{
    typedef Tile<E, BM, BN, WM, WN, false, false, NB> T;
    __shared__ __align__(1024) char lds[T::LDS];
    // the tokens' targets among the tile's rows: asked for before the products, so that nothing waits for them behind
    __shared__ int s_target[BN];
    uint32_t tx, ty;
    tile_place(tile_of_block(blockIdx.x, nx * ny), nx, ny, group, &tx, &ty);
    const int64_t x0 = (int64_t)tx * BM, y0 = (int64_t)ty * BN;
    T t;
    t.start(X, Y, x0, y0, 0, bytes, lds);
    if (threadIdx.x < BN) {
        const int64_t y = y0 + threadIdx.x, target = y < Y.rows ? tg_row_of(targets, targets64, y, n_rows) - v0 - x0 : -1;
        s_target[threadIdx.x] = target >= 0 && target < BM ? (int)target : -1;
    }
    t.loop();
    // (the tile's memory is free: a pair for every token and wave along x)
    float2* const s_pair = reinterpret_cast<float2*>(lds) + (threadIdx.x >> 6) / WN * BN;
    static_assert(WM * BN * sizeof(float2) <= T::LDS, "the pairs' place");
    const int have = x0 + BM <= X.rows ? BM : (int)(X.rows - x0);
    const int none = (threadIdx.x >> 6) / WN * (T::HM * 16);        // the wave's first row: where the table ends before it there are no logits
    const float base = scale * XENT_LOG2E;
#pragma unroll
    for (int j = 0; j < T::FN; ++j) {
        const int64_t y = y0 + t.y_of(j);
        const int target = s_target[t.y_of(j)];
        float m = -__builtin_inff(), l = 0.0f;
#pragma unroll
        for (int i = 0; i < T::FM; ++i) {
            const int x = t.x_of(i);
            if ((unsigned)(target - x) < 4u) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (x + e == target) at_target[y] = t.acc[i][j][e] * scale;
            }
            if (x + 4 <= have) {
#pragma unroll
                for (int e = 0; e < 4; ++e) m = fmaxf(m, t.acc[i][j][e] * scale);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (x + e < have) m = fmaxf(m, t.acc[i][j][e] * scale);
            }
        }
        m = fmaxf(m, __shfl_xor(m, 16));
        m = fmaxf(m, __shfl_xor(m, 32));
        const bool near = xent_near(m, base) || have <= none;
        const float f = near ? base : 1.0f, b = near ? m * XENT_LOG2E : 0.0f;
        if (__builtin_expect(!__all(near), 0)) {           // (out of the way: code that is jumped over is fetched late)
#pragma unroll
            for (int i = 0; i < T::FM; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) t.acc[i][j][e] = near ? t.acc[i][j][e] : xent_far<true>(t.acc[i][j][e], scale, m);
        }
#pragma unroll
        for (int i = 0; i < T::FM; ++i) {
            const int x = t.x_of(i);
            if (x + 4 <= have) {
#pragma unroll
                for (int e = 0; e < 4; ++e) l += __builtin_amdgcn_exp2f(fmaf(t.acc[i][j][e], f, -b));
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (x + e < have) l += __builtin_amdgcn_exp2f(fmaf(t.acc[i][j][e], f, -b));
            }
        }
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (tg_lane() < 16) s_pair[t.y_of(j)] = make_float2(m, l);
    }
    __syncthreads();
    if (threadIdx.x < BN && y0 + threadIdx.x < Y.rows) {
        const float2* pair = reinterpret_cast<const float2*>(lds) + threadIdx.x;
        float m = pair[0].x, l = pair[0].y;
#pragma unroll
        for (int w = 1; w < WM; ++w) xent_join(m, l, pair[w * BN].x, pair[w * BN].y);
        parts[(int64_t)tx * parts_pitch + y0 + threadIdx.x] = make_float2(m, l);
    }
}

// TOK tokens a workgroup, 1024 / TOK lanes a token: lane j joins every so manieth part from j on, then the lanes are joined as a tree
template <int TOK>
__global__ __launch_bounds__(1024) void xent_join_kernel(const float2* __restrict__ parts, int64_t count, int64_t n, int64_t n_rows,
                                                         const void* __restrict__ targets, int targets64, const float* __restrict__ at_target,
                                                         float* __restrict__ loss, float* __restrict__ lse)
{
    constexpr int LANES = 1024 / TOK;
    __shared__ float s_m[LANES][TOK + 1], s_l[LANES][TOK + 1];
    const int c = threadIdx.x % TOK, j = threadIdx.x / TOK;
    for (int64_t y0 = (int64_t)blockIdx.x * TOK; y0 < n; y0 += (int64_t)gridDim.x * TOK) {
        const int64_t y = y0 + c;
        float m = -__builtin_inff(), l = 0.0f;
        if (y < n) {
            for (int64_t p0 = j; p0 < count; p0 += 4 * LANES) {
                float2 v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = p0 + i * LANES < count ? parts[(p0 + i * LANES) * n + y] : make_float2(-__builtin_inff(), 0.0f);
#pragma unroll
                for (int i = 0; i < 4; ++i) xent_join(m, l, v[i].x, v[i].y);
            }
        }
        s_m[j][c] = m;
        s_l[j][c] = l;
        __syncthreads();
#pragma unroll
        for (int h = LANES / 2; h >= 1; h >>= 1) {
            if (j < h) {
                xent_join(m, l, s_m[j + h][c], s_l[j + h][c]);
                s_m[j][c] = m;
                s_l[j][c] = l;
            }
            __syncthreads();
        }
        if (j == 0 && y < n) {
            const float v = m + logf(l);
            lse[y] = v;
            loss[y] = tg_row_of(targets, targets64, y, n_rows) >= 0 ? v - at_target[y] : 0.0f;
        }
    }
}

// ---- gradient

// With the entropy's gradient dH, P = scale (dloss ([v = target]'s part as without) - dH p (z - lse + H)): a token whose dH is not 0 has a part in the gradients
// without a target too.
__device__ inline bool xent_has_part(int64_t target, const float* __restrict__ dentropy, int64_t t) { return target >= 0 || (dentropy && dentropy[t] != 0.0f); }

// h without the rows of tokens that have no part (nothing of theirs, not even a NaN, may reach dw), packed for the tiles.  The last
// workgroup finds, for fp16, the power of two that P is kept under: P is at most |scale| max |dloss|, so that times c[0] it stays below 2^14, and
// values down to 2^-28 of the largest keep all their bits (bf16 and fp32 have the range as they are: c[0] = 1); c[1] = 1 / c[0].  The entropy's part is at most
// |scale dH| (H + 1 / e).
template <class E>
__global__ __launch_bounds__(256) void xent_prepare_kernel(const E* __restrict__ h, int64_t ld, int64_t n, int64_t n_rows, int d, int per,
                                                           const void* __restrict__ targets, int targets64, const float* __restrict__ dloss,
                                                           const float* __restrict__ entropy, const float* __restrict__ dentropy,
                                                           float scale, E* __restrict__ out, float* __restrict__ c)
{
    constexpr bool NARROW = __is_same(E, tg_f16);
    if (blockIdx.x < gridDim.x - 1) {
        const int64_t all = n * per;
        for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)(gridDim.x - 1) * 256) {
            typedef TgPiece<E> P;
            const int64_t r = i / per;
            const int at = (int)(i - r * per) * P::E;
            *reinterpret_cast<typename P::vec*>(out + r * per * P::E + at) = P::raw(h + r * ld + at, xent_has_part(tg_row_of(targets, targets64, r, n_rows), dentropy, r) ? d - at : 0);
        }
        return;
    }
    float top = 0.0f;
    if (NARROW) {
        __shared__ float s[4];
        for (int64_t t = threadIdx.x; t < n; t += 256) {
            float most = tg_row_of(targets, targets64, t, n_rows) >= 0 ? fabsf(dloss[t] * scale) : 0.0f;
            if (dentropy && dentropy[t] != 0.0f) most += fabsf(dentropy[t] * scale) * (fabsf(entropy[t]) + 0.375f);
            top = fmaxf(top, most);
        }
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) top = fmaxf(top, __shfl_xor(top, m));
        if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = top;
        __syncthreads();
        top = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
    }
    if (threadIdx.x) return;
    int up = 0;
    if (NARROW && top > 0.0f && top <= 3.4028234e38f) {
        int e;
        (void)frexpf(top, &e);                        // top in [2^(e-1), 2^e)
        up = 14 - e;
        up = up < -100 ? -100 : up > 100 ? 100 : up;
    }
    c[0] = ldexpf(1.0f, up);
    c[1] = ldexpf(1.0f, -up);
}

// P of a piece: x: rows v0.. of the table, y: tokens; p: n rows, `pitch` elements apart, zeros behind the piece's rows up to `width`.  lost: for types
// of 16 bits, what rounding took from P at the token's target, the entry that outweighs all others together.  ENTROPY: with the entropy's gradient,
// p (g + h t) for t = (z - lse) log2(e), g = scale (dloss - dH H) and h = -scale dH log(2), and at the target g less (scale dloss) beside it.
//
// The exponent t is one multiply-add, product base - b, whose terms are rounded: base = scale log2(e) by a step or two, and b, at the size of lse, by up to 2^-8.  So b is lse unit for unit = base / scale,
// which makes base's error one of the difference, and what rounding takes from b goes into the token's factors: 2^-rest, and h rest of g.  (fp32: P's norm is off by 9.2e-7
// at an lse of 52 and 4.9e-4 at 30 000 without it, by 3.6e-8 at either with it; exp(z - lse) in 32 bits 2.5e-8.  8192 tokens, 131 072 rows of 1024 bf16: the time is the same.)
template <class E, int BM, int BN, int WM, int WN, int NB, bool ENTROPY>
__global__ __launch_bounds__(64 * WM * WN) void xent_p_kernel(TileRows X, TileRows Y, int bytes, XentTokens tokens,
                                                              const float* __restrict__ c, float scale, double unit, int64_t v0, int64_t n_rows, uint32_t nx,
                                                              uint32_t ny, uint32_t group, E* __restrict__ p, int64_t pitch, int width, float* __restrict__ lost)
{
    typedef Tile<E, BM, BN, WM, WN, false, false, NB> T;
    __shared__ __align__(1024) char lds[T::LDS];
    // what a token's logits become P with: its target among the tile's rows, its factor and its lse.  A token without a target has no part in
    // anything, whatever its logits are.
    struct Token { int hit, there; float g, b; };                // there: 0 without a part, 1, or 2 with an lse that is not near, which b then is as it is
    struct More { float h, less; };                              // without the entropy's gradient: h: what the rest makes of a power
    __shared__ Token s_token[BN];
    __shared__ More s_more[BN];
    const float up = c[0];
    uint32_t tx, ty;
    tile_place(tile_of_block(blockIdx.x, nx * ny), nx, ny, group, &tx, &ty);
    const int64_t x0 = (int64_t)tx * BM, y0 = (int64_t)ty * BN;
    T t;
    t.start(X, Y, x0, y0, 0, bytes, lds);
    if (threadIdx.x < BN) {
        // (all of it is asked for at once: one way to memory, not four)
        const int64_t y = y0 + threadIdx.x, at = y < Y.rows ? y : 0;
        const float lse = tokens.lse[at], dloss = tokens.dloss[at], dentropy = ENTROPY ? tokens.dentropy[at] : 0.0f, entropy = ENTROPY ? tokens.entropy[at] : 0.0f;
        const int64_t target = y < Y.rows ? tg_row_of(tokens.targets, tokens.targets64, at, n_rows) : -1, hit = target - v0 - x0;
        Token k{target >= 0 && hit >= 0 && hit < BM ? (int)hit : -1, 0, 0.0f, 0.0f};
        More more{ENTROPY ? 0.0f : 1.0f, 0.0f};
        if (y < Y.rows && (target >= 0 || dentropy != 0.0f)) {
            if (target >= 0) k.g = more.less = dloss * tokens.gain * scale * up;
            if (ENTROPY && dentropy != 0.0f) {
                const float dh = dentropy * scale * up;
                k.g = fmaf(-dh, entropy, k.g);
                more.h = dh * -0.6931471805599453f;
            }
            const bool near = xent_near(lse, scale * XENT_LOG2E);
            k.there = near ? 1 : 2;
            k.b = lse;
            if (near) {
                const double b = (double)lse * unit;
                k.b = (float)b;
                const float rest = (float)(b - (double)k.b), by = __builtin_amdgcn_exp2f(-rest);
                k.g = (ENTROPY ? fmaf(-more.h, rest, k.g) : k.g) * by;
                more.h = ENTROPY ? more.h * by : by;
            }
        }
        s_token[threadIdx.x] = k;
        s_more[threadIdx.x] = more;
    }
    t.loop();
    const int have = x0 + BM <= X.rows ? BM : (int)(X.rows - x0), room = x0 + BM <= width ? BM : (int)(width - x0);
    // A lane has four neighbours of 16 rows at a time; the tile goes through its memory, which is free, to be stored as whole rows.  Piece c of row r lies at
    // place c ^ (r & SWAP): the lanes that write one column of pieces at a time are in different banks.
    constexpr int W = 16 / (int)sizeof(E), PIECES = BM / W, SWAP = PIECES < 16 ? PIECES - 1 : 15;
    static_assert(BM * BN * sizeof(E) <= T::LDS && (PIECES & (PIECES - 1)) == 0, "the tile's place");
    typedef E four __attribute__((ext_vector_type(4)));
    typedef E vec __attribute__((ext_vector_type(W)));
    // (r & SWAP, whatever j)
    int swap = threadIdx.x & SWAP;
    float base = scale;
    asm volatile("" : "+v"(base));
    base *= XENT_LOG2E;
#pragma unroll
    for (int j = 0; j < T::FN; ++j) {
        // (nothing of this is made out in front of the products, in whose loop no register is free)
        asm volatile("" : "+v"(swap) : : "memory");
#pragma unroll
        for (int i = 0; i < T::FM; ++i) asm volatile("" : "+v"(t.acc[i][j]));
        const int r = t.y_of(j);
        const Token k = s_token[r];
        More more{0.0f, 0.0f};
        if (ENTROPY) more = s_more[r];
        // what the power of an exponent is multiplied with (below XENT_BELOW the power is 0, and the entropy's part with it)
        const auto by = [&](float u) { return ENTROPY ? fmaf(more.h, fmaxf(u, XENT_BELOW), k.g) : k.g; };
        const bool near = k.there < 2;
        const float f = near ? base : 1.0f, b = near ? k.b : 0.0f;
        if (__builtin_expect(!__all(near), 0)) {           // (out of the way: code that is jumped over is fetched late)
#pragma unroll
            for (int i = 0; i < T::FM; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) t.acc[i][j][e] = near ? t.acc[i][j][e] : xent_far<false>(t.acc[i][j][e], scale, k.b);
        }
        char* const row = lds + r * (PIECES * 16);
#pragma unroll
        for (int i = 0; i < T::FM; ++i) {
            const int x = t.x_of(i);
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float u = fmaf(t.acc[i][j][e], f, -b);
                v[e] = __builtin_amdgcn_exp2f(u) * by(u);
            }
            if ((unsigned)(k.hit - x) < 4u) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (x + e == k.hit) {
                        const float u = fmaf(t.acc[i][j][e], f, -b);
                        const More at = s_more[r];
                        v[e] = ENTROPY ? fmaf(__builtin_amdgcn_exp2f(u), by(u), -at.less) : fmaf(__builtin_amdgcn_exp2f(u), at.h, -1.0f) * at.less;
                        if (sizeof(E) == 2) lost[y0 + r] = v[e] - (float)(E)v[e];
                    }
            }
            if (!k.there || x + 4 > have) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (!k.there || x + e >= have) v[e] = 0.0f;
            }
            *reinterpret_cast<four*>(row + ((x / W) ^ swap) * 16 + x % W * (int)sizeof(E)) = four{(E)v[0], (E)v[1], (E)v[2], (E)v[3]};
        }
    }
    __syncthreads();
    // (a row's room is whole pieces)
    constexpr int THREADS = 64 * WM * WN;
#pragma unroll 4
    for (int at = threadIdx.x; at < BN * PIECES; at += THREADS) {
        const int r = at / PIECES, piece = at % PIECES;
        if (y0 + r < Y.rows && piece * W < room)
            *reinterpret_cast<vec*>(p + (y0 + r) * pitch + x0 + piece * W) = *reinterpret_cast<const vec*>(lds + (r * PIECES + (piece ^ (r & SWAP))) * 16);
    }
}

// The two products of a piece in one launch, the first workgroups dh's (they fill the card in whole rounds together where each does not).
//
// dh: x: columns of w (turned), y: tokens, over the rows of the piece, in `splits` parts.  sums: splits x n x d, added to but for the first
// piece; or, where there is one piece and one part, dh itself.
// dw: x: columns of h (turned), y: columns of P, rows of the piece (turned), over the tokens.
struct XentProducts {
    TileRows w, h, p;
    int64_t v0, rows, n_rows;       // the piece's first row of the table, its rows, the table's
    int d;
    int p_bytes, each, h_bytes;     // contractions: of dh, of one part of it, of dw
    uint32_t dh_x, dh_y, dw_x, dw_y;
    int splits, first, direct;
    const void* targets;
    int targets64;
    const float* dentropy;          // or null
    const void* table;              // the caller's w
    int64_t ld_table;
    const float *c, *lost;
    float* sums;
    void *dh, *dw;
};
// four neighbours (or one) of row y of dh, with what rounding took from P at the target
template <class E, int W = 4>
__device__ inline void xent_put_dh(const XentProducts& a, int64_t y, int x, float* v)
{
    const int64_t target = tg_row_of(a.targets, a.targets64, y, a.n_rows);
    const float l = sizeof(E) == 2 && target >= 0 ? a.lost[y] : 0.0f;
    const E* row = (const E*)a.table + (target < 0 ? 0 : target) * a.ld_table + x;
#pragma unroll
    for (int e = 0; e < W; ++e) {
        if (sizeof(E) == 2 && x + e < a.d) v[e] = fmaf(l, (float)row[e], v[e]);
        v[e] = xent_has_part(target, a.dentropy, y) ? v[e] * a.c[1] : 0.0f;
    }
    if (W == 1) ((E*)a.dh)[y * a.d + x] = (E)v[0];
    else tile_put((E*)a.dh + y * a.d + x, v, a.d - x);
}
// What rounding took from P at the targets among a tile's rows, given back to dw's tile of 16-bit values: a row that is the target of few tokens is mostly
// theirs, and their roundings are whole in it, whatever the number of tokens.  The tokens are looked through for targets among the rows; those found are
// listed in their order, and 128 at a time (all is asked for at once) they are up to four more steps of the contraction, of their rows of h and of a matrix that
// holds a token's lost part (rounded to the type: an error's error) in its target's row alone.  It is a chain of loads and barriers that nothing of the
// tile overlaps: 8192 tokens, 131 072 rows of 1024, bf16: 7.53 ms there and back without it, 7.57 with it; 500, 30 000 of 512: 108 and 116 us; 900, 5000 of 700: 77 and 82.
template <class E, int B, int THREADS>
struct XentGiveBack {
    static constexpr int WAVES = THREADS / 64, EACH = 16, CHUNK = EACH * THREADS;        // tokens that are looked through at a time
    struct Lost { int row; float v; };
    struct Memory {
        Lost lost[128];
        uint32_t counts[WAVES];
        uint16_t mine[THREADS];              // (no register is free in the products' loop)
        uint16_t list[CHUNK];                // token, from the chunk's first on
    };
    static_assert(CHUNK <= 1 << 16, "16 bits a token");
    Memory& m;
    const XentProducts& a;
    const int64_t v0;                        // the tile's first row of the table, and its rows
    const int rows;
    __device__ inline XentGiveBack(Memory& m, const XentProducts& a, int64_t y0)
        : m(m), a(a), v0(a.v0 + y0), rows(a.rows - y0 < B ? (int)(a.rows - y0) : B) {}

    __device__ inline int row_of(int64_t token) const
    {
        const int64_t r = tg_row_of(a.targets, a.targets64, token, a.n_rows) - v0;
        return r >= 0 && r < rows ? (int)r : -1;
    }
    // a wave's tokens of the chunk from c0 on, 64 at a time: an equal part each
    __device__ inline int all_of(int64_t c0) const { return a.p.rows - c0 < CHUNK ? (int)(a.p.rows - c0) : CHUNK; }
    __device__ inline int first_of(int64_t c0) const
    {
        return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * ((all_of(c0) + THREADS - 1) / THREADS * 64) + tg_lane();
    }
    // which of the lane's tokens have a target here, and how many each wave found
    __device__ inline void look(int64_t c0)
    {
        const int all = all_of(c0), turns = (all + THREADS - 1) / THREADS, first = first_of(c0);
        // (asked for at once; a place behind the end is the first token's, and no hit)
        int64_t target[EACH];
        const auto ask = [&](auto* targets) {
#pragma unroll
            for (int k = 0; k < EACH; ++k)
                if (k < turns) target[k] = targets[c0 + (first + k * 64 < all ? first + k * 64 : 0)];
        };
        if (a.targets64) ask(reinterpret_cast<const int64_t*>(a.targets));
        else ask(reinterpret_cast<const int32_t*>(a.targets));
        uint32_t mine = 0, count = 0;
#pragma unroll
        for (int k = 0; k < EACH; ++k)
            if (k < turns) {
                const bool hit = first + k * 64 < all && target[k] >= v0 && target[k] < v0 + rows;
                mine |= hit ? 1u << k : 0u;
                count += __popcll(__ballot(hit));
            }
        m.mine[threadIdx.x] = (uint16_t)mine;
        if (tg_lane() == 0) m.counts[threadIdx.x >> 6] = count;
    }
    // behind a barrier: their list, which all waves have behind the next one, and its length
    __device__ inline uint32_t list(int64_t c0)
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), first = first_of(c0);
        uint32_t at = 0, found = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            at += w < wave ? m.counts[w] : 0;
            found += m.counts[w];
        }
        if (m.counts[wave]) {
            const uint32_t mine = m.mine[threadIdx.x];
#pragma unroll
            for (int k = 0; k < EACH; ++k) {
                const bool hit = mine >> k & 1;
                const u64 hits = __ballot(hit);
                if (hit) m.list[at + __popcll(hits & tg_lanemask_lt())] = (uint16_t)(first + k * 64);
                at += __popcll(hits);
            }
        }
        return found;
    }
    // Behind `look` for the first chunk, and the products.  lds: the tile's memory, which no wave reads any more.
    template <class T>
    __device__ inline void run(T& t, int64_t x0, char* lds)
    {
#ifdef __HIP_DEVICE_COMPILE__
        typedef typename T::SX S;
        typedef E vec __attribute__((ext_vector_type(8)));
        static_assert(4 * S::BYTES <= T::LDS && S::DEPTH == 64, "two buffers of 64 rows of h, as the tile reads them");
        const int lane = tg_lane(), q = lane >> 4;
        for (int64_t c0 = 0;;) {
            const uint32_t found = list(c0);
            if (found) __syncthreads();
            for (uint32_t s0 = 0; s0 < found; s0 += 128) {
                const int have = found - s0 < 128 ? (int)(found - s0) : 128, steps = (have + 31) / 32;
                constexpr int PIECES = B / 8, TURNS = 128 * PIECES / THREADS;     // pieces of a row of h, 8 columns each; half of them a unit's
                static_assert(THREADS >= 128 && THREADS % PIECES == 0, "a lane a token, whole rows a turn");
                // (everything is asked for before anything is waited for: places behind the list's end are its last token's, and become zeros)
                const int r0 = threadIdx.x / PIECES, c = threadIdx.x % PIECES, column = (int)x0 * 2 + c * 16;
                int64_t token[TURNS];
#pragma unroll
                for (int k = 0; k < TURNS; ++k) {
                    const int r = k * (THREADS / PIECES) + r0;
                    token[k] = c0 + m.list[s0 + (r < have ? r : have - 1)];
                }
                const int mine = (int)threadIdx.x < have ? threadIdx.x : have - 1;
                const int64_t own = c0 + m.list[s0 + mine];
                const float rounded = a.lost[own];
                vec v[TURNS];
#pragma unroll
                for (int k = 0; k < TURNS; ++k)
                    if (k * (THREADS / PIECES) < steps * 32)
                        v[k] = *reinterpret_cast<const vec*>(a.h.p + token[k] * a.h.pitch + (column < (int)a.h.width ? column : 0));
                const int row = row_of(own);
                if (threadIdx.x < 128) m.lost[threadIdx.x] = Lost{(int)threadIdx.x < have ? row : -1, rounded};
#pragma unroll
                for (int k = 0; k < TURNS; ++k) {
                    const int r = k * (THREADS / PIECES) + r0;
                    if (k * (THREADS / PIECES) < steps * 32)
                        *reinterpret_cast<vec*>(lds + ((r >> 6) * 2 + c / (PIECES / 2)) * S::BYTES + (r & 63) * S::ROW + ((c % (PIECES / 2)) ^ S::exchange(r)) * 16) =
                            r < have && column < (int)a.h.width ? v[k] : vec{};
                }
                __syncthreads();
                for (int g = 0; g < steps; ++g) {
                    Lost l[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) l[e] = m.lost[g * 32 + q * 8 + e];
                    tg_i32x4 one[T::FN];
#pragma unroll
                    for (int j = 0; j < T::FN; ++j) {
                        const int y = t.y_of(j);
                        vec o;
#pragma unroll
                        for (int e = 0; e < 8; ++e) o[e] = l[e].row == y ? (E)l[e].v : (E)0.0f;
                        one[j] = __builtin_bit_cast(tg_i32x4, o);
                    }
#pragma unroll
                    for (int i = 0; i < T::FM; ++i) {
                        const tg_i32x4 x = t.r.sx.read(lds + ((g >> 1) * 2 + i / T::HM) * S::BYTES, t.r.wm * (T::HM * 16), i % T::HM, g & 1, lane);
#pragma unroll
                        for (int j = 0; j < T::FN; ++j) t.acc[i][j] = TileMul<E>::mul(x, one[j], t.acc[i][j]);
                    }
                }
                __syncthreads();
            }
            c0 += CHUNK;
            if (c0 >= a.p.rows) return;
            __syncthreads();                        // (all have the counts)
            look(c0);
            __syncthreads();
        }
#endif
    }
};

template <class E, int B, int WM, int WN, int NB>
__global__ __launch_bounds__(64 * WM * WN) void xent_products_kernel(XentProducts a)
{
    typedef Tile<E, B, B, WM, WN, true, false, NB> TH;
    typedef Tile<E, B, B, WM, WN, true, true, NB> TW;
    static_assert(TH::LDS == TW::LDS, "one memory for both");
    __shared__ __align__(1024) char lds[TH::LDS];
    const uint32_t dh_all = a.dh_x * a.dh_y * a.splits;
    uint32_t tx, ty;
    if (blockIdx.x < dh_all) {
        const uint32_t b = tile_of_block(blockIdx.x, dh_all);
        const uint32_t s = (uint32_t)__builtin_amdgcn_readfirstlane((int)(b / (a.dh_x * a.dh_y)));
        tile_place(b - s * (a.dh_x * a.dh_y), a.dh_x, a.dh_y, 1, &tx, &ty);
        const int64_t x0 = (int64_t)tx * B, y0 = (int64_t)ty * B;
        const int k0 = (int)s * a.each, k1 = k0 + a.each < a.p_bytes ? k0 + a.each : a.p_bytes;
        TH t;
        t.run(a.w, a.p, x0, y0, k0, k1, lds);
#pragma unroll
        for (int j = 0; j < TH::FN; ++j) {
            const int64_t y = y0 + t.y_of(j);
            if (y >= a.p.rows) continue;
#pragma unroll
            for (int i = 0; i < TH::FM; ++i) {
                const int x = (int)x0 + t.x_of(i);
                if (x >= a.d) continue;
                float v[4];
                float* o = a.sums + ((int64_t)s * a.p.rows + y) * a.d + x;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = t.acc[i][j][e] + (!a.first && x + e < a.d ? o[e] : 0.0f);
                if (a.direct) xent_put_dh<E>(a, y, x, v);
                else tile_put(o, v, a.d - x);
            }
        }
        return;
    }
    tile_place(tile_of_block(blockIdx.x - dh_all, a.dw_x * a.dw_y), a.dw_x, a.dw_y, 1, &tx, &ty);
    const int64_t x0 = (int64_t)tx * B, y0 = (int64_t)ty * B;
    TW t;
    if constexpr (sizeof(E) == 2) {
        typedef XentGiveBack<E, B, 64 * WM * WN> GiveBack;
        __shared__ typename GiveBack::Memory memory;
        GiveBack back(memory, a, y0);
        back.look(0);
        t.run(a.h, a.p, x0, y0, 0, a.h_bytes, lds);
        back.run(t, x0, lds);
    } else t.run(a.h, a.p, x0, y0, 0, a.h_bytes, lds);
    const float down = a.c[1];
#pragma unroll
    for (int j = 0; j < TW::FN; ++j) {
        const int64_t y = y0 + t.y_of(j);
        if (y >= a.rows) continue;
#pragma unroll
        for (int i = 0; i < TW::FM; ++i) {
            const int x = (int)x0 + t.x_of(i);
            if (x >= a.d) continue;
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = t.acc[i][j][e] * down;
            tile_put((E*)a.dw + y * a.d + x, v, a.d - x);
        }
    }
}
// dh out of its parts: four neighbours a lane, WHOLE where rows are whole fours; or one (W = 1) where there are few outputs and rows are not: a question for what is left of a
// row would stand between the loads (301 tokens of 50 fp32 values, 64 parts: 11.5 us with it, 6.2; 2000 of 701, 2 us more in ones).
template <class E, int W, bool WHOLE>
__global__ __launch_bounds__(256) void xent_dh_kernel(XentProducts a, int pieces)
{
    typedef float vec __attribute__((ext_vector_type(W)));
    const int64_t n = a.p.rows, all = n * pieces, each = n * a.d;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < all; i += (int64_t)gridDim.x * blockDim.x) {
        const int64_t y = i / pieces;
        const int at = (int)(i - y * pieces) * W;
        const float* p = a.sums + y * a.d + at;
        TgPiece<float> sum;
        if constexpr (WHOLE) {
            vec x = *reinterpret_cast<const vec*>(p);
#pragma unroll 8
            for (int s = 1; s < a.splits; ++s) x += *reinterpret_cast<const vec*>(p + s * each);
#pragma unroll
            for (int e = 0; e < W; ++e) sum.v[e] = x[e];
        } else {
            sum.load(p, a.d - at);
#pragma unroll 8
            for (int s = 1; s < a.splits; ++s) {
                TgPiece<float> q;
                q.load(p + s * each, a.d - at);
#pragma unroll
                for (int e = 0; e < 4; ++e) sum.v[e] += q.v[e];
            }
        }
        xent_put_dh<E, W>(a, y, at, sum.v);
    }
}

// ---- workspaces and launches
struct XentRows {
    TileRows h, w;
    void *ph, *pw;            // copies, or null
};
static void xent_rows(XentRows* r, TgCarve* c, const void* h, int64_t ld_h, const void* w, int64_t ld_w, int64_t n, int64_t n_rows, int d, int e,
                      bool ready_h, bool ready_w)
{
    const uint32_t pitch = tile_pitch(d, e);
    r->ph = ready_h ? nullptr : c->take<char>((size_t)n * pitch);
    r->pw = ready_w ? nullptr : c->take<char>((size_t)n_rows * pitch);
    r->h = ready_h ? TileRows{(const char*)h, n, (uint32_t)(ld_h * e), pitch} : TileRows{(const char*)r->ph, n, pitch, pitch};
    r->w = ready_w ? TileRows{(const char*)w, n_rows, (uint32_t)(ld_w * e), pitch} : TileRows{(const char*)r->pw, n_rows, pitch, pitch};
}

// The tile of the logits: 256 x 256 where that leaves every CU one, smaller ones for fewer tokens.  fp32, whose products take sixteen times as long
// a byte, is fed by the smallest, 64 x 64, of which a CU holds four that wait for each other's loads and epilogues (1003 tokens, 37 511 rows of 96, there and back:
// 398 us in tiles of 128 x 128, 359 in these; 2048 tokens, 8000 rows of 1500: 1502 and 1444).
#define XENT_STRETCH 64         // rows of the table that leave one (maximum, sum) at least (BM)

size_t tg_xent_space(int64_t n, int64_t n_rows, int d, int dtype, int aligned)
{
    if (n == 0) return 0;
    const int e = (int)tg_type_bytes(dtype);
    TgCarve c{nullptr, 0};
    XentRows r;
    const bool whole = (d * e & 15) == 0;
    xent_rows(&r, &c, nullptr, d, nullptr, d, n, n_rows, d, e, whole && (aligned == 1 || aligned == 3), whole && (aligned == 1 || aligned == 2));
    c.take<float2>((size_t)((n_rows + XENT_STRETCH - 1) / XENT_STRETCH + 8) * n);
    c.take<float>(n);
    return c.used;
}

// Logits of so few tiles that each has a CU of its own: what counts is then how long a stage is on its way, and tiles of 64 x 64 (or of 32 tokens)
// have four of them in flight.
static bool xent_small(int64_t rows, int64_t n) { return ((rows + 127) / 128) * ((n + 127) / 128) <= 128; }
template <class E, int BM, int BN, int WM, int WN, int NB = 2>
static int64_t launch_parts(const TileRows& X, const TileRows& Y, int bytes, const void* targets, int targets64, float scale, float2* parts,
                            float* at_target, hipStream_t s)
{
    const int64_t nx = (X.rows + BM - 1) / BM;
    // as many tiles along the table as a launch's work-items allow (all of them up to 2^29 rows), then as many tokens
    constexpr int64_t TILES = TILE_LAUNCH_ITEMS / (64 * WM * WN);
    for (int64_t t0 = 0; t0 < nx; t0 += TILES) {
        const int64_t tiles = nx - t0 < TILES ? nx - t0 : TILES, v0 = t0 * BM, most = TILES / tiles * BN;
        const TileRows table{X.p + v0 * X.pitch, X.rows - v0 < tiles * BM ? X.rows - v0 : tiles * BM, X.pitch, X.width};
        for (int64_t y0 = 0; y0 < Y.rows; y0 += most) {
            const int64_t rows = Y.rows - y0 < most ? Y.rows - y0 : most;
            const uint32_t ny = (uint32_t)((rows + BN - 1) / BN);
            const TileRows part{Y.p + y0 * Y.pitch, rows, Y.pitch, Y.width};
            hipLaunchKernelGGL((xent_part_kernel<E, BM, BN, WM, WN, NB>), dim3((unsigned)(tiles * ny)), dim3(64 * WM * WN), 0, s, table, part, bytes,
                               (const char*)targets + y0 * (targets64 ? 8 : 4), targets64, scale, v0, X.rows, (uint32_t)tiles, ny, 8u,
                               parts + t0 * Y.rows + y0, Y.rows, at_target + y0);
        }
    }
    return nx;
}

void tg_launch_xent(const void* h, int64_t ld_h, const void* w, int64_t ld_w, int dtype, int64_t n, int64_t n_rows, int d, const void* targets,
                    int targets64, float scale, float* loss, float* lse, void* space, hipStream_t s)
{
    const int e = (int)tg_type_bytes(dtype);
    TgCarve c{(char*)space, 0};
    XentRows r;
    const bool rh = tile_ready(h, ld_h, d, e), rw = tile_ready(w, ld_w, d, e);
    xent_rows(&r, &c, h, ld_h, w, ld_w, n, n_rows, d, e, rh, rw);
    if (!rh) tg_launch_pack(h, ld_h, n, d, e, r.ph, s);
    if (!rw) tg_launch_pack(w, ld_w, n_rows, d, e, r.pw, s);
    float2* parts = c.take<float2>((size_t)((n_rows + XENT_STRETCH - 1) / XENT_STRETCH + 8) * n);
    float* at = c.take<float>(n);
    int64_t count = 0;
    TG_WITH_TYPE(dtype, E, {
        const bool small = xent_small(n_rows, n);
        if (n <= 32 && small) count = launch_parts<E, 128, 32, 4, 1, 4>(r.w, r.h, r.w.width, targets, targets64, scale, parts, at, s);
        else if (n <= 32) count = launch_parts<E, 128, 32, 4, 1>(r.w, r.h, r.w.width, targets, targets64, scale, parts, at, s);
        else if (small) count = launch_parts<E, 64, 64, 2, 2, 4>(r.w, r.h, r.w.width, targets, targets64, scale, parts, at, s);
        else if (n <= 64) count = launch_parts<E, 128, 64, 4, 1>(r.w, r.h, r.w.width, targets, targets64, scale, parts, at, s);
        else {
            bool wide = false;
            if constexpr (sizeof(E) == 2) {
                wide = ((n_rows + 255) / 256) * ((n + 255) / 256) >= 200;
                if (wide) count = launch_parts<E, 256, 256, 2, 4>(r.w, r.h, r.w.width, targets, targets64, scale, parts, at, s);
            }
            if constexpr (sizeof(E) == 4) count = launch_parts<E, 64, 64, 2, 2>(r.w, r.h, r.w.width, targets, targets64, scale, parts, at, s);
            else if (!wide) count = launch_parts<E, 128, 128, 2, 2>(r.w, r.h, r.w.width, targets, targets64, scale, parts, at, s);
        }
    });
    // few tokens: more lanes each, and more workgroups
    const int tok = n <= 1024 ? 4 : 16;
    const int64_t wgs = (n + tok - 1) / tok;
    const dim3 grid((unsigned)(wgs < 65536 ? wgs : 65536));
    if (tok == 4) hipLaunchKernelGGL(xent_join_kernel<4>, grid, dim3(1024), 0, s, parts, count, n, n_rows, targets, targets64, at, loss, lse);
    else hipLaunchKernelGGL(xent_join_kernel<16>, grid, dim3(1024), 0, s, parts, count, n, n_rows, targets, targets64, at, loss, lse);
}

#define XENT_PIECE_BYTES (256ll << 20)     // of P, where the workspace has them
#define XENT_PAD 256
#define XENT_LEAST_ROWS 256                // of a piece
#define XENT_MOST_ROWS (1ll << 20)         // (256 rows of P stay within a buffer of 32 bits)

struct XentGrad {
    int64_t piece;        // rows of the table at a time, a multiple of 256 unless it is all of them
    int side;             // products in tiles of 256 x 256, 128 x 128 or 64 x 64
    bool few;             // tiles: 64 x 64, with four stages in flight
    int splits;           // of dh's contraction
    bool direct;          // one piece, one part: dh is written at once
};
static int64_t round_up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }
// bytes between the rows of P.  Its tiles are stored sixteen rows at a time: at a distance of a power of two those would meet in one channel of
// the caches.
static uint32_t xent_pitch(int64_t rows, int e) { return (uint32_t)round_up(rows * e, 16) + XENT_PAD; }
static void xent_splits(XentGrad* g, int64_t n, int64_t n_rows, int d, int e, bool table)
{
    // both products take tiles of 256 x 256, of which a CU holds one, where those are enough; else of 128 x 128, of which it holds two, in fp32 of
    // 64 x 64, of which it holds four; and of 64 x 64, with four stages in flight, where each of 128 x 128 would have a CU of its own
    const auto tiles = [](int64_t x, int64_t y, int64_t side) { return ((x + side - 1) / side) * ((y + side - 1) / side); };
    // Without dw, dh's parts alone are to fill the card: the tiles are those that as many parts as the contraction is long enough for would make.
    const int64_t all_stages = (g->piece * e + TILE_BYTES - 1) / TILE_BYTES;
    const auto parts = [&](int64_t side) { return tiles(n, d, side) * (all_stages >= 64 * 16 ? 64 : all_stages >= 16 ? all_stages / 16 : 1); };
    g->few = table ? tiles(n, d, 128) + tiles(g->piece, d, 128) <= 128 : n <= 64 || parts(128) <= 128;
    g->side = e == 2 && n > 128 && d > 128 && (table ? tiles(g->piece, d, 256) : parts(256)) >= 200 ? 256 : g->few || e == 4 ? 64 : 128;
    // dh in as many parts as fill the card, each with sixteen stages of the contraction or more; where dw, beside it, has fewer, with as many as
    // that, but four, up to 32 parts whose bytes are half of the table's (there and back, bf16: 7 tokens, 6938 rows of 688: 39.8 us with sixteen, 37.2;
    // 900 tokens, 5000 rows of 700: 77.7 and 75.2)
    const int64_t fill = g->side == 256 ? 256 : g->few || g->side == 128 ? 512 : 1024, dw_stages = table ? (n * e + TILE_BYTES - 1) / TILE_BYTES : 0;
    const int64_t least = g->few || dw_stages < 4 ? 4 : dw_stages < 16 ? dw_stages : 16, light = g->piece * e / (8 * n);
    const int64_t dh = tiles(n, d, g->side), stages = (g->piece * e + TILE_BYTES - 1) / TILE_BYTES;
    int64_t s = (fill + dh - 1) / dh;
    const int64_t long_parts = stages / 16;
    if (s > long_parts) {
        int64_t more = stages / least;
        if (!g->few && more > light) more = light;
        if (!g->few && more > 32) more = 32;
        if (more < long_parts) more = long_parts;
        if (s > more) s = more;
    }
    g->splits = (int)(s < 1 ? 1 : s > 64 ? 64 : s);
    g->direct = g->splits == 1 && g->piece >= n_rows;
}
static size_t carve_xent_grad(XentRows* r, TgCarve* c, const void* h, int64_t ld_h, const void* w, int64_t ld_w, int64_t n, int64_t n_rows, int d,
                              int e, bool ready_w, XentGrad g, float** consts, char** p, float** sums, float** lost)
{
    xent_rows(r, c, h, ld_h, w, ld_w, n, n_rows, d, e, false, ready_w);       // (h is always copied: see xent_prepare_kernel)
    *consts = c->take<float>(2);
    *lost = c->take<float>(e == 2 ? n : 0);
    *sums = c->take<float>(g.direct ? 0 : (size_t)g.splits * n * d);
    *p = c->take<char>((size_t)n * xent_pitch(g.piece, e));
    return c->used;
}
static XentGrad xent_grad_shape(int64_t n, int64_t n_rows, int d, int e, int64_t p_bytes, bool table)
{
    XentGrad g;
    g.piece = p_bytes / ((n > 0 ? n : 1) * e) / 256 * 256;
    if (g.piece < XENT_LEAST_ROWS) g.piece = XENT_LEAST_ROWS;
    if (g.piece > XENT_MOST_ROWS) g.piece = XENT_MOST_ROWS;
    if (g.piece >= n_rows) g.piece = n_rows;
    else {
        // equal pieces
        const int64_t count = (n_rows + g.piece - 1) / g.piece;
        g.piece = round_up((n_rows + count - 1) / count, 256);
    }
    xent_splits(&g, n, n_rows, d, e, table);
    return g;
}
static size_t xent_grad_bytes(int64_t n, int64_t n_rows, int d, int e, bool ready, int64_t p_bytes, bool table)
{
    TgCarve c{nullptr, 0};
    XentRows r;
    float *k, *sums, *lost;
    char* p;
    return carve_xent_grad(&r, &c, nullptr, d, nullptr, d, n, n_rows, d, e, ready && (d * e & 15) == 0, xent_grad_shape(n, n_rows, d, e, p_bytes, table), &k, &p, &sums, &lost);
}
size_t tg_xent_grad_space(int64_t n, int64_t n_rows, int d, int dtype, int aligned, bool least, bool table)
{
    if (n == 0) return 0;
    const bool ready = aligned == 1 || aligned == 2;           // (h is always copied)
    const size_t asked = xent_grad_bytes(n, n_rows, d, (int)tg_type_bytes(dtype), ready, XENT_PIECE_BYTES, table);
    if (!least) return asked;
    // (one piece can do with less than many: dh then needs no sums)
    const size_t pieces = xent_grad_bytes(n, n_rows, d, (int)tg_type_bytes(dtype), ready, 0, table);
    return pieces < asked ? pieces : asked;
}

template <class E>
static void launch_xent_grad(const XentRows& r, const XentGrad& g, const void* h, int64_t ld_h, const void* w, int64_t ld_w, int64_t n, int64_t n_rows,
                             int d, const XentTokens& t, float scale, float* consts, char* p, float* sums, float* lost, E* dh, E* dw, hipStream_t s)
{
    const int e = (int)sizeof(E), per = (int)(r.h.pitch / 16);
    // (base as the kernels make it; one below the normal numbers is off by more than a step or two, of logits that are all next to 0)
    const double unit = fabsf(scale) >= 0x1p-126f ? (double)(scale * XENT_LOG2E) / (double)scale : 1.4426950408889634;
    const int64_t wgs = (n * per + 255) / 256;
    hipLaunchKernelGGL(xent_prepare_kernel<E>, dim3((unsigned)(wgs < 16384 ? wgs : 16384) + 1), dim3(256), 0, s, (const E*)h, ld_h, n, n_rows, d, per,
                       t.targets, t.targets64, t.dloss, t.entropy, t.dentropy, scale, (E*)r.ph, consts);
    XentProducts a;
    a.h = r.h;
    a.n_rows = n_rows;
    a.d = d;
    a.h_bytes = (int)(n * e);
    a.splits = g.splits;
    a.direct = g.direct ? 1 : 0;
    a.targets = t.targets;
    a.targets64 = t.targets64;
    a.dentropy = t.dentropy;
    a.table = w;
    a.ld_table = ld_w;
    a.c = consts;
    a.lost = lost;
    a.sums = sums;
    a.dh = dh;
    const int side = g.side;
    const auto over = [](int64_t x, int64_t by) { return (uint32_t)((x + by - 1) / by); };
    a.dh_x = a.dw_x = over(d, side);
    a.dh_y = over(n, side);
    for (int64_t v0 = 0; v0 < n_rows; v0 += g.piece) {
        const int64_t rows = n_rows - v0 < g.piece ? n_rows - v0 : g.piece;
        const uint32_t pitch = xent_pitch(rows, e);
        a.w = TileRows{r.w.p + v0 * r.w.pitch, rows, r.w.pitch, r.w.width};
        const uint32_t width = (uint32_t)round_up(rows * e, 16);
        a.p = TileRows{p, n, pitch, width};
        const auto logits = [&](auto kernel, int bm, int bn, int threads) {
            const uint32_t nx = over(rows, bm), ny = over(n, bn);
            hipLaunchKernelGGL(kernel, dim3(nx * ny), dim3(threads), 0, s, a.w, r.h, (int)a.w.width, t, (const float*)consts, scale, unit, v0, n_rows, nx, ny, 8u, (E*)p, (int64_t)(pitch / e),
                               (int)(width / e), lost);
        };
        const auto all_logits = [&](auto with) {
            constexpr bool ENTROPY = decltype(with)::value;
            if (xent_small(rows, n)) logits(xent_p_kernel<E, 64, 64, 2, 2, 4, ENTROPY>, 64, 64, 256);
            else if (n <= 64) logits(xent_p_kernel<E, 128, 64, 4, 1, 2, ENTROPY>, 128, 64, 256);
            else {
                bool wide = false;
                if constexpr (sizeof(E) == 2) {
                    wide = (int64_t)over(rows, 256) * over(n, 256) >= 200;
                    if (wide) logits(xent_p_kernel<E, 256, 256, 2, 4, 2, ENTROPY>, 256, 256, 512);
                }
                if constexpr (sizeof(E) == 4) logits(xent_p_kernel<E, 64, 64, 2, 2, 2, ENTROPY>, 64, 64, 256);
                else if (!wide) logits(xent_p_kernel<E, 128, 128, 2, 2, 2, ENTROPY>, 128, 128, 256);
            }
        };
        if (t.dentropy) all_logits(std::true_type{});
        else all_logits(std::false_type{});
        const int stages = (int)((width + TILE_BYTES - 1) / TILE_BYTES);
        a.v0 = v0;
        a.rows = rows;
        a.p_bytes = (int)width;
        a.each = (stages + g.splits - 1) / g.splits * TILE_BYTES;
        a.first = v0 == 0 ? 1 : 0;
        a.dw = dw ? dw + v0 * d : nullptr;
        a.dw_y = dw ? over(rows, side) : 0;
        const dim3 grid(a.dh_x * a.dh_y * g.splits + a.dw_x * a.dw_y);
        const auto products = [&](auto kernel, int threads) { hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, s, a); };
        if constexpr (sizeof(E) == 2) {
            if (g.side == 256) products(xent_products_kernel<E, 256, 2, 4, 2>, 512);
        }
        if (g.few) products(xent_products_kernel<E, 64, 2, 2, 4>, 256);
        else if constexpr (sizeof(E) == 4) products(xent_products_kernel<E, 64, 2, 2, 2>, 256);
        else if (g.side == 128) products(xent_products_kernel<E, 128, 2, 2, 2>, 256);
    }
    if (g.direct) return;
    // (few outputs: a wave a workgroup, so that more CUs ask for their parts)
    const int by = d % 4 == 0 || n * d >= 256 * 1024 ? 4 : 1;
    const int64_t outs = n * ((d + by - 1) / by), threads = outs < 64 * 1024 ? 64 : 256, out_wgs = (outs + threads - 1) / threads;
    const dim3 out_grid((unsigned)(out_wgs < 16384 ? out_wgs : 16384)), out_block((unsigned)threads);
    if (d % 4 == 0) hipLaunchKernelGGL((xent_dh_kernel<E, 4, true>), out_grid, out_block, 0, s, a, d / 4);
    else if (by == 1) hipLaunchKernelGGL((xent_dh_kernel<E, 1, true>), out_grid, out_block, 0, s, a, d);
    else hipLaunchKernelGGL((xent_dh_kernel<E, 4, false>), out_grid, out_block, 0, s, a, (d + 3) / 4);
}

void tg_launch_xent_grad(const void* h, int64_t ld_h, const void* w, int64_t ld_w, int dtype, int64_t n, int64_t n_rows, int d, const XentTokens& t,
                         float scale, void* dh, void* dw, void* space, size_t bytes, hipStream_t s)
{
    const int e = (int)tg_type_bytes(dtype);
    if (n == 0) {
        if (dw) tg_launch_zero(dw, (size_t)n_rows * d * e, s);
        return;
    }
    const bool ready = tile_ready(w, ld_w, d, e);
    // the largest piece that the workspace holds
    int64_t p_bytes = XENT_PIECE_BYTES * 64;
    while (p_bytes > 0 && xent_grad_bytes(n, n_rows, d, e, ready, p_bytes, dw != nullptr) > bytes) p_bytes = p_bytes > (1 << 20) ? p_bytes / 2 : 0;
    const XentGrad g = xent_grad_shape(n, n_rows, d, e, p_bytes, dw != nullptr);
    TgCarve c{(char*)space, 0};
    XentRows r;
    float *consts, *sums, *lost;
    char* p;
    carve_xent_grad(&r, &c, h, ld_h, w, ld_w, n, n_rows, d, e, ready, g, &consts, &p, &sums, &lost);
    if (!ready) tg_launch_pack(w, ld_w, n_rows, d, e, r.pw, s);
    TG_WITH_TYPE(dtype, E, launch_xent_grad<E>(r, g, h, ld_h, w, ld_w, n, n_rows, d, t, scale, consts, p, sums, lost, (E*)dh, (E*)dw, s));
}
