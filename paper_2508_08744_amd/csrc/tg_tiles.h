// Products of two row-major matrices whose rows run along the contraction (out[t][u] = sum_k Y[t][k] X[u][k]), in tiles on the matrix
// instructions, for 8-bit integers, bf16, fp16 and fp32 alike: everything up to the multiplication works on bytes.
//
// A workgroup owns BM rows of X and BN rows of Y.  128 bytes of each row are in LDS at a time, in one of two stages: while one is
// multiplied the other is filled, straight from memory (buffer loads with LDS as their destination; rows and bytes beyond the matrices come as
// zeros from the buffer's own bounds check).  A stage holds 8 pieces of 16 bytes a row; piece c of row r lies at place c ^ (r & 7), so
// that the eight rows that a matrix instruction's lanes read at a time lie in different banks.  The loads write LDS in lane order, so
// the exchange is made by the lanes' addresses in memory.
//
// The lane's share of a product of 16 x 16: column t = lane % 16 and rows u = 4 (lane / 16) + 0..3, so that it holds neighbours of an
// output row (they run along u).
#pragma once
#include "tg_embed.h"
#include "tg_device.h"

typedef float tg_f32x4 __attribute__((ext_vector_type(4)));
typedef int tg_i32x4 __attribute__((ext_vector_type(4)));
typedef tg_bf16 tg_bf16x8 __attribute__((ext_vector_type(8)));
typedef tg_f16 tg_f16x8 __attribute__((ext_vector_type(8)));

// 16 bytes of a lane on either side: 64 bytes of 16 rows each
template <class E> struct TileMul;
template <> struct TileMul<int8_t> {
    typedef tg_i32x4 acc;
    static __device__ inline acc mul(tg_i32x4 x, tg_i32x4 y, acc c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(x, y, c, 0, 0, 0); }
};
template <> struct TileMul<tg_bf16> {
    typedef tg_f32x4 acc;
    static __device__ inline acc mul(tg_i32x4 x, tg_i32x4 y, acc c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(tg_bf16x8, x), __builtin_bit_cast(tg_bf16x8, y), c, 0, 0, 0);
    }
};
template <> struct TileMul<tg_f16> {
    typedef tg_f32x4 acc;
    static __device__ inline acc mul(tg_i32x4 x, tg_i32x4 y, acc c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(tg_f16x8, x), __builtin_bit_cast(tg_f16x8, y), c, 0, 0, 0);
    }
};
template <> struct TileMul<float> {
    typedef tg_f32x4 acc;
    // the instruction takes one value a lane and side: value i of the four is its k, the same on both sides
    static __device__ inline acc mul(tg_i32x4 x, tg_i32x4 y, acc c)
    {
        const tg_f32x4 a = __builtin_bit_cast(tg_f32x4, x), b = __builtin_bit_cast(tg_f32x4, y);
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
        return c;
    }
};

// A matrix as the tiles read it: 16-byte aligned rows, `width` bytes of each used, the next row `pitch` bytes on (a multiple of 16, at
// most TILE_MAX_PITCH: what a stage reads stays within a buffer's 32-bit offsets).  A side whose rows run along the contraction needs a
// width that is a multiple of 16.  A side can also be given the other way round, its rows being the contraction's (`turned`).
struct TileRows {
    const char* p;
    int64_t rows;
    uint32_t pitch, width;
};

typedef __attribute__((address_space(3))) char tg_lds_char;

// Rows that are not made like that are copied: `bytes` of each, then zeros up to a multiple of 16.
#define TILE_MAX_PITCH (1u << 20)
static inline uint32_t tile_pitch(int64_t d, int e) { return (uint32_t)((d * e + 15) & ~(int64_t)15); }
static inline bool tile_ready(const void* p, int64_t ld, int64_t d, int e)
{
    return ((uintptr_t)p & 15) == 0 && (ld * e & 15) == 0 && (d * e & 15) == 0 && ld * e <= (int64_t)TILE_MAX_PITCH;
}
void tg_launch_pack(const void* p, int64_t ld, int64_t rows, int d, int e, void* out, hipStream_t s);

#define TILE_BYTES 128    // of a row, per stage

// One side of a stage: B rows of 128 bytes, or, turned, 128 / sizeof(E) rows of B elements.  Both take B * 128 bytes.
//
// Turned, the lanes need values of a column: 16-bit values come through the LDS reads that hand every lane of a group of 16 the four values of
// one column out of four rows, 32-bit values one by one.  Rows that are read at a time have their pieces exchanged in pairs (16 bit) or in
// fours (32 bit), so that they too lie in different banks.
template <class E, int B, int WAVES, bool TURNED>
struct TileSide {
    static constexpr int DEPTH = TILE_BYTES / (int)sizeof(E);          // of the contraction, per stage
    static constexpr int ROW = TURNED ? B * (int)sizeof(E) : TILE_BYTES;
    static constexpr int PIECES = ROW / 16;                            // of a row
    static constexpr int LOADS = B / 8 / WAVES;                        // of a wave, 1024 bytes each
    static_assert((B / 8) % WAVES == 0 && ROW <= 1024, "whole loads");
    static_assert(!TURNED || (sizeof(E) > 1 && ROW >= 128), "turned bytes are not read");

    // which piece of row r lies at place 0: place c holds piece c ^ that
    static __device__ inline int exchange(int r)
    {
        if (!TURNED) return r & 7;
        if (sizeof(E) == 4) return ((r >> 2) & 3) << 2;
        return ((r & 3) | (PIECES >= 16 ? ((r >> 3) & 1) << 2 : 0)) << 1;
    }

    uint32_t offset[LOADS];
    int in_row;                  // !TURNED: where the lane's piece is in the stage's bytes of a row

#ifdef __HIP_DEVICE_COMPILE__              // (the host's compiler does not know the buffers' types)
    __amdgpu_buffer_rsrc_t rsrc;

    __device__ inline void begin(const TileRows& m, int64_t first, int wave, int lane)
    {
        const int64_t have = m.rows - first;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int at = (i * WAVES + wave) * 1024 + lane * 16, r = at / ROW, c = (at % ROW) / 16;
            offset[i] = r * m.pitch + ((c ^ exchange(r)) * 16);
        }
        in_row = ((lane & 7) ^ ((lane >> 3) & 7)) * 16;
        // (rows from `first` on: none behind the last; what a row holds behind k1 is never asked for)
        if (!TURNED)
            rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)(m.p + first * m.pitch), 0, (int)(uint32_t)((have < B ? have : B) * m.pitch), 0x00020000);
    }
    // the stage that begins at byte k of the rows (element k / sizeof(E) of the contraction), up to byte k1
    __device__ inline void fill(const TileRows& m, int64_t first, char* stage, int64_t k, int64_t k1, int wave)
    {
        if (TURNED) {
            // columns from `first` on: those behind the width belong to the next row (results that nobody stores), or to nobody
            const int64_t r = k / (int)sizeof(E);
            const int64_t left = m.rows - r < DEPTH ? m.rows - r : DEPTH;
            const int64_t bytes = (left - 1) * m.pitch + m.width - first * (int)sizeof(E);
            rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)(m.p + r * m.pitch + first * (int)sizeof(E)), 0, (int)(uint32_t)bytes, 0x00020000);
        }
        const bool in = TURNED || k + in_row < k1;
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (tg_lds_char*)(stage + (i * WAVES + wave) * 1024), 16,
                                                     !in ? 0x80000000u /* behind every buffer's end */ : TURNED ? offset[i] : offset[i] + (uint32_t)k, 0, 0, 0);
    }
    // the lane's 16 bytes of the 16 rows (columns) from b0 on, of the first or second half of the stage
    static __device__ inline tg_i32x4 read(const char* stage, int b0, int h, int lane)
    {
        const int row = lane & 15, q = lane >> 4;
        if (!TURNED) return *reinterpret_cast<const tg_i32x4*>(stage + (b0 + row) * TILE_BYTES + (((q + 4 * h) ^ (row & 7)) * 16));
        if (sizeof(E) == 4) {
            tg_i32x4 v;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = h * 16 + q * 4 + i;
                v[i] = *reinterpret_cast<const int*>(stage + r * ROW + ((((b0 + row) / 4) ^ exchange(r)) * 16) + (row & 3) * 4);
            }
            return v;
        }
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        s16x4 v[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int r = h * 32 + q * 8 + s * 4 + (row >> 2);
            v[s] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(tg_lds_char*)(stage + r * ROW + (((b0 / 8) ^ exchange(r)) * 16) + (row & 3) * 8));
        }
        return __builtin_bit_cast(tg_i32x4, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
    }
#endif
};

// BM x BN in WM x WN waves
template <class E, int BM, int BN, int WM, int WN, bool XT = false, bool YT = false>
struct Tile {
    static constexpr int WAVES = WM * WN, THREADS = 64 * WAVES;
    static constexpr int FM = BM / WM / 16, FN = BN / WN / 16;       // products of 16 x 16 of a wave
    static constexpr int STAGE = (BM + BN) * TILE_BYTES;
    typedef typename TileMul<E>::acc acc_t;
    typedef TileSide<E, BM, WAVES, XT> SX;
    typedef TileSide<E, BN, WAVES, YT> SY;

    acc_t acc[FM][FN];

    // rows (columns, where turned) x0.. of X and y0.. of Y, contraction bytes [k0, k1) (multiples of TILE_BYTES, k1 of 16 at its end)
    __device__ inline void run(const TileRows& X, const TileRows& Y, int64_t x0, int64_t y0, int64_t k0, int64_t k1, char* stage0, char* stage1)
    {
#ifdef __HIP_DEVICE_COMPILE__
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = tg_lane();
        const int wm = wave / WN, wn = wave % WN;
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[i][j] = acc_t{0, 0, 0, 0};
        SX sx;
        SY sy;
        sx.begin(X, x0, wave, lane);
        sy.begin(Y, y0, wave, lane);
        const auto fill = [&](char* stage, int64_t k) {
            sx.fill(X, x0, stage, k, k1, wave);
            sy.fill(Y, y0, stage + BM * TILE_BYTES, k, k1, wave);
        };
        const auto multiply = [&](const char* stage) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                tg_i32x4 x[FM], y[FN];
#pragma unroll
                for (int i = 0; i < FM; ++i) x[i] = SX::read(stage, wm * (BM / WM) + i * 16, h, lane);
#pragma unroll
                for (int j = 0; j < FN; ++j) y[j] = SY::read(stage + BM * TILE_BYTES, wn * (BN / WN) + j * 16, h, lane);
#pragma unroll
                for (int i = 0; i < FM; ++i)
#pragma unroll
                    for (int j = 0; j < FN; ++j) acc[i][j] = TileMul<E>::mul(x[i], y[j], acc[i][j]);
            }
        };
        // a stage is there when every wave's loads have landed, and may be filled again when every wave has read it
        const auto meet = [] {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
        };
        if (k0 >= k1) return;
        fill(stage0, k0);
        for (int64_t k = k0; k < k1; k += 2 * TILE_BYTES) {
            meet();
            if (k + TILE_BYTES < k1) fill(stage1, k + TILE_BYTES);
            multiply(stage0);
            if (k + TILE_BYTES >= k1) break;
            meet();
            if (k + 2 * TILE_BYTES < k1) fill(stage0, k + 2 * TILE_BYTES);
            multiply(stage1);
        }
        __syncthreads();
#endif
    }
    // the rows of X and Y that acc[i][j][0] belongs to; acc[i][j][e] is for x + e
    __device__ inline int x_of(int i) const { return ((threadIdx.x >> 6) / WN) * (BM / WM) + i * 16 + (tg_lane() >> 4) * 4; }
    __device__ inline int y_of(int j) const { return ((threadIdx.x >> 6) % WN) * (BN / WN) + j * 16 + (tg_lane() & 15); }
};

// four neighbours of an output row
template <class O>
__device__ inline void tile_put(O* p, const float* v, int64_t left)
{
    typedef O vec __attribute__((ext_vector_type(4), aligned(sizeof(O))));
    if (left >= 4) {
        vec o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = (O)v[e];
        *reinterpret_cast<vec*>(p) = o;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) p[e] = (O)v[e];
    }
}

// a launch has fewer than 2^32 work-items
#define TILE_LAUNCH_ITEMS (1ll << 31)

// Workgroups go to the eight dies in turn: tile number `b` of `count` such that every die gets a stretch of neighbours, whose rows its
// own L2 then holds.
__device__ inline uint32_t tile_of_block(uint32_t b, uint32_t count)
{
    const uint32_t die = b & 7, at = b >> 3, each = count >> 3, more = count & 7;
    return die * each + (die < more ? die : more) + at;
}
// ... and its place: stretches of `group` tiles along y for every tile along x, then the next group
__device__ inline void tile_place(uint32_t t, uint32_t nx, uint32_t ny, uint32_t group, uint32_t* tx, uint32_t* ty)
{
    const uint32_t per = nx * group, g = t / per, first = g * group;
    const uint32_t high = ny - first < group ? ny - first : group, in = t - g * per;
    *tx = in / high;
    *ty = first + in % high;
}
