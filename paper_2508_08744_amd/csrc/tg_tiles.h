// Products of two row-major matrices whose rows run along the contraction (out[t][u] = sum_k Y[t][k] X[u][k]), in tiles on the matrix
// instructions, for 8-bit integers, bf16, fp16 and fp32 alike: everything up to the multiplication works on bytes.
//
// A workgroup owns BM rows of X and BN rows of Y.  They pass through LDS in stages of 128 bytes a row (a line of the caches: shorter
// stretches halve the rate of the loads), filled straight from memory by buffer loads with LDS as their destination; rows and bytes beyond the
// matrices come as zeros from the buffer's own bounds check.
//
// Each side's stage is two units, its first and second half of the rows, and every wave has as many rows of one as of the other.  The
// four products of halves are four phases; they go round the halves so that each phase needs one unit more than the phase before, which
// is read from LDS into registers one phase ahead, and every phase frees one unit, which is filled for NB stages on.  So a load has
// 4 NB - 1 phases (of 16 products of 16 x 16 each, at 256 x 256) to land, the matrix instructions find their operands in registers, and a phase
// costs one barrier, at which all waves have the unit they read next and none still reads the one that is filled next.  NB is 2; where there
// are too few tiles for all CUs, each alone on its own, a load's way is what a stage costs, and smaller tiles have room for 4.
//
// A unit holds 8 pieces of 16 bytes a row; piece c of row r lies at place c ^ (r & 7), so that the eight rows that a matrix instruction's lanes
// read at a time lie in different banks.  The loads write LDS in lane order, so the exchange is made by the lanes' addresses in memory.
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

// One side of a workgroup's tile: B rows, in two units of B / 2.  Turned, a unit is 128 / sizeof(E) rows of the contraction of B / 2 elements.
// Both take B / 2 * 128 bytes.
//
// Turned, the lanes need values of a column: 16-bit values come through the LDS reads that hand every lane of a group of 16 the four values of
// one column out of four rows, 32-bit values one by one.  Rows that are read at a time have their pieces exchanged in pairs (16 bit) or in
// fours (32 bit), so that they too lie in different banks.
template <class E, int B, int WAVES, bool TURNED>
struct TileSide {
    static constexpr int UNIT = B / 2;
    static constexpr int DEPTH = TILE_BYTES / (int)sizeof(E);          // of the contraction, per stage
    static constexpr int ROW = TURNED ? UNIT * (int)sizeof(E) : TILE_BYTES;
    static constexpr int PIECES = ROW / 16;                            // of a row
    static constexpr int LOADS = (UNIT * TILE_BYTES / 1024 + WAVES - 1) / WAVES;   // of a wave and unit, 1024 bytes each
    static constexpr int BYTES = LOADS * WAVES * 1024;                 // of a unit, behind its end what surplus loads write
    static_assert(ROW <= 1024, "a load has whole rows");
    static_assert(!TURNED || (sizeof(E) > 1 && ROW >= 64 && LOADS * WAVES * 1024 == UNIT * TILE_BYTES), "turned bytes, short or odd rows are not read");

    // which piece of row r lies at place 0: place c holds piece c ^ that
    static __device__ inline int exchange(int r)
    {
        if (!TURNED) return r & 7;
        if (sizeof(E) == 4) return ((r >> 2) & (PIECES >= 16 ? 3 : 1)) << 2;
        if (PIECES == 4) return (r & 1) << 1;
        return ((r & 3) | (PIECES >= 16 ? ((r >> 3) & 1) << 2 : 0)) << 1;
    }

    uint32_t offset[LOADS];
    int in_row;                  // !TURNED: where the lane's piece is in the stage's bytes of a row
    // Kept for whole waves, in 32 bits where that will do: the scalar unit compares no more.
    uint64_t base;               // the first row (column) of the tile, at the contraction's beginning
    uint32_t pitch;
    int have;                    // !TURNED: bytes from there to behind the last row, TURNED: of a row, behind that place
    int depth;                   // TURNED: rows of the contraction

    __device__ inline void begin(const TileRows& m, int64_t first, int wave, int lane)
    {
        pitch = m.pitch;
        if (TURNED) {
            base = (uint64_t)m.p + first * (int)sizeof(E);
            have = (int)((int64_t)m.width - first * (int)sizeof(E));
            depth = (int)m.rows;
        } else {
            const int64_t left = m.rows - first;
            base = (uint64_t)m.p + first * m.pitch;
            have = (int)(left < B ? left : B) * (int)m.pitch;
        }
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int at = (i * WAVES + wave) * 1024 + lane * 16, r = at / ROW, c = (at % ROW) / 16;
            // (surplus loads: rows of the other unit, which nobody reads there)
            offset[i] = r * m.pitch + ((c ^ exchange(r)) * 16);
        }
        in_row = ((lane & 7) ^ (lane >> 3)) * 16;
    }
    // Unit h, the stage that begins at byte k of the contraction, up to byte k1; behind k1 all of it is zeros.  The load is written out, since the
    // compiler, which knows the built-in one as a store to LDS, waits for all of them in front of every read; it has no result, and
    // `meet` waits for it.  M0 (which nothing else in these kernels uses) holds where in LDS the wave's 1024 bytes go.
    __device__ inline void fill(int h, uint32_t unit, int k, int k1, int wave) const
    {
        uint64_t from;
        int bytes;
        if (TURNED) {
            // (columns behind the width belong to the next row, for results that nobody stores, or to nobody)
            const int r = k / (int)sizeof(E), left = depth - r < DEPTH ? depth - r : DEPTH;
            from = base + (uint64_t)r * pitch + h * UNIT * (int)sizeof(E);
            bytes = (left - 1) * (int)pitch + have - h * UNIT * (int)sizeof(E);
            if (k >= k1 || left < 1) bytes = 0;
        } else {
            // (what a row holds behind k1 is never asked for)
            from = base + (uint64_t)(h * UNIT) * pitch;
            bytes = have - h * UNIT * (int)pitch;
        }
        bytes = bytes < 0 ? 0 : bytes;
        const tg_i32x4 buffer = {(int)(uint32_t)from, (int)((uint32_t)(from >> 32) & 0xFFFFu), bytes, 0x00020000};
        const bool in = TURNED || in_row < k1 - k;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const uint32_t at = !in ? 0x80000000u /* behind every buffer's end */ : TURNED ? offset[i] : offset[i] + (uint32_t)k;
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(unit + (i * WAVES + wave) * 1024), "v"(at), "s"(buffer) : "memory");
        }
    }
#ifdef __HIP_DEVICE_COMPILE__              // (the host's compiler does not know the built-ins)
    // Where the lane's bytes of the 16 rows (columns) from b0 on are in a unit, for the first and second 64 bytes of the stage; the rows
    // 16 further on are at a distance that the reads carry, except where the exchange has a part in it.
    int at[TURNED ? (sizeof(E) == 4 ? 4 : 2) : 2];
    __device__ inline void begin_reads(int b0, int lane)
    {
        const int row = lane & 15, q = lane >> 4;
        if (!TURNED) {
#pragma unroll
            for (int h = 0; h < 2; ++h) at[h] = (b0 + row) * TILE_BYTES + (((q + 4 * h) ^ (row & 7)) * 16);
        } else if (sizeof(E) == 4) {
#pragma unroll
            for (int i = 0; i < 4; ++i) at[i] = (q * 4 + i) * ROW + (row & 3) * 4;
        } else {
#pragma unroll
            for (int s = 0; s < 2; ++s) at[s] = (q * 8 + s * 4 + (row >> 2)) * ROW + (row & 3) * 8;
        }
    }
    // i: 16 rows (columns) behind b0 times i
    __device__ inline tg_i32x4 read(const char* unit, int b0, int i, int h, int lane) const
    {
        const int row = lane & 15, q = lane >> 4;
        if (!TURNED) return *reinterpret_cast<const tg_i32x4*>(unit + at[h] + i * 16 * TILE_BYTES);
        b0 += i * 16;
        if (sizeof(E) == 4) {
            tg_i32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e)        // (exchange(row of the stage) is that of q alone)
                v[e] = *reinterpret_cast<const int*>(unit + at[e] + h * 16 * ROW + ((((b0 + row) / 4) ^ exchange(q * 4)) * 16));
            return v;
        }
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        s16x4 v[2];
#pragma unroll
        for (int s = 0; s < 2; ++s)            // (exchange(row of the stage): bits 0, 1 of row >> 2, bit 3 of q * 8)
            v[s] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(tg_lds_char*)(unit + at[s] + h * 32 * ROW + (((b0 / 8) ^ exchange(q * 8 + (row >> 2))) * 16)));
        return __builtin_bit_cast(tg_i32x4, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
    }
#endif
};

// the sum of the squares of a lane's 16 bytes, added to c
template <class E> __device__ inline float tile_squares(tg_i32x4 x, float c)
{
#ifdef __HIP_DEVICE_COMPILE__
    typedef tg_bf16 bf16x2 __attribute__((ext_vector_type(2)));
    typedef tg_f16 f16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (__is_same(E, tg_bf16)) c = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, x[i]), __builtin_bit_cast(bf16x2, x[i]), c, false);
        else if constexpr (__is_same(E, tg_f16)) c = __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, x[i]), __builtin_bit_cast(f16x2, x[i]), c, false);
        else c = fmaf(__builtin_bit_cast(float, x[i]), __builtin_bit_cast(float, x[i]), c);
    }
#endif
    return c;
}

// BM x BN in WM x WN waves, NB stages in LDS.  SQUARES: the sums of the squares of X's rows as well, from the registers that feed the products (a lane's share
// in squares[i], of row 16 (i % HM) + lane % 16 of the wave's rows in half i / HM; lanes 16, 32 and 48 on have the others), and all bits of them together in bits.
template <class E, int BM, int BN, int WM, int WN, bool XT = false, bool YT = false, int NB = 2, bool SQUARES = false>
struct Tile {
    static constexpr int WAVES = WM * WN, THREADS = 64 * WAVES;
    static constexpr int FM = BM / WM / 16, FN = BN / WN / 16;       // products of 16 x 16 of a wave
    static constexpr int HM = FM / 2, HN = FN / 2;                   // ... of half of its rows
    typedef typename TileMul<E>::acc acc_t;
    typedef TileSide<E, BM, WAVES, XT> SX;
    typedef TileSide<E, BN, WAVES, YT> SY;
    static constexpr int LX = SX::LOADS, LY = SY::LOADS;
    static constexpr int LDS = 2 * NB * (SX::BYTES + SY::BYTES);
    static_assert(FM % 2 == 0 && FN % 2 == 0 && (NB == 2 || NB == 4), "halves");

    acc_t acc[FM][FN];
    float squares[SQUARES ? FM : 1];
    int bits;

#ifdef __HIP_DEVICE_COMPILE__
    struct Run {
        int k, k1;
        int wave, lane, wm, wn;
        char* lds;
        SX sx;
        SY sy;
    };
    struct Halves {
        tg_i32x4 x[2][2][HM], y[2][2][HN];                           // [half of the rows][half of the stage]
    };
    // the memory of unit h of buffer b
    static __device__ inline char* unit_x(const Run& r, int b, int h) { return r.lds + (b * 2 + h) * SX::BYTES; }
    static __device__ inline char* unit_y(const Run& r, int b, int h) { return r.lds + 2 * NB * SX::BYTES + (b * 2 + h) * SY::BYTES; }
    static __device__ inline void fill_x(const Run& r, int b, int h, int k)
    {
        r.sx.fill(h, (uint32_t)(uintptr_t)(tg_lds_char*)unit_x(r, b, h), k, r.k1, r.wave);
    }
    static __device__ inline void fill_y(const Run& r, int b, int h, int k)
    {
        r.sy.fill(h, (uint32_t)(uintptr_t)(tg_lds_char*)unit_y(r, b, h), k, r.k1, r.wave);
    }
    // one of the 2 HM (2 HN) reads of a unit
    static __device__ inline void read_x(const Run& r, Halves& f, int b, int h, int n) { f.x[h][n / HM][n % HM] = r.sx.read(unit_x(r, b, h), r.wm * (HM * 16), n % HM, n / HM, r.lane); }
    static __device__ inline void read_y(const Run& r, Halves& f, int b, int h, int n) { f.y[h][n / HN][n % HN] = r.sy.read(unit_y(r, b, h), r.wn * (HN * 16), n % HN, n / HN, r.lane); }
    // All but the last `LATER` loads of every wave have landed, and no wave has reads under way.
    template <int LATER>
    static __device__ inline void meet()
    {
        static_assert(LATER < 64, "loads that are counted");
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LATER) : "memory");
        __builtin_amdgcn_sched_barrier(0);
    }
    // The products of halves hx and hy, out of registers; between them the reads of a unit of X (XU) or Y for the next phase, and the loads
    // of one, so that the matrix instructions wait for neither's turn to be issued.
    template <bool XU, bool SQ, class Fill>
    __device__ inline void phase(const Run& r, Halves& f, int hx, int hy, int read_buffer, int read_half, Fill fill)
    {
        constexpr int PRODUCTS = 2 * HM * HN, READS = XU ? 2 * HM : 2 * HN;
#pragma unroll
        for (int m = 0; m < PRODUCTS; ++m) {
            const int s = m / (HM * HN), i = m / HN % HM, j = m % HN;
            acc[hx * HM + i][hy * HN + j] = TileMul<E>::mul(f.x[hx][s][i], f.y[hy][s][j], acc[hx * HM + i][hy * HN + j]);
            if constexpr (SQ) {
                if (j == 0) {
                    const tg_i32x4 x = f.x[hx][s][i];
                    squares[hx * HM + i] = tile_squares<E>(x, squares[hx * HM + i]);
                    bits |= (x[0] | x[1]) | (x[2] | x[3]);
                }
            }
#pragma unroll
            for (int n = 0; n < READS; ++n)
                if (n * PRODUCTS / READS == m) {
                    if (XU) read_x(r, f, read_buffer, read_half, n);
                    else read_y(r, f, read_buffer, read_half, n);
                }
            if (m == PRODUCTS / 2) fill();
            __builtin_amdgcn_sched_barrier(0);      // (the order as it is written)
        }
    }
    // Stage of buffer B; Y's units in the order P, 1 - P.  Of the loads that a phase waits for, those of the 4 NB - 2 phases before it may be on
    // their way: FAR of them, and the last six phases' by kind.
    template <int B>
    __device__ inline void stage(Run& r, Halves& f)
    {
        constexpr int P = B & 1, NEXT = (B + 1) % NB, FAR = (NB - 2) * (2 * LX + 2 * LY);
        meet<FAR + 4 * LX + 2 * LY>();
        phase<false, SQUARES>(r, f, 0, P, B, 1 - P, [&] { fill_y(r, B, P, r.k + NB * TILE_BYTES); });
        meet<FAR + 3 * LX + 3 * LY>();
        phase<true, false>(r, f, 0, 1 - P, B, 1, [&] { fill_y(r, B, 1 - P, r.k + NB * TILE_BYTES); });
        meet<FAR + 2 * LX + 4 * LY>();
        phase<true, SQUARES>(r, f, 1, 1 - P, NEXT, 0, [&] { fill_x(r, B, 1, r.k + NB * TILE_BYTES); });
        meet<FAR + 3 * LX + 3 * LY>();
        phase<false, false>(r, f, 1, P, NEXT, 1 - P, [&] { fill_x(r, NEXT, 0, r.k + (NB + 1) * TILE_BYTES); });
        r.k += TILE_BYTES;
    }
    Run r;
#endif

    // Asks for the first stages of rows (columns, where turned) x0.. of X and y0.. of Y, contraction bytes [k0, k1) (k0 a multiple of TILE_BYTES, k1 of
    // 16; below 2^31 - 2^10).  lds: LDS bytes that begin at a multiple of 1024, and that no wave reads any more.  acc is left alone.
    __device__ inline void start(const TileRows& X, const TileRows& Y, int64_t x0, int64_t y0, int k0, int k1, char* lds)
    {
#ifdef __HIP_DEVICE_COMPILE__
        r.wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        r.lane = tg_lane();
        r.wm = r.wave / WN;
        r.wn = r.wave % WN;
        r.lds = lds;
        r.k = k0;
        r.k1 = k1;
        r.sx.begin(X, x0, r.wave, r.lane);
        r.sy.begin(Y, y0, r.wave, r.lane);
        r.sx.begin_reads(r.wm * (HM * 16), r.lane);
        r.sy.begin_reads(r.wn * (HN * 16), r.lane);
        // in the order of the phases that would have asked for them
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            fill_x(r, b, 0, k0 + b * TILE_BYTES);
            fill_y(r, b, b & 1, k0 + b * TILE_BYTES);
            fill_y(r, b, 1 - (b & 1), k0 + b * TILE_BYTES);
            fill_x(r, b, 1, k0 + b * TILE_BYTES);
        }
#endif
    }
    // ... and the products (an empty stretch is one stage of zeros).  Behind it no wave reads the memory any more.
    __device__ inline void loop()
    {
#ifdef __HIP_DEVICE_COMPILE__
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[i][j] = acc_t{0, 0, 0, 0};
        if constexpr (SQUARES) {
#pragma unroll
            for (int i = 0; i < FM; ++i) squares[i] = 0.0f;
            bits = 0;
        }
        constexpr int FAR = (NB - 2) * (2 * LX + 2 * LY);
        Halves f;
        // the reads of the two phases in front of the first
        meet<FAR + 2 * LX + 4 * LY>();
#pragma unroll
        for (int n = 0; n < 2 * HM; ++n) read_x(r, f, 0, 0, n);
        meet<FAR + 3 * LX + 3 * LY>();
#pragma unroll
        for (int n = 0; n < 2 * HN; ++n) read_y(r, f, 0, 0, n);
        fill_x(r, 0, 0, r.k + NB * TILE_BYTES);
        for (;;) {
            stage<0>(r, f);
            if (r.k >= r.k1) break;
            stage<1>(r, f);
            if (r.k >= r.k1) break;
            if constexpr (NB == 4) {
                stage<2>(r, f);
                if (r.k >= r.k1) break;
                stage<3>(r, f);
                if (r.k >= r.k1) break;
            }
        }
        // (loads of zeros behind the end may still be on their way into LDS)
        meet<0>();
#endif
    }
    __device__ inline void run(const TileRows& X, const TileRows& Y, int64_t x0, int64_t y0, int k0, int k1, char* lds)
    {
        start(X, Y, x0, y0, k0, k1, lds);
        loop();
    }
    // the rows of X and Y that acc[i][j][0] belongs to; acc[i][j][e] is for x + e (from the thread's number alone: the products' loop has no register for more)
    __device__ inline int x_of(int i) const { return (i / HM) * (BM / 2) + ((threadIdx.x >> 6) / WN) * (HM * 16) + (i % HM) * 16 + (threadIdx.x >> 4 & 3) * 4; }
    __device__ inline int y_of(int j) const { return (j / HN) * (BN / 2) + ((threadIdx.x >> 6) % WN) * (HN * 16) + (j % HN) * 16 + (threadIdx.x & 15); }
};

// four neighbours of an output row
template <class O>
__device__ inline void tile_put(O* p, const float* v, int left)
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
    // (the divisions are the vector unit's: the results go back to where the addresses of whole waves are formed)
    *tx = (uint32_t)__builtin_amdgcn_readfirstlane((int)(in / high));
    *ty = (uint32_t)__builtin_amdgcn_readfirstlane((int)(first + in % high));
}
