// Log probabilities of given rows of a table, the entropy of the softmax over all of them, and the best rows, without the logits.
//
// A tile of logits stays in the registers of the workgroup that formed it.  For every token it leaves the maximum m, the sum l of 2^t and the
// sum s of t 2^t, t = (z - m) log2(e): joined over the table they give lse = m + log l and the entropy log l - log(2) s / l.  2 n n_rows d operations on the
// matrix instructions bound it, or, for few tokens, the bytes of the table.  (131 072 rows of 1024 bf16: 4096 tokens 921 us, 1.19 PFLOP/s, with 8 best rows 1047, 44 for the
// norms and 39 to 54 for the join; one token 39 us, 6.8 TB/s, and 13 for the join.)
//
// The best rows are those of the largest logits in 64 bits, and the logits of the tiles are in 32.  So every lane of a tile leaves, of its 8, 16 or 32
// logits of a token (a group), the largest with its row and an upper bound of the second: at most a byte a logit (which two waves of a tile of 256 x 256 store half a line each: 1.7 times as much is written).  With 64 lanes over a token's groups, the k-th largest of the lanes' largest is below the k-th
// logit but for what the roundings of 32 bits reach (a bound from the norms of the token's row and of the longest row of the logit's tile, see LpMargin); whatever does not come up to it with its own bound is none of
// the k best.  What is left, some k rows, is scored again in 64 bits and put in order.  A group whose second is not out of reach is scored as a whole.
// (Bounds by tile: 4096 tokens, 32 768 rows of 4096 bf16, one of them 30 or 1000 times as long as the others: 1.06 and 1.6 ms; 46 and 105 with the table's longest row in all bounds; without such a row 0.99.)
#include "tg_embed.h"
#include "tg_softmax.h"
#include "tg_tiles.h"

#define LP_GROUP_LEAST 8        // logits of a token that leave their largest, in the smallest tiles
#define LP_MAX_TOP 32           // best rows; half the lanes of a wave, see lp_kth
#define LP_NORM_ROWS 256        // of the table, where the tiles, which have as many, leave no norms
#define LP_BELOW (-1000.0f)     // exponents below have a power of 0: so is their part in s, at -infinity too

// A stretch of the table whose largest square is 0 has rows of zeros alone: squares too small for their type are taken for the least above it.
#define LP_LEAST 1.17549435e-38f
#define LP_BITS(E) (sizeof(E) == 4 ? 0x7FFFFFFF : 0x7FFF7FFF)     // but the signs

typedef unsigned int lp_u32;

// (maximum, sum, sum below it) over stretches of a table; one that stands for nothing is (-infinity, 0, 0)
struct LpSum { float m, l, s; };
__device__ inline void lp_join(LpSum& a, const LpSum& b)
{
    const float top = fmaxf(a.m, b.m);
    const float wa = a.m == top ? 1.0f : xent_exp(a.m - top), wb = b.m == top ? 1.0f : xent_exp(b.m - top);
    // (a weight of 0 may come from a difference that is infinite)
    const float sa = a.m == top ? a.s : wa > 0.0f ? wa * (a.s + (a.m - top) * XENT_LOG2E * a.l) : 0.0f;
    const float sb = b.m == top ? b.s : wb > 0.0f ? wb * (b.s + (b.m - top) * XENT_LOG2E * b.l) : 0.0f;
    a.l = a.l * wa + b.l * wb;
    a.s = sa + sb;
    a.m = top;
}

// The second of a group, rounded up, with the largest one's row in the tile (below 256) in its last bits.  As a value it is no smaller than the second; beyond
// fp32's range it is a NaN, which is below nothing.
__device__ inline lp_u32 lp_pack(float second, int row) { return ((tg_ord(fmaxf(second, -3.38e38f)) & ~255u) + 256u) | (lp_u32)row; }
__device__ inline float lp_second(lp_u32 key) { return tg_unord(key); }
__device__ inline int lp_row(lp_u32 key) { return (int)(key & 255u); }

// a product that is no smaller than the exact one
__device__ inline float lp_times_up(float x, float by)
{
    const float z = x * by;
    return fmaf(fabsf(z), 0x1p-23f, z);
}

// x: rows of the table from v0 on, y: tokens.  parts: for every token the tiles along x; groups: for every token, tile and group (largest, packed second).  The epilogue asks nothing per
// value: targets, infinities and the table's end are branches that whole tiles pass by (8192 tokens, 50 000 rows of 128 bf16: 228 us, 271 with a question every four values).
template <class E, int BM, int BN, int WM, int WN, int NB, bool TOP>
__global__ __launch_bounds__(64 * WM * WN) void lp_part_kernel(TileRows X, TileRows Y, int bytes, const void* __restrict__ targets, int targets64,
                                                               float scale, int64_t v0, int64_t n_rows, uint32_t nx, uint32_t ny, uint32_t group,
                                                               float4* __restrict__ parts, int64_t parts_pitch, uint2* __restrict__ groups,
                                                               float* __restrict__ norms, float* __restrict__ at_target)
{
    // (the norms' squares ride along where registers are left for their sums: tiles of up to 128 rows)
    constexpr bool SQUARES = TOP && BM <= 128;
    typedef Tile<E, BM, BN, WM, WN, false, false, NB, SQUARES> T;
    constexpr int GROUPS = 4 * WM;                 // of a tile: one for each quarter of a wave (16 lanes), which has 4 FM of its rows
    static_assert(4 * T::FM <= 32, "five bits for a place");
    __shared__ __align__(1024) char lds[T::LDS];
    // the tokens' targets among the tile's rows: asked for before the products, so that nothing waits for them behind
    __shared__ int s_target[BN];
    __shared__ float s_norm[WM * WN];
    uint32_t tx, ty;
    tile_place(tile_of_block(blockIdx.x, nx * ny), nx, ny, group, &tx, &ty);
    const int64_t x0 = (int64_t)tx * BM, y0 = (int64_t)ty * BN;
    T t;
    t.start(X, Y, x0, y0, 0, bytes, lds);
    if (threadIdx.x < BN) {
        const int64_t y = y0 + threadIdx.x, target = targets && y < Y.rows ? tg_row_of(targets, targets64, y, n_rows) - v0 - x0 : -1;
        s_target[threadIdx.x] = target >= 0 && target < BM ? (int)target : -1;
    }
    t.loop();
    if constexpr (SQUARES) {
        float top = 0.0f;
#pragma unroll
        for (int i = 0; i < T::FM; ++i) {
            float q = t.squares[i];
            q += __shfl_xor(q, 16);
            q += __shfl_xor(q, 32);
            top = fmaxf(top, q);
        }
#pragma unroll
        for (int m = 1; m < 16; m <<= 1) top = fmaxf(top, __shfl_xor(top, m));
        const bool some = __any((t.bits & LP_BITS(E)) != 0);
        if (tg_lane() == 0) s_norm[threadIdx.x >> 6] = some ? fmaxf(top, LP_LEAST) : 0.0f;
    }
    // (the tile's memory is free: a sum for every token and wave along x)
    LpSum* const s_sum = reinterpret_cast<LpSum*>(lds) + (threadIdx.x >> 6) / WN * BN;
    static_assert(WM * BN * sizeof(LpSum) <= T::LDS, "the sums' place");
    // From here on the factor is above 0, so that the largest logit is the largest product times it (rounding keeps the order), and there is no row behind the table's end
    // that anything is taken of.
    if (__builtin_expect(!(scale > 0.0f), 0)) {
        const float by = scale < 0.0f ? -1.0f : scale;             // (0, or a NaN)
#pragma unroll
        for (int i = 0; i < T::FM; ++i)
#pragma unroll
            for (int j = 0; j < T::FN; ++j) t.acc[i][j] *= by;
        scale = scale < 0.0f ? -scale : 1.0f;
    }
    const int have = x0 + BM <= X.rows ? BM : (int)(X.rows - x0);
    if (__builtin_expect(have < BM, 0)) {
#pragma unroll
        for (int i = 0; i < T::FM; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (t.x_of(i) + e >= have)
#pragma unroll
                    for (int j = 0; j < T::FN; ++j) t.acc[i][j][e] = -__builtin_inff();
    }
    const int none = (threadIdx.x >> 6) / WN * (T::HM * 16);        // the wave's first row: where the table ends before it there are no logits
    const float base = scale * XENT_LOG2E;
#pragma unroll
    for (int j = 0; j < T::FN; ++j) {
        const int64_t y = y0 + t.y_of(j);
        const int target = s_target[t.y_of(j)];
        if (__any(target >= 0)) {
#pragma unroll
            for (int i = 0; i < T::FM; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (t.x_of(i) + e == target) at_target[y] = t.acc[i][j][e] * scale;
        }
        float m = -__builtin_inff(), least = -m, l = 0.0f, s = 0.0f;
#pragma unroll
        for (int i = 0; i < T::FM; ++i) {
            m = fmaxf(fmaxf(m, t.acc[i][j][0]), t.acc[i][j][1]);
            m = fmaxf(fmaxf(m, t.acc[i][j][2]), t.acc[i][j][3]);
            if (TOP) {
                least = fminf(fminf(least, t.acc[i][j][0]), t.acc[i][j][1]);
                least = fminf(fminf(least, t.acc[i][j][2]), t.acc[i][j][3]);
            }
        }
        const float largest = m;
        m *= scale;
        if (TOP) {
            // The largest and the second with their place in the last five bits, as numbers: off by less than 2^-18 of them.  Where that makes another one the largest, the
            // second, rounded up, is no smaller than the largest.  (Infinite ones have no such bits: they are compared as they are.)
            float first = -__builtin_inff(), second = first;
            int at = 0;
            if (__builtin_expect(__all(largest < __builtin_inff() && least > -__builtin_inff()), 1)) {
#pragma unroll
                for (int i = 0; i < T::FM; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float z = __uint_as_float((__float_as_uint(t.acc[i][j][e]) & ~31u) | (unsigned)(i * 4 + e));
                        second = __builtin_amdgcn_fmed3f(first, second, z);
                        first = fmaxf(first, z);
                    }
                at = (int)(__float_as_uint(first) & 31u);
                const lp_u32 bits = __float_as_uint(second);
                second = __uint_as_float(bits >> 31 ? bits & ~31u : bits | 31u);
            } else {
#pragma unroll
                for (int i = 0; i < T::FM; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float z = t.acc[i][j][e];
                        at = z > first ? i * 4 + e : at;
                        second = fmaxf(second, fminf(first, z));
                        first = fmaxf(first, z);
                    }
            }
            const int i = at >> 2;
            // (x_of for an i that is not known in advance)
            const int quarter = threadIdx.x >> 4 & 3, x = (i / T::HM) * (BM / 2) + none + (i % T::HM) * 16 + quarter * 4 + (at & 3);
            if (y < Y.rows)
                groups[(y * parts_pitch + tx) * GROUPS + (threadIdx.x >> 6) / WN * 4 + quarter] = make_uint2(__float_as_uint(m), lp_pack(lp_times_up(second, scale), x));
        }
        m = fmaxf(m, __shfl_xor(m, 16));
        m = fmaxf(m, __shfl_xor(m, 32));
        const bool near = xent_near(m, base) || have <= none;
        const float f = near ? base : 1.0f, b = near && have > none ? m * XENT_LOG2E : 0.0f;
        if (__builtin_expect(!__all(near), 0)) {           // (out of the way: code that is jumped over is fetched late)
#pragma unroll
            for (int i = 0; i < T::FM; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) t.acc[i][j][e] = near ? t.acc[i][j][e] : xent_far<true>(t.acc[i][j][e], scale, m);
        }
#pragma unroll
        for (int i = 0; i < T::FM; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float u = fmaf(t.acc[i][j][e], f, -b), p = __builtin_amdgcn_exp2f(u);
                l += p;
                s = fmaf(p, u, s);
            }
        if (__builtin_expect(__any(s != s), 0)) {          // (a power of 0 times the -infinity that it is of)
            s = 0.0f;
#pragma unroll
            for (int i = 0; i < T::FM; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float u = fmaf(t.acc[i][j][e], f, -b);
                    s = fmaf(__builtin_amdgcn_exp2f(u), fmaxf(u, LP_BELOW), s);
                }
        }
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        s += __shfl_xor(s, 16);
        s += __shfl_xor(s, 32);
        if (tg_lane() < 16) s_sum[t.y_of(j)] = LpSum{m, l, s};
    }
    __syncthreads();
    if (threadIdx.x < BN && y0 + threadIdx.x < Y.rows) {
        const LpSum* sum = reinterpret_cast<const LpSum*>(lds) + threadIdx.x;
        LpSum a = sum[0];
#pragma unroll
        for (int w = 1; w < WM; ++w) lp_join(a, sum[w * BN]);
        parts[(y0 + threadIdx.x) * parts_pitch + tx] = make_float4(a.m, a.l, a.s, 0.0f);
    }
    // (every column of tiles has the same: the first says it)
    if (SQUARES && norms && ty == 0 && threadIdx.x == 0) {
        float top = s_norm[0];
#pragma unroll
        for (int w = 1; w < WM * WN; ++w) top = fmaxf(top, s_norm[w]);
        norms[tx] = top;
    }
}

// The largest sum of the squares of LP_NORM_ROWS rows at a time.  `lanes` lanes a row; four rows are asked for at once.  Bound by the table's bytes (268 MB: 44 us, 6.1 TB/s).
template <class E>
__global__ __launch_bounds__(1024) void lp_norms_kernel(const E* __restrict__ w, int64_t ld, int64_t n_rows, int d, int lanes, float* __restrict__ out, int64_t count)
{
    __shared__ float s_top[16];
    typedef TgPiece<E> P;
    const int of = threadIdx.x & (lanes - 1), rows = 1024 / lanes, first = threadIdx.x / lanes;
    for (int64_t b = blockIdx.x; b < count; b += gridDim.x) {
        float top = 0.0f;
        for (int r = first; r < LP_NORM_ROWS; r += 4 * rows) {
            float sum[4] = {};
            bool some = false;
            for (int c = of * P::E; c < d; c += lanes * P::E) {
                typename P::vec v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int64_t row = b * LP_NORM_ROWS + r + i * rows;
                    v[i] = P::raw(w + (row < n_rows ? row : 0) * ld + c, r + i * rows < LP_NORM_ROWS && row < n_rows ? d - c : 0);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int e = 0; e < P::E; ++e) sum[i] = fmaf((float)v[i][e], (float)v[i][e], sum[i]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const tg_i32x4 x = __builtin_bit_cast(tg_i32x4, v[i]);
                    some |= (((x[0] | x[1]) | (x[2] | x[3])) & LP_BITS(E)) != 0;
                }
            }
            if (some) top = fmaxf(top, LP_LEAST);
            for (int m = 1; m < lanes; m <<= 1)
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[i] += __shfl_xor(sum[i], m);
            top = fmaxf(fmaxf(fmaxf(sum[0], sum[1]), fmaxf(sum[2], sum[3])), top);
        }
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) top = fmaxf(top, __shfl_xor(top, m));
        if ((threadIdx.x & 63) == 0) s_top[threadIdx.x >> 6] = top;
        __syncthreads();
        top = s_top[threadIdx.x & 15];
#pragma unroll
        for (int m = 1; m < 16; m <<= 1) top = fmaxf(top, __shfl_xor(top, m));
        if (threadIdx.x == 0) out[b] = top;
        __syncthreads();
    }
}

// How far a logit of a tile is from its exact value at most.  Every one of the d products and sums is off by less than 2^-23 of the sum of the products'
// magnitudes (twice the step of rounding to the nearest: nothing is taken for granted of how the matrix instructions add), or by 2^-126 where it is below the normal numbers (which
// may be taken for 0), the factor's product by as much, and that
// sum is at most |h| |w|.  The squares' sums are off by less than d 2^-23 themselves, and what of them is too small for the type's products is added.
template <class E>
struct LpMargin {
    double by, least;
    float lost, more;
    // h2: the token's square; exact: its logits are (a row of zeros, a factor of 0)
    __device__ inline LpMargin(float scale, int d, double h2, bool exact) : lost((__is_same(E, tg_f16) ? 0x1p-28f : 0x1p-126f) * (float)d), more(1.0f + (float)d * 0x1p-22f)
    {
        // (roots in 32 bits, of normal numbers and a step off at most: 2^-20 more makes up for that)
        by = exact ? 0.0 : fabs((double)scale) * (d + 2) * 0x1.00001p-23 * (double)__builtin_amdgcn_sqrtf((float)((h2 + lost) * more));
        least = exact ? 0.0 : fabs((double)scale) * d * 0x1p-125 + 0x1p-120;
    }
    // of the logits of a tile with rows of squares up to w2
    __device__ inline double of(float w2) const { return w2 == 0.0f || by == 0.0 ? 0.0 : fma(by, (double)__builtin_amdgcn_sqrtf((w2 + lost) * more), least); }
};

// What the k-th largest of a wave's values is not below, in all lanes: its first 20 bits (a NaN counts as the smallest; less than everything is a NaN itself).
__device__ inline float lp_kth(float v, int k)
{
    const lp_u32 mine = v != v ? 0u : tg_ord(v);
    lp_u32 least = 0;
#pragma unroll
    for (int bit = 31; bit >= 12; --bit) {
        const lp_u32 more = least | 1u << bit;
        least = __popcll(__ballot(mine >= more)) >= k ? more : least;
    }
    return tg_unord(least);
}

__device__ inline double lp_lane64(double x, int lane)
{
    const u64 b = __double_as_longlong(x);
    const u64 lo = (u32)__builtin_amdgcn_readlane((int)(u32)b, lane), hi = (u32)__builtin_amdgcn_readlane((int)(u32)(b >> 32), lane);
    return __longlong_as_double((long long)(hi << 32 | lo));
}
__device__ inline double lp_xor64(double x, int m) { return __longlong_as_double((long long)tg_shfl_xor64((u64)__double_as_longlong(x), m)); }

// A wave's k best so far, the i-th in lane i: by logit, then by row.
struct LpBest {
    static constexpr int NONE = 0x7FFFFFFF;
    double z;
    int row;
    int k;
    double last_z;               // the k-th
    int last_row;

    __device__ inline void begin(int count)
    {
        z = last_z = 0.0;             // (no 64-bit infinity: hipcc 7.2 moves such a constant into scalar registers by an instruction that holds 32 bits of it)
        row = last_row = NONE;
        k = count;
    }
    // (a place without a row is behind all)
    static __device__ inline bool before(double az, int ar, double bz, int br) { return br == NONE ? ar != NONE : ar != NONE && (az > bz || (az == bz && ar < br)); }
    // whether a row of a logit up to `most` is worth a look (what a NaN says nothing of is)
    __device__ inline bool wants(double most, int r) const { return last_row == NONE || !(most < last_z || (most == last_z && r > last_row)); }
    // (the same in all lanes)
    __device__ inline void add(double cz, int cr)
    {
        if (!before(cz, cr, last_z, last_row)) return;
        const u64 ahead = __ballot(before(z, row, cz, cr));
        const int at = __popcll(ahead);             // (in order: those ahead are the first lanes)
        const double up_z = __longlong_as_double((long long)tg_shfl64((u64)__double_as_longlong(z), (tg_lane() + 63) & 63));
        const int up_row = __shfl(row, (tg_lane() + 63) & 63);
        if (tg_lane() == at) {
            z = cz;
            row = cr;
        } else if (tg_lane() > at) {
            z = up_z;
            row = up_row;
        }
        last_z = lp_lane64(z, k - 1);
        last_row = __builtin_amdgcn_readlane(row, k - 1);
    }
};

struct LpTop {
    const void *h, *w;           // the caller's
    int64_t ld_h, ld_w;
    int d, tile_shift, per_shift, half_shift;     // log2 of a tile's rows, of its groups, and of the blocks of 16 rows that a wave has in half of a tile
    int top;
    const float* norms;          // one a tile
    const uint2* groups;
    int n_groups;                // below 2^28
    int32_t* rows;
    float* row_logp;
};

// R rows' logits in 64 bits, by one wave: row i's in the lanes 64 / R i and on.  Every lane has the same places of all rows, so a row's sum does not depend
// on where it was found.
template <int R, class E>
__device__ inline double lp_score(const LpTop& a, const E* h, double scale, const int (&rows)[R])
{
    typedef TgPiece<E> P;
    const int lane = tg_lane();
    const E* w[R];
#pragma unroll
    for (int i = 0; i < R; ++i) w[i] = (const E*)a.w + (int64_t)__builtin_amdgcn_readfirstlane(rows[i]) * a.ld_w;
    double sum[R] = {};
    for (int c = lane * P::E; c < a.d; c += 64 * P::E) {
        typename P::vec x[R];
        P hp;
#pragma unroll
        for (int i = 0; i < R; ++i) x[i] = P::raw(w[i] + c, a.d - c);
        hp.load(h + c, a.d - c);
#pragma unroll
        for (int e = 0; e < P::E; ++e)
#pragma unroll
            for (int i = 0; i < R; ++i) sum[i] = fma((double)hp.v[e], (double)(float)x[i][e], sum[i]);
    }
    // half of the rows goes to either half of the lanes, as long as there are two
#pragma unroll
    for (int left = R, m = 32; m >= 1; m >>= 1) {
        if (left > 1) {
            left /= 2;
#pragma unroll
            for (int i = 0; i < left; ++i) sum[i] = (lane & m ? sum[i + left] : sum[i]) + lp_xor64(lane & m ? sum[i] : sum[i + left], m);
        } else sum[0] += lp_xor64(sum[0], m);
    }
    return sum[0] * scale;
}

// The groups of a token that reach `least` with their tile's margin, as a wave goes through them: W waves in turn, LP_AHEAD times 64 tiles' maxima asked for at once, then the groups of those
// tiles that do.  Some lanes' groups at a time: take(whether the lane has one, its number, its largest, its packed second, its margin).  look(a tile's maximum and its margin, its number): whether its
// groups are still of interest.
#define LP_AHEAD 8
template <int W, class Margin, class Look, class Take>
__device__ inline void lp_reach(const float4* __restrict__ parts, const float* __restrict__ norms, int tiles, const uint2* __restrict__ groups, int per_shift, int wave, double least,
                                const Margin& margin, Look look, Take take)
{
    for (int t0 = wave * 64 + tg_lane(); t0 - tg_lane() < tiles; t0 += LP_AHEAD * 64 * W) {
        float v[LP_AHEAD], w2[LP_AHEAD];
#pragma unroll
        for (int i = 0; i < LP_AHEAD; ++i) {
            v[i] = t0 + i * 64 * W < tiles ? parts[t0 + i * 64 * W].x : 0.0f;
            w2[i] = t0 + i * 64 * W < tiles ? norms[t0 + i * 64 * W] : 0.0f;
        }
        unsigned hits = 0;
#pragma unroll
        for (int i = 0; i < LP_AHEAD; ++i) hits |= t0 + i * 64 * W < tiles && !((double)v[i] + margin.of(w2[i]) < least) ? 1u << i : 0u;      // (what a NaN is compared with is not out of reach)
        for (; __any(hits != 0); hits &= hits - 1) {
            const int i = hits ? __builtin_ctz(hits) : 0, t = t0 + i * 64 * W;
            float max = v[0], square = w2[0];
#pragma unroll
            for (int j = 1; j < LP_AHEAD; ++j) {
                max = i == j ? v[j] : max;
                square = i == j ? w2[j] : square;
            }
            const double off = margin.of(square);
            const bool in = hits && look((double)max + off, t);
            if (!__any(in)) continue;
            for (int g0 = t << per_shift, end = 0; end < 1 << per_shift; g0 += 8, end += 8) {        // (8 or 16 a tile)
                uint2 q[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) q[j] = in ? groups[g0 + j] : make_uint2(0u, 0u);
                unsigned deep = 0;
#pragma unroll
                for (int j = 0; j < 8; ++j) deep |= in && !((double)__uint_as_float(q[j].x) + off < least) ? 1u << j : 0u;
                for (; __any(deep != 0); deep &= deep - 1) {
                    const int at = deep ? __builtin_ctz(deep) : 0;
                    uint2 x = q[0];
#pragma unroll
                    for (int j = 1; j < 8; ++j) x = at == j ? q[j] : x;
                    take(deep != 0, g0 + at, __uint_as_float(x.x), x.y, off);
                }
            }
        }
    }
}
// a group's rows, and its row number `lane` below that: value lane % 4 of the lane's block lane / 4, as lp_part_kernel has them
__device__ inline int lp_group_rows(const LpTop& a) { return 8 << a.half_shift; }
__device__ inline int lp_group_row(const LpTop& a, int g, int lane)
{
    const int tile = g >> a.per_shift, in = g & ((1 << a.per_shift) - 1), i = lane >> 2;
    return (tile << a.tile_shift) + ((i >> a.half_shift) << (a.tile_shift - 1)) + ((in >> 2) << (a.half_shift + 4)) + (i & ((1 << a.half_shift) - 1)) * 16 + (in & 3) * 4 + (lane & 3);
}

// The tiles' sums joined, and the best rows, by W waves a token: eight where there are few tokens (one token, 1024 tiles: 13 us, of which ways to memory, one behind the other, are most), one where
// there are many (4096, 512 tiles: 39 to 54 us by what the caches still hold, 191 to 202 with eight; 1003, 587 smaller tiles: 16 and 38).  Four waves a SIMD, at some 50 registers spilt in the rare paths:
// three take 49 to 60.
//
// What is not below the threshold is listed and scored, eight rows at a time a wave; a long list is thinned by the k-th of its lanes' largest, and a row's place is the number of those
// before it (23 tokens, 553 rows, 20 best: 32 us with the call, 283 through sorted lists of a wave).  Where the list does not hold
// them (rows that are equal, or nearly, by the hundreds) every wave goes through its groups again with its k best so far in order in its lanes, and passes over
// what cannot be among them.
template <class E, int W, bool TOP>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W, W == 1 ? 4 : 1) void lp_join_kernel(const float4* __restrict__ parts, int64_t count, int64_t n, int64_t n_rows,
                                                                       const void* __restrict__ targets, int targets64, const float* __restrict__ at_target,
                                                                       float scale, LpTop a, float* __restrict__ logp, float* __restrict__ entropy,
                                                                       float* __restrict__ lse)
{
    constexpr int TOKENS = W == 1 ? 4 : 1;
    constexpr int LIST = W == 1 ? 512 : 1024;
    __shared__ float s_m[W], s_l[W], s_s[W];
    __shared__ double s_h2[W];
    __shared__ float2 s_top[W > 1 ? W : 1][W > 1 ? 64 : 1];
    __shared__ int s_list[TOP ? TOKENS : 1][TOP ? LIST : 1];
    __shared__ double s_z[TOP ? TOKENS : 1][TOP ? LIST : 1];
    __shared__ int s_found, s_zero[W];
    const int lane = tg_lane(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int of = W == 1 ? lane : threadIdx.x;                  // of the token's lanes
    const int mine = W == 1 ? 0 : wave, team = W == 1 ? wave : 0;
    for (int64_t y = (int64_t)blockIdx.x * TOKENS + team; y < n; y += (int64_t)gridDim.x * TOKENS) {
        const E* const h = (const E*)a.h + y * a.ld_h;
        const float4* const own = parts + y * count;
        const uint2* const groups = a.groups + y * (int64_t)a.n_groups;
        // the token's square, its first pieces asked for in front of everything
        double h2 = 0.0;
        bool zero = true;                        // a row of zeros (padding): its logits are exact, and all equal (as with a factor of 0)
        typedef TgPiece<E> P;
        typename P::vec h_first;
        if (TOP) h_first = P::raw(h + (of * P::E < a.d ? of * P::E : 0), a.d - of * P::E);
        LpSum sum{-__builtin_inff(), 0.0f, 0.0f};
        // The largest of the lane's, and the square of its tile: the tiles' maxima, or, where they are so few that many tiles have two of the best, the groups'.
        const bool by_tile = count >= 4 * a.top;
        float high = -__builtin_inff(), high_w2 = 0.0f;
        for (int64_t p0 = of; p0 < count; p0 += 4 * 64 * W) {
            float4 v[4];
            float w2[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[i] = p0 + i * 64 * W < count ? own[p0 + i * 64 * W] : make_float4(-__builtin_inff(), 0.0f, 0.0f, 0.0f);
                if (TOP) w2[i] = a.norms[p0 + i * 64 * W < count ? p0 + i * 64 * W : 0];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                lp_join(sum, LpSum{v[i].x, v[i].y, v[i].z});
                if (TOP && by_tile && v[i].x > high) {
                    high = v[i].x;
                    high_w2 = w2[i];
                }
            }
        }
        if (TOP) {
#pragma unroll
            for (int e = 0; e < P::E; ++e) {
                h2 = fma((double)(float)h_first[e], (double)(float)h_first[e], h2);
                zero = zero && h_first[e] == (E)0.0f;
            }
            for (int c = (of + 64 * W) * P::E; c < a.d; c += 64 * W * P::E) {
                P p;
                p.load(h + c, a.d - c);
#pragma unroll
                for (int e = 0; e < P::E; ++e) {
                    h2 = fma((double)p.v[e], (double)p.v[e], h2);
                    zero = zero && p.v[e] == 0.0f;
                }
            }
            zero = __all(zero);
            if (!by_tile)
                for (int g = of; g < a.n_groups; g += 64 * W) {
                    const float m = __uint_as_float(groups[g].x), w2 = a.norms[g >> a.per_shift];
                    if (m > high) {
                        high = m;
                        high_w2 = w2;
                    }
                }
        }
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            lp_join(sum, LpSum{__shfl_xor(sum.m, m), __shfl_xor(sum.l, m), __shfl_xor(sum.s, m)});
            if (TOP) h2 += lp_xor64(h2, m);
        }
        if (W > 1) {
            __syncthreads();                                     // (the token before is done with these)
            if (lane == 0) {
                s_m[wave] = sum.m;
                s_l[wave] = sum.l;
                s_s[wave] = sum.s;
                s_h2[wave] = h2;
                s_zero[wave] = zero;
            }
            if (threadIdx.x == 0) s_found = 0;
            if (TOP) s_top[wave][lane] = make_float2(high, high_w2);
            __syncthreads();
            // (every wave has all waves' W times over)
            sum = LpSum{s_m[lane % W], s_l[lane % W], s_s[lane % W]};
            h2 = s_h2[lane % W];
            zero = __all(s_zero[lane % W] != 0);
#pragma unroll
            for (int m = 1; m < W; m <<= 1) {
                lp_join(sum, LpSum{__shfl_xor(sum.m, m), __shfl_xor(sum.l, m), __shfl_xor(sum.s, m)});
                if (TOP) h2 += lp_xor64(h2, m);
            }
            if (TOP) {
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    const float2 x = s_top[i][lane];
                    high_w2 = x.x > high ? x.y : high_w2;
                    high = fmaxf(high, x.x);
                }
            }
        }
        // (the first lane's: the others joined the same in other orders)
        const float all = __uint_as_float((lp_u32)__builtin_amdgcn_readfirstlane((int)__float_as_uint(sum.m + logf(sum.l))));
        if (of == 0) {
            lse[y] = all;
            const float below = logf(sum.l) - 0.6931471805599453f * (sum.s / sum.l);
            // (probabilities of infinite logits are not defined)
            entropy[y] = fabsf(all) <= 3.4028234e38f ? fmaxf(below, 0.0f) : __builtin_nanf("");
            // (without a list of targets nobody has one; lse, rounded, can be below the largest logit)
            if (logp) {
                const float p = targets && tg_row_of(targets, targets64, y, n_rows) >= 0 ? at_target[y] - all : 0.0f;
                logp[y] = p > 0.0f ? 0.0f : p;
            }
        }
        if (!TOP) continue;
        const auto put = [&](int place, double z, int row) {
            const double p = z - (double)all;
            a.rows[y * a.top + place] = row == LpBest::NONE ? -1 : row;
            a.row_logp[y * a.top + place] = row == LpBest::NONE ? -__builtin_inff() : (float)(p > 0.0 ? 0.0 : p);
        };
        if (all != all) {                                        // a NaN among the logits
            if (of < a.top) {
                a.rows[y * a.top + of] = -1;
                a.row_logp[y * a.top + of] = all;
            }
            continue;
        }
        // What the k-th best logit is not below: the lanes' largest, a margin down (one that is infinite may have been made so by the last step).  A row is out of reach where a margin more does not
        // bring it there; margins are those of its tile, so that a few rows far longer than the others make nothing of theirs hard to tell apart.
        const LpMargin<E> margin(scale, a.d, h2, zero || scale == 0.0f);
        const float kth = lp_kth((float)((double)fminf(high, 3.4028234e38f) - margin.of(high_w2)), a.top);
        const double low = (double)kth - (fabs((double)kth) * 0x1p-22 + 0x1p-140);       // (32 bits of it: a step down)
        int* const list = s_list[TOP ? team : 0];
        double* const score = s_z[TOP ? team : 0];
        int found = 0;
        // `some` rows more for the list: the place of the first, and of what is behind the last
        const auto room = [&](int some) {
            int at = found;
            if (W > 1) {
                if (lane == 0) at = atomicAdd(&s_found, some);
                at = __builtin_amdgcn_readfirstlane(at);
            }
            found = at + some;
            return at;
        };
        lp_reach<W>(own, a.norms, (int)count, groups, a.per_shift, mine, low, margin, [&](double, int) { return found <= LIST; }, [&](bool hit, int g, float, lp_u32 second, double off) {
            const bool alone = (double)lp_second(second) + off < low;
            u64 many = __ballot(hit && !alone);
            const int row = (g >> a.per_shift << a.tile_shift) + lp_row(second);
            const u64 one = __ballot(hit && alone && row < (int)n_rows);
            if (one) {
                const int at = room(__popcll(one)) + __popcll(one & tg_lanemask_lt());
                if ((one >> lane & 1) && at < LIST) list[at] = row;
            }
            for (; many && found <= LIST; many &= many - 1) {
                const int r = lp_group_row(a, __builtin_amdgcn_readlane(g, __builtin_ctzll(many)), lane);
                const u64 some = __ballot(lane < lp_group_rows(a) && r < (int)n_rows);
                const int at = room(__popcll(some)) + __popcll(some & tg_lanemask_lt());
                if ((some >> lane & 1) && at < LIST) list[at] = r;
            }
        });
        if (W > 1) {
            __syncthreads();
            found = s_found;
        } else __builtin_amdgcn_wave_barrier();
        if (__builtin_expect(found <= LIST, 1)) {
            const auto some = [&](auto rows) {
                constexpr int R = sizeof(rows) / sizeof(int);
                for (int c0 = mine; c0 < found; c0 += R * W) {
#pragma unroll
                    for (int i = 0; i < R; ++i) rows.v[i] = list[c0 + i * W < found ? c0 + i * W : c0];
                    const double z = lp_score<R, E>(a, h, (double)scale, rows.v);
                    const int c = c0 + lane / (64 / R) * W;
                    if (lane % (64 / R) == 0 && c < found) score[c] = z;
                }
            };
            struct Two { int v[2]; };
            struct Eight { int v[8]; };
            if (W > 1 && found <= 2 * W) some(Two{});
            else some(Eight{});
            if (W > 1) __syncthreads();
            else __builtin_amdgcn_wave_barrier();
            if (mine != 0) continue;
            if (found > 64) {
                // those that the k-th of the lanes' largest does not rule out, to the front (32 bits of them: a step down)
                float largest = -__builtin_inff();
                for (int c = lane; c < found; c += 64) largest = fmaxf(largest, (float)score[c]);
                const float last = lp_kth(largest, a.top);
                const double least = (double)last - fabs((double)last) * 0x1p-22 - 0x1p-140;
                int kept = 0;
                for (int c0 = 0; c0 < found; c0 += 64) {
                    const int c = c0 + lane < found ? c0 + lane : 0;
                    const double z = score[c];
                    const int row = list[c];
                    const u64 in = __ballot(c0 + lane < found && !(z < least));
                    __builtin_amdgcn_wave_barrier();
                    if (in >> lane & 1) {
                        score[kept + __popcll(in & tg_lanemask_lt())] = z;
                        list[kept + __popcll(in & tg_lanemask_lt())] = row;
                    }
                    __builtin_amdgcn_wave_barrier();
                    kept += __popcll(in);
                }
                found = kept;
            }
            for (int c = lane; c < found || c < a.top; c += 64) {
                if (c >= found) {
                    put(c, 0.0, LpBest::NONE);
                    continue;
                }
                const double z = score[c];
                const int row = list[c];
                int place = 0;
                for (int i0 = 0; i0 < found; i0 += 8) {
                    double zs[8];
                    int rows[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        zs[i] = score[i0 + i];
                        rows[i] = list[i0 + i];
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) place += i0 + i < found && (zs[i] > z || (zs[i] == z && rows[i] < row)) ? 1 : 0;
                }
                if (place < a.top) put(place, z, row);
            }
            continue;
        }
        LpBest best;
        best.begin(a.top);
        const auto look = [&](double most, int t) { return best.wants(most, t << a.tile_shift); };
        lp_reach<W>(own, a.norms, (int)count, groups, a.per_shift, mine, low, margin, look, [&](bool hit, int g, float first, lp_u32 second, double off) {
            const int row0 = g >> a.per_shift << a.tile_shift;
            u64 hits = __ballot(hit && best.wants((double)first + off, row0));
            const u64 many = __ballot(!((double)lp_second(second) + off < low));
            for (; hits; hits &= hits - 1) {
                const int from = __builtin_ctzll(hits);
                const double most = lp_lane64((double)first + off, from);
                const bool all_rows = many >> from & 1;
                const int r = all_rows ? lp_group_row(a, __builtin_amdgcn_readlane(g, from), lane) : __builtin_amdgcn_readlane(row0 + lp_row(second), from);
                u64 some = __ballot(lane < (all_rows ? lp_group_rows(a) : 1) && r < (int)n_rows && best.wants(most, r));
                while (some) {
                    int rows[8], have = 0;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        rows[i] = some ? __builtin_amdgcn_readlane(r, __builtin_ctzll(some)) : rows[0];
                        have += some ? 1 : 0;
                        some &= some - 1;
                    }
                    const double z = lp_score<8, E>(a, h, (double)scale, rows);
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (i < have) best.add(lp_lane64(z, i * 8), rows[i]);
                }
            }
        });
        if (W > 1) {
            // the waves' lists, one behind the other, to the first
            for (int i = 1; i < W; ++i) {
                if (wave == i && lane < a.top) {
                    score[lane] = best.z;
                    list[lane] = best.row;
                }
                __syncthreads();
                if (wave == 0)
                    for (int j = 0; j < a.top; ++j) {
                        const double z = score[j];
                        const int r = __builtin_amdgcn_readfirstlane(list[j]);
                        if (r == LpBest::NONE || !best.wants(z, r)) break;        // (theirs are in order too)
                        best.add(z, r);
                    }
                __syncthreads();
            }
        }
        if (mine == 0 && lane < a.top) put(lane, best.z, best.row);
    }
}

// ---- workspaces and launches
struct LpShape {
    int bm, bn, groups;          // the tile, and its groups
    bool few;                    // four stages in flight
    int64_t tiles;               // along the table
    int64_t tokens;              // at a time
};
// tokens at a time: as many as the groups' stretches have room for, in whole tiles
#define LP_GROUP_BYTES (1ll << 30)

static LpShape lp_shape(int64_t n, int64_t n_rows, int e, int top)
{
    LpShape s;
    // The tiles of the cross entropy's logits; but where the best rows are asked for those of 128 rows, which have the norms' squares beside their products, up to 384 tokens
    // (131 072 rows of 1024 bf16, 8 best: 100 tokens 122 us in tiles of 256 rows behind a pass for the norms, 77 in these; 300: 202 and 178; 512: the other way round).
    int64_t most = LP_GROUP_BYTES / (int64_t)sizeof(uint2) / ((n_rows + LP_GROUP_LEAST - 1) / LP_GROUP_LEAST);
    most = most >= 256 ? most / 256 * 256 : most >= 64 ? 64 : n_rows <= 1ll << 28 ? 32 : 8;        // (2^28 rows: 8 GiB for 32 tokens)
    s.tokens = n < most ? n : most;
    const auto tiles = [&](int64_t x, int64_t y) { return ((n_rows + x - 1) / x) * ((s.tokens + y - 1) / y); };
    // A CU holds one tile of 256 x 256, or two of 128 x 128, which take 1.28 times as long for as many logits: the smaller ones where the larger leave more of their last round, or of
    // their last tokens, unused (bf16: 300 tokens, 40 000 rows of 512: 38.0 us in the larger, 30.2 in the smaller; 8192, 3000 of 1000, 3 best: 154 and 143; 2003, 50 257 of 500: 158 and 176).
    const auto rounds = [](int64_t count, int64_t at_once) { return (count + at_once - 1) / at_once; };
    const bool larger = (double)rounds(tiles(256, 256), 256) * 256 * 65536 <= 1.28 * (double)rounds(tiles(128, 128), 512) * 512 * 16384;
    s.few = tiles(128, 128) <= 128;
    if (s.tokens <= 32) s.bm = 128, s.bn = 32, s.groups = 16;
    else if (s.few || (e == 4 && s.tokens > 64)) s.bm = 64, s.bn = 64, s.groups = 8;
    else if (s.tokens <= 64) s.bm = 128, s.bn = 64, s.groups = 16;
    else if ((!top || (s.tokens > 384 && n_rows >= 256 * (int64_t)top)) && tiles(256, 256) >= 200 && larger) s.bm = 256, s.bn = 256, s.groups = 8;
    else s.bm = 128, s.bn = 128, s.groups = 8;
    s.tiles = (n_rows + s.bm - 1) / s.bm;
    return s;
}
struct LpSpace {
    TileRows h, w;
    void *ph, *pw;               // copies, or null
    float4* parts;
    float *at_target, *norms;
    int64_t n_norms;             // stretches of the table with a largest square of a norm each
    uint2* groups;
};
static size_t carve_lp(LpSpace* r, TgCarve* c, const LpShape& s, const void* h, int64_t ld_h, const void* w, int64_t ld_w, int64_t n, int64_t n_rows, int d, int e,
                       bool ready_h, bool ready_w, int top)
{
    const uint32_t pitch = tile_pitch(d, e);
    r->ph = ready_h ? nullptr : c->take<char>((size_t)n * pitch);
    r->pw = ready_w ? nullptr : c->take<char>((size_t)n_rows * pitch);
    r->h = ready_h ? TileRows{(const char*)h, n, (uint32_t)(ld_h * e), pitch} : TileRows{(const char*)r->ph, n, pitch, pitch};
    r->w = ready_w ? TileRows{(const char*)w, n_rows, (uint32_t)(ld_w * e), pitch} : TileRows{(const char*)r->pw, n_rows, pitch, pitch};
    r->parts = c->take<float4>((size_t)s.tiles * s.tokens);
    r->at_target = c->take<float>(s.tokens);
    r->n_norms = s.tiles;
    r->norms = c->take<float>(top ? r->n_norms : 0);
    r->groups = c->take<uint2>(top ? (size_t)s.tiles * s.groups * s.tokens : 0);
    return c->used;
}
size_t tg_log_probs_space(int64_t n, int64_t n_rows, int d, int dtype, int top, int aligned)
{
    if (n == 0) return 0;
    const int e = (int)tg_type_bytes(dtype);
    TgCarve c{nullptr, 0};
    LpSpace r;
    const bool whole = (d * e & 15) == 0;
    return carve_lp(&r, &c, lp_shape(n, n_rows, e, top), nullptr, d, nullptr, d, n, n_rows, d, e, whole && (aligned == 1 || aligned == 3),
                    whole && (aligned == 1 || aligned == 2), top);
}

struct LpCall {
    const void* targets;         // of the tokens at hand
    int targets64;
    float scale;
    bool first;                  // of the calls for a table
    hipStream_t s;
};
template <class E, int BM, int BN, int WM, int WN, int NB, bool TOP>
static void launch_parts(const LpShape& shape, const LpSpace& r, const TileRows& Y, const LpCall& call)
{
    // as many tiles along the table as a launch's work-items allow (all of them up to 2^29 rows), then as many tokens
    constexpr int64_t TILES = TILE_LAUNCH_ITEMS / (64 * WM * WN);
    const TileRows& X = r.w;
    for (int64_t t0 = 0; t0 < shape.tiles; t0 += TILES) {
        const int64_t tiles = shape.tiles - t0 < TILES ? shape.tiles - t0 : TILES, v0 = t0 * BM, most = TILES / tiles * BN;
        const TileRows table{X.p + v0 * X.pitch, X.rows - v0 < tiles * BM ? X.rows - v0 : tiles * BM, X.pitch, X.width};
        for (int64_t y0 = 0; y0 < Y.rows; y0 += most) {
            const int64_t rows = Y.rows - y0 < most ? Y.rows - y0 : most;
            const uint32_t ny = (uint32_t)((rows + BN - 1) / BN);
            const TileRows part{Y.p + y0 * Y.pitch, rows, Y.pitch, Y.width};
            hipLaunchKernelGGL((lp_part_kernel<E, BM, BN, WM, WN, NB, TOP>), dim3((unsigned)(tiles * ny)), dim3(64 * WM * WN), 0, call.s, table, part, (int)X.width,
                               call.targets ? (const char*)call.targets + y0 * (call.targets64 ? 8 : 4) : nullptr, call.targets64, call.scale, v0, X.rows,
                               (uint32_t)tiles, ny, 8u, r.parts + y0 * shape.tiles + t0, shape.tiles,
                               TOP ? r.groups + (y0 * shape.tiles + t0) * shape.groups : nullptr,
                               y0 == 0 && call.first ? r.norms + t0 : nullptr, r.at_target + y0);
        }
    }
}
template <class E, bool TOP>
static void launch_all_parts(const LpShape& shape, const LpSpace& r, const TileRows& Y, const LpCall& call)
{
    if (shape.bn == 32) {
        if (shape.few) launch_parts<E, 128, 32, 4, 1, 4, TOP>(shape, r, Y, call);
        else launch_parts<E, 128, 32, 4, 1, 2, TOP>(shape, r, Y, call);
    } else if (shape.bm == 64) {
        if (shape.few) launch_parts<E, 64, 64, 2, 2, 4, TOP>(shape, r, Y, call);
        else if constexpr (sizeof(E) == 4) launch_parts<E, 64, 64, 2, 2, 2, TOP>(shape, r, Y, call);
    } else if (shape.bn == 64) launch_parts<E, 128, 64, 4, 1, 2, TOP>(shape, r, Y, call);
    else if constexpr (sizeof(E) == 2) {
        if (shape.bm == 256) launch_parts<E, 256, 256, 2, 4, 2, TOP>(shape, r, Y, call);
        else launch_parts<E, 128, 128, 2, 2, 2, TOP>(shape, r, Y, call);
    }
}
template <class E, bool TOP>
static void launch_join(const LpShape& shape, const LpSpace& r, int64_t n, int64_t n_rows, const LpTop& a, const LpCall& call, float* logp, float* entropy, float* lse)
{
    const auto go = [&](auto kernel, int waves) {
        const int64_t wgs = waves == 1 ? (n + 3) / 4 : n;
        hipLaunchKernelGGL(kernel, dim3((unsigned)(wgs < 65536 ? wgs : 65536)), dim3(waves == 1 ? 256 : 64 * waves), 0, call.s, r.parts, shape.tiles, n, n_rows,
                           call.targets, call.targets64, r.at_target, call.scale, a, logp, entropy, lse);
    };
    if (n <= 256) go(lp_join_kernel<E, 8, TOP>, 8);
    else go(lp_join_kernel<E, 1, TOP>, 1);
}

void tg_launch_log_probs(const void* h, int64_t ld_h, const void* w, int64_t ld_w, int dtype, int64_t n, int64_t n_rows, int d, const void* targets,
                         int targets64, float scale, int top, float* logp, float* entropy, float* lse, int32_t* rows, float* row_logp, void* space,
                         hipStream_t s)
{
    const int e = (int)tg_type_bytes(dtype);
    const LpShape shape = lp_shape(n, n_rows, e, top);
    TgCarve c{(char*)space, 0};
    LpSpace r;
    const bool rh = tile_ready(h, ld_h, d, e), rw = tile_ready(w, ld_w, d, e);
    carve_lp(&r, &c, shape, h, ld_h, w, ld_w, n, n_rows, d, e, rh, rw, top);
    if (!rh) tg_launch_pack(h, ld_h, n, d, e, r.ph, s);
    if (!rw) tg_launch_pack(w, ld_w, n_rows, d, e, r.pw, s);
    // (a group has bm / groups rows, in blocks of 4: half of them in either half of the tile)
    LpTop a{h, w, ld_h, ld_w, d, __builtin_ctz(shape.bm), __builtin_ctz(shape.groups), __builtin_ctz(shape.bm / shape.groups / 8), top, r.norms, r.groups,
            (int)(shape.tiles * shape.groups), rows, row_logp};
    TG_WITH_TYPE(dtype, E, {
        if constexpr (sizeof(E) == 2) {
            if (top && shape.bm == 256) {
                int lanes = 1;
                while (lanes < 64 && lanes * TgPiece<E>::E < d) lanes *= 2;
                hipLaunchKernelGGL(lp_norms_kernel<E>, dim3((unsigned)(r.n_norms < 65536 ? r.n_norms : 65536)), dim3(1024), 0, s, (const E*)w, ld_w, n_rows, d,
                                   lanes, r.norms, r.n_norms);
            }
        }
        for (int64_t y0 = 0; y0 < n; y0 += shape.tokens) {
            const int64_t now = n - y0 < shape.tokens ? n - y0 : shape.tokens;
            const LpCall call{targets ? (const char*)targets + y0 * (targets64 ? 8 : 4) : nullptr, targets64, scale, y0 == 0, s};
            const TileRows Y{r.h.p + y0 * r.h.pitch, now, r.h.pitch, r.h.width};
            a.h = (const E*)h + y0 * ld_h;
            a.rows = top ? rows + y0 * top : nullptr;
            a.row_logp = top ? row_logp + y0 * top : nullptr;
            float* const out = logp ? logp + y0 : nullptr;
            if (top) {
                launch_all_parts<E, true>(shape, r, Y, call);
                launch_join<E, true>(shape, r, now, n_rows, a, call, out, entropy + y0, lse + y0);
            } else {
                launch_all_parts<E, false>(shape, r, Y, call);
                launch_join<E, false>(shape, r, now, n_rows, a, call, out, entropy + y0, lse + y0);
            }
        }
    });
}
