// Rows of a table by id, and the gradient that goes back to them.
//
// The lookup is a copy: bound by its bytes (65 536 rows of 1024 bf16 out of 131 072, all as frequent: 42 us, 6.4 TB/s;
// where few take most of the tokens 32).  The gradient is a sum over the tokens of an id.  Adding them to the table with atomics
// would make the result depend on the order of arrival and, where few ids take most tokens, wait for the same words; so the
// tokens are sorted by id (ties by position) and the sorted list is cut into tiles of equal length, whatever the ids: a run of one id that lies inside a
// tile is written at once, one that crosses tiles leaves its parts in fp32 and is added up by a second kernel in the tiles' order.
#include "tg_embed.h"
#include "tg_device.h"

#define LOOKUP_GRID 65536          // workgroups of a launch at most: the rest is walked

// ---- lookup: G lanes (a power of two) a row
template <class E>
__global__ __launch_bounds__(256) void lookup_kernel(const E* __restrict__ table, int64_t ld, int64_t n_rows, int d, const void* __restrict__ ids,
                                                     int ids64, int64_t n, float scale, int gshift, E* __restrict__ out)
{
    typedef TgPiece<E> P;
    const int lane = threadIdx.x & ((1 << gshift) - 1);
    const int64_t step = (int64_t)gridDim.x * (256 >> gshift);
    for (int64_t t = (int64_t)blockIdx.x * (256 >> gshift) + (threadIdx.x >> gshift); t < n; t += step) {
        const int64_t v = tg_row_of(ids, ids64, t, n_rows);
        for (int at = lane * P::E; at < d; at += P::E << gshift) {
            P p;
            p.load(table + (v < 0 ? 0 : v) * ld + at, v < 0 ? 0 : d - at);
#pragma unroll
            for (int i = 0; i < P::E; ++i) p.v[i] *= v < 0 ? 0.0f : scale;       // (no row is zero at any scale)
            p.store(out + t * d + at, d - at);
        }
    }
}

static int lanes_shift(int pieces)
{
    int s = 0;
    while (s < 6 && (1 << s) < pieces) ++s;
    return s;
}

void tg_launch_lookup(const void* table, int64_t ld, int dtype, int64_t n_rows, int d, const void* ids, int ids64, int64_t n, float scale,
                      void* out, hipStream_t s)
{
    if (n == 0) return;
    TG_WITH_TYPE(dtype, E, {
        const int gs = lanes_shift((d + TgPiece<E>::E - 1) / TgPiece<E>::E);
        const int64_t wgs = (n + (256 >> gs) - 1) / (256 >> gs);
        hipLaunchKernelGGL(lookup_kernel<E>, dim3((unsigned)(wgs < LOOKUP_GRID ? wgs : LOOKUP_GRID)), dim3(256), 0, s, (const E*)table, ld, n_rows,
                           d, ids, ids64, n, scale, gs, (E*)out);
    });
}

// ---- zeros: `halves` values of 16 bits, the first `head` of them in front of a 16-byte boundary.  The sort has few workgroups and
// waits for memory most of the time, so the gradient's rows are cleared beside it: every launch of it takes a part of them.
struct ZeroPart {
    uint16_t* p;
    size_t halves, head;
    uint32_t part, parts;        // which part of the 16-byte pieces this launch clears
    uint32_t first;              // its workgroups are the ones from here on
};
__device__ inline void zero_part(const ZeroPart& z)
{
    const size_t i = (size_t)(blockIdx.x - z.first) * blockDim.x + threadIdx.x, step = (size_t)(gridDim.x - z.first) * blockDim.x;
    uint4* q = reinterpret_cast<uint4*>(z.p + z.head);
    const size_t pieces = (z.halves - z.head) / 8, from = pieces * z.part / z.parts, to = pieces * (z.part + 1) / z.parts;
    for (size_t j = from + i; j < to; j += step) q[j] = make_uint4(0, 0, 0, 0);
    if (z.part) return;
    if (i < z.head) z.p[i] = 0;
    if (i < (z.halves - z.head) % 8) z.p[z.head + pieces * 8 + i] = 0;
}
__global__ __launch_bounds__(256) void zero_kernel(ZeroPart z) { zero_part(z); }
static ZeroPart zero_of(void* p, size_t bytes)
{
    ZeroPart z{(uint16_t*)p, bytes / 2, ((16 - ((uintptr_t)p & 15)) & 15) / 2, 0, 1, 0};
    if (z.head > z.halves) z.head = z.halves;
    return z;
}
// workgroups that clear a part: 16 KB each, up to 2048
static unsigned zero_wgs(const ZeroPart& z)
{
    if (z.halves == 0) return 0;
    const size_t w = z.halves / 8192 / z.parts + 1;
    return (unsigned)(w < 2048 ? w : 2048);
}
void tg_launch_zero(void* p, size_t bytes, hipStream_t s)
{
    const ZeroPart z = zero_of(p, bytes);
    if (z.halves) hipLaunchKernelGGL(zero_kernel, dim3(zero_wgs(z)), dim3(256), 0, s, z);
}

// ---- the tokens sorted by id.  A token without a row gets the key n_rows and ends up behind the others.
__device__ inline u32 token_key(const void* ids, int ids64, int64_t t, int64_t n_rows)
{
    const int64_t v = tg_row_of(ids, ids64, t, n_rows);
    return (u32)(v < 0 ? n_rows : v);
}

// Few tokens: the place of a token is the number of those in front of it, counted.  16 lanes count for one token, over all keys in LDS.
// One launch instead of the four of the digits' sort: at 4000 tokens and rows of 50 fp32 20 against 26 us of the whole gradient, at 6000 25 against 27,
// at 8000 30 against 26.
#define RANK_MAX 6144
__global__ __launch_bounds__(256) void rank_sort_kernel(const void* __restrict__ ids, int ids64, int n, int64_t n_rows, u32* __restrict__ skey,
                                                        u32* __restrict__ spos, u32* __restrict__ runs, ZeroPart z)
{
    if (blockIdx.x >= z.first) { zero_part(z); return; }
    if (blockIdx.x == 0 && threadIdx.x < 2) runs[threadIdx.x] = 0;
    extern __shared__ __align__(16) u32 s_rank_keys[];      // n rounded up to 64, the rest larger than any key
    const int full = (n + 63) & ~63;
    for (int i = threadIdx.x; i < full; i += 256) s_rank_keys[i] = i < n ? token_key(ids, ids64, i, n_rows) : 0xFFFFFFFFu;
    __syncthreads();
    const int part = threadIdx.x & 15;
    const int t = blockIdx.x * 16 + (threadIdx.x >> 4);
    if (t >= n) return;                                     // (16 lanes together: their sums stay among themselves)
    const u32 key = s_rank_keys[t];
    // in front of the token equal keys count, behind it they do not: up to its own 64 keys, and from them on, one comparison each
    int before = 0;
    const int own = t & ~63;
    for (int i = part * 4; i < own; i += 64) {
        const uint4 k = *reinterpret_cast<const uint4*>(s_rank_keys + i);
        before += (int)(k.x <= key) + (int)(k.y <= key) + (int)(k.z <= key) + (int)(k.w <= key);
    }
    {
        const int i = own + part * 4;
        const uint4 k = *reinterpret_cast<const uint4*>(s_rank_keys + i);
        before += (k.x < key || (k.x == key && i < t)) + (k.y < key || (k.y == key && i + 1 < t)) +
                  (k.z < key || (k.z == key && i + 2 < t)) + (k.w < key || (k.w == key && i + 3 < t));
    }
    for (int i = own + 64 + part * 4; i < full; i += 64) {
        const uint4 k = *reinterpret_cast<const uint4*>(s_rank_keys + i);
        before += (int)(k.x < key) + (int)(k.y < key) + (int)(k.z < key) + (int)(k.w < key);
    }
#pragma unroll
    for (int m = 1; m < 16; m <<= 1) before += __shfl_xor(before, m);
    if (part == 0) {
        skey[before] = key;
        spos[before] = (u32)t;
    }
}

// Many tokens: by digits of up to 10 bits, the lowest first, every pass keeping the order of equal digits.  A workgroup takes a
// chunk of the tokens, each of its sixteen waves a sixteenth of it in one piece.  Up to SORT_FUSED chunks a workgroup adds up the counts of those
// before it by itself; of more that would be as much work as the sort, and a launch in between does it once for all.
#define DIGIT_MAX 10
#define SORT_WAVES 16
#define SORT_FUSED 64
#define SORT_WGS 256
struct SortShape {
    int passes, bits;        // digits, and bits of one
    int64_t wgs, chunk;      // workgroups, and tokens of one (a multiple of 1024)
    bool fused;
};
static SortShape sort_shape(int64_t n, int64_t n_rows)
{
    SortShape f;
    int b = 1;
    while (b < 31 && (n_rows >> b) != 0) ++b;               // bits of the largest key, n_rows
    f.passes = (b + DIGIT_MAX - 1) / DIGIT_MAX;
    f.bits = (b + f.passes - 1) / f.passes;
    f.fused = n <= (int64_t)SORT_FUSED * 4096;
    const int64_t wgs = f.fused ? SORT_FUSED : SORT_WGS;
    f.chunk = ((n + wgs - 1) / wgs + 1023) & ~(int64_t)1023;
    f.wgs = (n + f.chunk - 1) / f.chunk;
    return f;
}
// how many of the wave's tokens have which digit: s_count[wave][digit]
__device__ inline u32 digit_of(u32 key, int shift, int bits) { return (key >> shift) & ((1u << bits) - 1u); }
__device__ inline void count_digits(const void* ids, int ids64, const u32* key_in, int64_t n, int64_t n_rows, int64_t from, int64_t to, int shift,
                                    int bits, u32* count)
{
    for (int64_t t = from + tg_lane(); t < to; t += 64) {
        const u32 key = key_in ? key_in[t] : token_key(ids, ids64, t, n_rows);
        atomicAdd(count + digit_of(key, shift, bits), 1u);
    }
}
// per workgroup and digit: how many.  table: the counts of a workgroup back to back
__global__ __launch_bounds__(64 * SORT_WAVES) void digit_count_kernel(const void* __restrict__ ids, int ids64, const u32* __restrict__ key_in, int64_t n,
                                                                      int64_t n_rows, int64_t chunk, int shift, int bits, u32* __restrict__ table,
                                                                      u32* __restrict__ runs, ZeroPart z)
{
    if (blockIdx.x >= z.first) { zero_part(z); return; }
    if (blockIdx.x == 0 && threadIdx.x < 2) runs[threadIdx.x] = 0;
    __shared__ u32 s_count[1 << DIGIT_MAX];
    const int digits = 1 << bits;
    for (int i = threadIdx.x; i < digits; i += 64 * SORT_WAVES) s_count[i] = 0;
    __syncthreads();
    const int64_t from = (int64_t)blockIdx.x * chunk + (threadIdx.x >> 6) * (chunk / SORT_WAVES);
    int64_t to = from + chunk / SORT_WAVES;
    if (to > n) to = n;
    count_digits(ids, ids64, key_in, n, n_rows, from, to, shift, bits, s_count);
    __syncthreads();
    for (int i = threadIdx.x; i < digits; i += 64 * SORT_WAVES) table[(int64_t)blockIdx.x * digits + i] = s_count[i];
}
// a thread a digit: its counts become the number of tokens in workgroups before, their sum goes to total[digit]
__global__ __launch_bounds__(256) void digit_scan_kernel(u32* __restrict__ table, int wgs, int digits, u32* __restrict__ total, ZeroPart z)
{
    if (blockIdx.x >= z.first) { zero_part(z); return; }
    const int digit = blockIdx.x * 256 + threadIdx.x;
    if (digit >= digits) return;
    u32 sum = 0;
#pragma unroll 16
    for (int w = 0; w < wgs; ++w) {
        const u32 c = table[(int64_t)w * digits + digit];
        table[(int64_t)w * digits + digit] = sum;
        sum += c;
    }
    total[digit] = sum;
}
// every token to its place: the smaller digits' tokens, those of its digit in workgroups before, in waves before, and in its wave before
template <bool FUSED>
__global__ __launch_bounds__(64 * SORT_WAVES) void digit_place_kernel(const void* __restrict__ ids, int ids64, const u32* __restrict__ key_in,
                                                                      const u32* __restrict__ pos_in, int64_t n, int64_t n_rows, int64_t chunk,
                                                                      int shift, int bits, const u32* __restrict__ table,
                                                                      const u32* __restrict__ total, u32* __restrict__ key_out,
                                                                      u32* __restrict__ pos_out, ZeroPart z)
{
    if (blockIdx.x >= z.first) { zero_part(z); return; }
    static_assert(1 << DIGIT_MAX <= 64 * SORT_WAVES, "a thread a digit");
    __shared__ u32 s_next[SORT_WAVES][1 << DIGIT_MAX];
    __shared__ u32 s_wave[SORT_WAVES];
    const int wave = threadIdx.x >> 6, lane = tg_lane(), digits = 1 << bits, i = threadIdx.x;
    if (i < digits) {
#pragma unroll
        for (int w = 0; w < SORT_WAVES; ++w) s_next[w][i] = 0;
    }
    __syncthreads();
    const int64_t from = (int64_t)blockIdx.x * chunk + wave * (chunk / SORT_WAVES);
    int64_t to = from + chunk / SORT_WAVES;
    if (to > n) to = n;
    count_digits(ids, ids64, key_in, n, n_rows, from, to, shift, bits, s_next[wave]);
    // the thread's digit: how many tokens have it, and how many of them are in workgroups before
    u32 all = 0, here = 0;
    if (i < digits) {
        if (FUSED) {
            const int wgs = (int)z.first, me = (int)blockIdx.x;
            u32 c[16];
            for (int w0 = 0; w0 < wgs; w0 += 16) {
#pragma unroll
                for (int w = 0; w < 16; ++w) c[w] = w0 + w < wgs ? table[(w0 + w) * digits + i] : 0u;
#pragma unroll
                for (int w = 0; w < 16; ++w) {
                    all += c[w];
                    here += w0 + w < me ? c[w] : 0u;
                }
            }
        } else {
            all = total[i];
            here = table[(int64_t)blockIdx.x * digits + i];
        }
    }
    // ... and how many have a smaller one
    u32 x = all;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const u32 y = (u32)__shfl_up((int)x, m);
        if (lane >= m) x += y;
    }
    if (lane == 63) s_wave[wave] = x;
    __syncthreads();                                        // (the waves' counts are there as well)
    if (i < digits) {
        u32 at = x - all + here;
        for (int j = 0; j < wave; ++j) at += s_wave[j];
#pragma unroll
        for (int j = 0; j < SORT_WAVES; ++j) {
            const u32 k = s_next[j][i];
            s_next[j][i] = at;
            at += k;
        }
    }
    __syncthreads();
    // (the wave's own words from here on; a row of tokens is placed before the next one reads them)
    for (int64_t t0 = from; t0 < to; t0 += 64) {
        const int64_t t = t0 + lane;
        const bool real = t < to;
        const u32 key = !real ? 0u : key_in ? key_in[t] : token_key(ids, ids64, t, n_rows);
        const u32 digit = digit_of(key, shift, bits);
        u64 same = __ballot(real);
        for (int b = 0; b < bits; ++b) {
            const bool one = (digit >> b) & 1u;
            const u64 ones = __ballot(one);
            same &= one ? ones : ~ones;
        }
        u32 at = 0;
        if (real) at = s_next[wave][digit];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        const int before = __popcll(same & tg_lanemask_lt());
        if (real) {
            key_out[at + before] = key;
            pos_out[at + before] = pos_in ? pos_in[t] : (u32)t;
            if (before == 0) s_next[wave][digit] = at + (u32)__popcll(same);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

// ---- sums over the runs of the sorted list
#define RUN_TILE 16
#define RUN_LONG 16
template <class E, class O>
__device__ inline void write_row(const float* v, int left, O* p, float scale, bool add)
{
    // in pieces of the output's type
    constexpr int EO = TgPiece<O>::E < TgPiece<E>::E ? TgPiece<O>::E : TgPiece<E>::E;
#pragma unroll
    for (int j = 0; j < TgPiece<E>::E; j += EO) {
        typedef O vec __attribute__((ext_vector_type(EO), aligned(sizeof(O))));
        if (left >= j + EO) {
            vec x;
            if (add) {
                x = *reinterpret_cast<const vec*>(p + j);
#pragma unroll
                for (int i = 0; i < EO; ++i) x[i] = (O)((float)x[i] + v[j + i] * scale);
            } else {
#pragma unroll
                for (int i = 0; i < EO; ++i) x[i] = (O)(v[j + i] * scale);
            }
            *reinterpret_cast<vec*>(p + j) = x;
        } else {
#pragma unroll
            for (int i = 0; i < EO; ++i)
                if (j + i < left) p[j + i] = (O)((add ? (float)p[j + i] : 0.0f) + v[j + i] * scale);
        }
    }
}

// G lanes a tile, a piece of the row a lane, as many columns of tiles as the row has G pieces.  All of a tile's rows are asked for before
// the first is added.  The end of a run stands in the code sixteen times, and its length is what the waves fetch: so pieces are whole (WHOLE, rows of a
// piece or more: the last one ends where the row does, and shares columns with the one before, which has the same sums) and a run's end
// is a store or two.  (131 072 rows of 1024 bf16, 65 536 tokens: 64 us with pieces of any length, 60 whole; 20 011 tokens, rows of 50 fp32: 11.8 and 8.8.)
// parts: two rows of d per tile: of a run that came from the tile before, and of one that goes on in the next
// but began here; such tiles are listed, in any order, from runs[2] on (runs[0] of them) or, where the run goes on for RUN_LONG tiles or
// more, from the list's other end (runs[1]).
template <class E, class O, bool ADD, bool WHOLE>
__global__ __launch_bounds__(256) void run_sum_kernel(const E* __restrict__ grad, int64_t ld, const u32* __restrict__ skey,
                                                      const u32* __restrict__ spos, int64_t n, int64_t n_rows, int d, float scale,
                                                      int gshift, int columns, O* __restrict__ out, float* __restrict__ parts,
                                                      u32* __restrict__ runs)
{
    typedef TgPiece<E> P;
    typedef float part __attribute__((ext_vector_type(4), aligned(4)));
    const int lane = threadIdx.x & ((1 << gshift) - 1);
    const int64_t unit = (int64_t)blockIdx.x * (256 >> gshift) + (threadIdx.x >> gshift);
    const int64_t tile = unit / columns;
    const int column = (int)(unit - tile * columns);
    const int piece = ((column << gshift) + lane) * P::E;
    const int64_t i0 = tile * RUN_TILE;
    if (i0 >= n || piece >= d) return;
    const int at = WHOLE && piece + P::E > d ? d - P::E : piece;
    // (what is added to has to be added once: the shared columns are the piece's before)
    const int skip = ADD ? piece - at : 0, left = WHOLE ? P::E : d;
    const int count = (int)(n - i0 < RUN_TILE ? n - i0 : RUN_TILE);
    const u32 none = (u32)n_rows;
    u32 key[RUN_TILE];
    typename P::vec g[RUN_TILE];
    {
        // (the arrays hold whole tiles)
        u32 pos[RUN_TILE];
#pragma unroll
        for (int j = 0; j < RUN_TILE; j += 4) {
            *reinterpret_cast<uint4*>(key + j) = *reinterpret_cast<const uint4*>(skey + i0 + j);
            *reinterpret_cast<uint4*>(pos + j) = *reinterpret_cast<const uint4*>(spos + i0 + j);
        }
#pragma unroll
        for (int j = 0; j < RUN_TILE; ++j) {
            if (j >= count) key[j] = none;
            // (a token without a row: the first token's values, which no run takes in)
            g[j] = P::raw(grad + (int64_t)(key[j] == none ? 0u : pos[j]) * ld + at, left);
        }
    }
    u32 cur = key[0];
    if (cur == none) return;                                // (from here on there are only tokens without a row)
    bool carried = i0 > 0 && skey[i0 - 1] == cur;
    const bool goes_on = i0 + count < n && skey[i0 + count] == key[RUN_TILE - 1] && key[RUN_TILE - 1] != none;
    float acc[P::E];
#pragma unroll
    for (int i = 0; i < P::E; ++i) acc[i] = 0.0f;
    const auto put_part = [&](int which) {
        float* p = parts + (2 * tile + which) * (int64_t)d + at;
        if (WHOLE) {
#pragma unroll
            for (int i = 0; i < P::E; i += 4) *reinterpret_cast<part*>(p + i) = part{acc[i], acc[i + 1], acc[i + 2], acc[i + 3]};
        } else {
#pragma unroll
            for (int i = 0; i < P::E; ++i)
                if (i < left) p[i] = acc[i];
        }
    };
    const auto put = [&] {
        O* p = out + (int64_t)cur * d + at;
        if (ADD && skip) {
#pragma unroll
            for (int i = 0; i < P::E; ++i)
                if (i >= skip) p[i] = (O)((float)p[i] + acc[i] * scale);
        } else write_row<E, O>(acc, left, p, scale, ADD);
    };
#pragma unroll
    for (int j = 0; j < RUN_TILE; ++j) {
        if (key[j] != cur) {
            if (carried) put_part(0);
            else put();
            carried = false;
            cur = key[j];
            if (cur == none) return;
#pragma unroll
            for (int i = 0; i < P::E; ++i) acc[i] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < P::E; ++i) acc[i] += (float)g[j][i];
    }
    if (!carried && !goes_on) { put(); return; }
    put_part(carried ? 0 : 1);
    if (!carried && column == 0 && lane == 0) {
        const int64_t far = i0 + (int64_t)RUN_LONG * RUN_TILE;
        if (far < n && skey[far] == cur) runs[1 + (n + RUN_TILE - 1) / RUN_TILE - atomicAdd(runs + 1, 1u)] = (u32)tile;
        else runs[2 + atomicAdd(runs, 1u)] = (u32)tile;
    }
}

// The parts of the listed runs are added in the tiles' order, 256 columns at a time.  Most runs have two or three: a wave each.  Of a long one
// sixteen waves take an equal stretch each, and are added in their order; the first RUN_JOIN_LONG workgroups look after those.
#define RUN_JOIN_LONG 128
#define RUN_JOIN_WAVES 16
template <class O>
__global__ __launch_bounds__(64 * RUN_JOIN_WAVES) void run_join_kernel(const u32* __restrict__ skey, int64_t n, int d, float scale, int add,
                                                       const float* __restrict__ parts, const u32* __restrict__ runs, O* __restrict__ out)
{
    typedef TgPiece<float> P;
    __shared__ float s_sum[RUN_JOIN_WAVES][64][4];
    const int wave = threadIdx.x >> 6, lane = tg_lane(), columns = (d + 255) / 256;
    const int64_t tiles = (n + RUN_TILE - 1) / RUN_TILE;
    const auto put = [&](u32 key, int c, const float* v) {
        O* p = out + (int64_t)key * d + c;
        write_row<float, O>(v, d - c, p, scale, add != 0);
    };
    if (blockIdx.x >= RUN_JOIN_LONG) {
        const int64_t all = (int64_t)runs[0] * columns;
        for (int64_t item = (int64_t)(blockIdx.x - RUN_JOIN_LONG) * RUN_JOIN_WAVES + wave; item < all;
             item += (int64_t)(gridDim.x - RUN_JOIN_LONG) * RUN_JOIN_WAVES) {
            const int64_t tile = runs[2 + item / columns];
            const int c = (int)(item % columns) * 256 + lane * 4;
            const u32 key = skey[tile * RUN_TILE + RUN_TILE - 1];
            // in how many tiles behind this one it begins the tile
            const int64_t at = (tile + 1 + lane) * RUN_TILE;
            const u64 same = __ballot(lane < RUN_LONG && at < n && skey[at] == key);
            const int more = __ffsll((unsigned long long)~same) - 1;
            P sum;
            sum.load(parts + (2 * tile + 1) * d + c, d - c);
#pragma unroll 4
            for (int t = 1; t <= more; ++t) {
                P q;
                q.load(parts + 2 * (tile + t) * d + c, d - c);
#pragma unroll
                for (int e = 0; e < 4; ++e) sum.v[e] += q.v[e];
            }
            if (c < d) put(key, c, sum.v);
        }
        return;
    }
    const int64_t all = (int64_t)runs[1] * columns;
    for (int64_t item = blockIdx.x; item < all; item += RUN_JOIN_LONG) {
        const int64_t tile = runs[1 + tiles - item / columns];
        const int c = (int)(item % columns) * 256 + lane * 4;
        const u32 key = skey[tile * RUN_TILE + RUN_TILE - 1];
        int64_t lo = (tile + RUN_LONG) * RUN_TILE, hi = n;                      // the first place with another key
        while (lo < hi) {
            const int64_t mid = (lo + hi) >> 1;
            if (skey[mid] == key) lo = mid + 1; else hi = mid;
        }
        const int64_t end = (lo - 1) / RUN_TILE;                                // its last tile
        const int64_t each = (end - tile + RUN_JOIN_WAVES - 1) / RUN_JOIN_WAVES, from = tile + 1 + wave * each, to = from + each < end + 1 ? from + each : end + 1;
        P sum;
        sum.load(parts + (2 * tile + 1) * d + c, wave == 0 ? d - c : 0);
#pragma unroll 8
        for (int64_t t = from; t < to; ++t) {
            P q;
            q.load(parts + 2 * t * d + c, d - c);
#pragma unroll
            for (int e = 0; e < 4; ++e) sum.v[e] += q.v[e];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) s_sum[wave][lane][e] = sum.v[e];
        __syncthreads();
        if (wave == 0 && c < d) {
#pragma unroll
            for (int w = 1; w < RUN_JOIN_WAVES; ++w)
#pragma unroll
                for (int e = 0; e < 4; ++e) sum.v[e] += s_sum[w][lane][e];
            put(key, c, sum.v);
        }
        __syncthreads();
    }
}

struct GradSpace {
    u32 *key[2], *pos[2], *table, *total, *runs;
    float* parts;
};
static size_t carve_grad(GradSpace* g, void* base, int64_t n, int64_t n_rows, int d)
{
    TgCarve c{(char*)base, 0};
    const bool few = n <= RANK_MAX;
    const SortShape f = sort_shape(n, n_rows);
    const size_t tiles = (size_t)((n + RUN_TILE - 1) / RUN_TILE), whole = tiles * RUN_TILE;
    g->key[0] = c.take<u32>(whole);
    g->pos[0] = c.take<u32>(whole);
    g->key[1] = few ? nullptr : c.take<u32>(whole);
    g->pos[1] = few ? nullptr : c.take<u32>(whole);
    g->table = few ? nullptr : c.take<u32>((size_t)f.wgs << f.bits);
    g->total = few ? nullptr : c.take<u32>((size_t)1 << f.bits);
    g->runs = c.take<u32>(tiles + 2);
    g->parts = c.take<float>(tiles * 2 * d);
    return c.used;
}
size_t tg_lookup_grad_space(int64_t n, int64_t n_rows, int d)
{
    GradSpace g;
    return n == 0 ? 0 : carve_grad(&g, nullptr, n, n_rows, d);
}

template <class E, class O>
static void launch_sums(const E* grad, int64_t ld, const u32* key, const u32* pos, int64_t n, int64_t n_rows, int d, float scale, int add, O* out,
                        const GradSpace& g, hipStream_t s)
{
    const int64_t tiles = (n + RUN_TILE - 1) / RUN_TILE;
    const int pieces = (d + TgPiece<E>::E - 1) / TgPiece<E>::E;
    const int gs = lanes_shift(pieces), columns = (pieces + (1 << gs) - 1) >> gs;
    const int64_t per = 256 >> gs;
    // (fewer than 2^32 work-items: 64 of them stand for 16 KB of a gradient that fits the card, or for 16 tokens of a short row)
    const auto sums = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)((tiles * columns + per - 1) / per)), dim3(256), 0, s, grad, ld, key, pos, n, n_rows, d, scale, gs,
                           columns, out, g.parts, g.runs);
    };
    const bool whole = d >= TgPiece<E>::E;
    if (add) whole ? sums(run_sum_kernel<E, O, true, true>) : sums(run_sum_kernel<E, O, true, false>);
    else whole ? sums(run_sum_kernel<E, O, false, true>) : sums(run_sum_kernel<E, O, false, false>);
    if (tiles > 1) {
        // (at most a listed run a tile)
        const int64_t waves = (tiles - 1) * ((d + 255) / 256), wgs = (waves + RUN_JOIN_WAVES - 1) / RUN_JOIN_WAVES;
        hipLaunchKernelGGL(run_join_kernel<O>, dim3((unsigned)(wgs < 512 ? wgs : 512) + RUN_JOIN_LONG), dim3(64 * RUN_JOIN_WAVES), 0, s, key, n, d, scale, add, g.parts,
                           g.runs, out);
    }
}

void tg_launch_lookup_grad(const void* grad, int64_t ld, int dtype, const void* ids, int ids64, int64_t n, int64_t n_rows, int d, float scale,
                           int accumulate, void* out, int out_dtype, void* space, hipStream_t s)
{
    const size_t all = accumulate ? 0 : (size_t)n_rows * d * tg_type_bytes(out_dtype);
    if (n == 0) {
        tg_launch_zero(out, all, s);
        return;
    }
    GradSpace g;
    carve_grad(&g, space, n, n_rows, d);
    ZeroPart z = zero_of(out, all);
    int at = 0;
    if (n <= RANK_MAX) {
        const int full = ((int)n + 63) & ~63;
        z.first = (uint32_t)((n + 15) / 16);
        hipLaunchKernelGGL(rank_sort_kernel, dim3(z.first + zero_wgs(z)), dim3(256), full * 4, s, ids, ids64, (int)n, n_rows, g.key[0], g.pos[0], g.runs, z);
    } else {
        const SortShape f = sort_shape(n, n_rows);
        const int digits = 1 << f.bits, each = f.fused ? 2 : 3;
        const dim3 threads(64 * SORT_WAVES);
        z.parts = each * f.passes;
        const unsigned zw = zero_wgs(z);
        for (int p = 0; p < f.passes; ++p) {
            const u32* ki = p ? g.key[at] : nullptr;
            const u32* pi = p ? g.pos[at] : nullptr;
            const int to = p ? at ^ 1 : 0, shift = p * f.bits;
            z.part = each * p;
            z.first = (uint32_t)f.wgs;
            hipLaunchKernelGGL(digit_count_kernel, dim3(z.first + zw), threads, 0, s, ids, ids64, ki, n, n_rows, f.chunk, shift, f.bits, g.table, g.runs, z);
            if (!f.fused) {
                z.part = each * p + 1;
                z.first = (uint32_t)((digits + 255) / 256);
                hipLaunchKernelGGL(digit_scan_kernel, dim3(z.first + zw), dim3(256), 0, s, g.table, (int)f.wgs, digits, g.total, z);
            }
            z.part = each * p + each - 1;
            z.first = (uint32_t)f.wgs;
            hipLaunchKernelGGL(f.fused ? digit_place_kernel<true> : digit_place_kernel<false>, dim3(z.first + zw), threads, 0, s, ids, ids64, ki, pi, n,
                               n_rows, f.chunk, shift, f.bits, g.table, g.total, g.key[to], g.pos[to], z);
            at = to;
        }
    }
    TG_WITH_TYPE(dtype, E, {
        if (out_dtype == 0) launch_sums<E, float>((const E*)grad, ld, g.key[at], g.pos[at], n, n_rows, d, scale, accumulate, (float*)out, g, s);
        else launch_sums<E, E>((const E*)grad, ld, g.key[at], g.pos[at], n, n_rows, d, scale, accumulate, (E*)out, g, s);
    });
}
