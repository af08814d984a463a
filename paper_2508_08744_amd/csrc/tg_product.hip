// Products of 8-bit rows with a scale per token and channel: out[i][j] = a_scale[i] b_scale[j] sum_k a[i][k] b[j][k] (+ bias[j]).
//
// The sum is a whole number below 2^31 and exact, in whatever order it is taken; the scales and the bias are the epilogue's.  Many
// tokens: tiles in LDS (tg_tiles.h), bound by the matrix instructions, or by the bytes of the output where rows are short.  A few
// tokens: every byte of b is needed once and nothing else counts, so a wave reads its rows of b straight into the matrix
// instructions' registers, with several loads in flight, and the waves of a workgroup share the contraction between them.
// (8192 x 8192 x 4096 to bf16: 220 us, 2.5 POP/s; 4 x 16 384 x 4096: 13 us, 5.2 TB/s.)
#include "tg_embed.h"
#include "tg_tiles.h"

#include <type_traits>

// what reads rows as they are: short ones, and those of few tokens
#define PRODUCT_FEW 64            // tokens up to which b is read straight into the registers
#define PRODUCT_SHORT 256         // bytes of a row up to which a product keeps its tokens' rows in registers
static bool product_as_is(int64_t m, int k) { return m <= PRODUCT_FEW || k <= PRODUCT_SHORT; }

// 16 bytes of a row that has `left` bytes from p on (rows may begin anywhere; what is not there reads as zero)
__device__ inline tg_i32x4 product_load(const char* p, int left)
{
    typedef int i32x4u __attribute__((ext_vector_type(4), aligned(1)));
    if (left >= 16) return *reinterpret_cast<const i32x4u*>(p);
    tg_i32x4 v = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 15; ++i)
        if (i < left) v[i / 4] |= (int)(uint8_t)p[i] << (i % 4 * 8);
    return v;
}

// 16 bytes from p on, of which those behind `end` read as zero: for rows whose other factor is zero behind their length, so that what follows a row
// in memory may be read with it.  (Only the matrix's last bytes take the loop.)
__device__ inline tg_i32x4 product_load_on(const char* p, const char* end)
{
    typedef int i32x4u __attribute__((ext_vector_type(4), aligned(1)));
    if (p + 16 <= end) return *reinterpret_cast<const i32x4u*>(p);
    uint64_t v[2] = {0, 0};
#pragma unroll 1
    for (int i = 0; i < 15 && p + i < end; ++i) {
        const uint64_t b = (uint64_t)(uint8_t)p[i] << (i % 8 * 8);
        v[0] |= i < 8 ? b : 0;
        v[1] |= i < 8 ? 0 : b;
    }
    return tg_i32x4{(int)v[0], (int)(v[0] >> 32), (int)v[1], (int)(v[1] >> 32)};
}

// x: channels, y: tokens.
template <class O, int BM, int BN, int WM, int WN, int NB, bool BIAS>
__global__ __launch_bounds__(64 * WM * WN) void product_kernel(TileRows X, TileRows Y, int bytes, const float* __restrict__ as,
                                                               const float* __restrict__ bs, const float* __restrict__ bias, uint32_t nx,
                                                               uint32_t ny, uint32_t group, O* __restrict__ out)
{
    typedef Tile<int8_t, BM, BN, WM, WN, false, false, NB> T;
    __shared__ __align__(1024) char lds[T::LDS];
    // the scales and the bias: asked for before the products, so that nothing waits for them behind
    __shared__ float s_as[BN], s_bs[BM], s_bias[BIAS ? BM : 1];
    uint32_t tx, ty;
    tile_place(tile_of_block(blockIdx.x, nx * ny), nx, ny, group, &tx, &ty);
    const int64_t x0 = (int64_t)tx * BM, y0 = (int64_t)ty * BN;
    T t;
    t.start(X, Y, x0, y0, 0, bytes, lds);
    const int i0 = threadIdx.x;
    if (i0 < BN && y0 + i0 < Y.rows) s_as[i0] = as[y0 + i0];
    if (i0 < BM && x0 + i0 < X.rows) {
        s_bs[i0] = bs[x0 + i0];
        if (BIAS) s_bias[i0] = bias[x0 + i0];
    }
    t.loop();
    const int have = x0 + BM <= X.rows ? BM : (int)(X.rows - x0);
    if constexpr (sizeof(O) == 2) {
        // A lane has four neighbours, 8 bytes, of 16 rows at a time; the tile goes through its memory, which is free, to be stored as whole rows.  Piece c of
        // row r lies at place c ^ (r & SWAP): the lanes that write one column of pieces at a time are in different banks.
        // (8192 x 8192 x 4096 to bf16: 236 us stored as the lanes have them, 222 so; 8000 x 4001 x 1024: 56 and 45.  Of fp32 a lane has 16 bytes.)
        constexpr int W = 8, PIECES = BM / W, SWAP = PIECES < 16 ? PIECES - 1 : 15;
        static_assert(BM * BN * sizeof(O) <= T::LDS && (PIECES & (PIECES - 1)) == 0, "the tile's place");
        typedef O four __attribute__((ext_vector_type(4)));
        typedef O vec __attribute__((ext_vector_type(W)));
        typedef O loose __attribute__((ext_vector_type(W), aligned(sizeof(O))));
        int swap = threadIdx.x & SWAP;                        // (r & SWAP, whatever j)
#pragma unroll
        for (int j = 0; j < T::FN; ++j) {
            // (nothing of this is made out in front of the products, in whose loop no register is free)
            asm volatile("" : "+v"(swap) : : "memory");
#pragma unroll
            for (int i = 0; i < T::FM; ++i) asm volatile("" : "+v"(t.acc[i][j]));
            const int r = t.y_of(j);
            const float s = s_as[r];
            char* const row = lds + r * (PIECES * 16);
#pragma unroll
            for (int i = 0; i < T::FM; ++i) {
                const int x = t.x_of(i);
                four v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = (O)((float)t.acc[i][j][e] * s * s_bs[x + e] + (BIAS ? s_bias[x + e] : 0.0f));
                *reinterpret_cast<four*>(row + ((x / W) ^ swap) * 16 + x % W * (int)sizeof(O)) = v;
            }
        }
        __syncthreads();
#pragma unroll 4
        for (int at = threadIdx.x; at < BN * PIECES; at += 64 * WM * WN) {
            const int r = at / PIECES, x = at % PIECES * W;
            if (y0 + r >= Y.rows || x >= have) continue;
            const vec v = *reinterpret_cast<const vec*>(lds + (r * PIECES + (at % PIECES ^ (r & SWAP))) * 16);
            O* o = out + (y0 + r) * X.rows + x0 + x;
            if (x + W <= have) *reinterpret_cast<loose*>(o) = v;
            else {
#pragma unroll
                for (int e = 0; e < W - 1; ++e)
                    if (x + e < have) o[e] = v[e];
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < T::FN; ++j) {
            const int64_t y = y0 + t.y_of(j);
            if (y >= Y.rows) continue;
            const float s = s_as[t.y_of(j)];
            O* row = out + y * X.rows + x0;
#pragma unroll
            for (int i = 0; i < T::FM; ++i) {
                const int x = t.x_of(i);
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = (float)t.acc[i][j][e] * s * s_bs[x + e] + (BIAS ? s_bias[x + e] : 0.0f);
                if (x < have) tile_put(row + x, v, have - x);
            }
        }
    }
}

// Up to 16 FN tokens.  A workgroup has 16 channels, a wave a quarter of the contraction in one piece, STEPS x 64 bytes of every row in
// flight.  (16 384 channels of 4096, 4 tokens, fp16: 16 steps 13.0 us, 5.2 TB/s; 4 steps 13.3.)
template <class O, int FN>
__global__ __launch_bounds__(256) void product_few_kernel(TileRows X, TileRows Y, int bytes, const float* __restrict__ as,
                                                          const float* __restrict__ bs, const float* __restrict__ bias, int64_t first,
                                                          O* __restrict__ out)
{
    constexpr int STEPS = 16 / FN;
    __shared__ tg_i32x4 s_part[3][FN][64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = tg_lane(), row = lane & 15, q = lane >> 4;
    const int64_t x0 = first + (int64_t)blockIdx.x * 16;
    // (rows that are not there are read as the first one: nobody stores their sums)
    const char* xp = X.p + (x0 + row < X.rows ? x0 + row : x0) * X.pitch + q * 16;
    const char* yp[FN];
#pragma unroll
    for (int j = 0; j < FN; ++j) yp[j] = Y.p + (int64_t)(j * 16 + row < Y.rows ? j * 16 + row : 0) * Y.pitch + q * 16;
    tg_i32x4 acc[FN];
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[j] = tg_i32x4{0, 0, 0, 0};
    const int each = ((bytes + 255) / 256) * 64, k1 = (wave + 1) * each < bytes ? (wave + 1) * each : bytes;
    int k = wave * each;
    // whole pieces of 64 bytes, STEPS at a time, then by fours and one by one, then what is left of a row
    const auto steps = [&](auto count) {
        constexpr int N = decltype(count)::value;
        for (; k + N * 64 <= k1; k += N * 64) {
            tg_i32x4 x[N], y[N][FN];
#pragma unroll
            for (int h = 0; h < N; ++h) x[h] = product_load(xp + k + h * 64, 16);
#pragma unroll
            for (int h = 0; h < N; ++h)
#pragma unroll
                for (int j = 0; j < FN; ++j) y[h][j] = product_load(yp[j] + k + h * 64, 16);
#pragma unroll
            for (int h = 0; h < N; ++h)
#pragma unroll
                for (int j = 0; j < FN; ++j) acc[j] = TileMul<int8_t>::mul(x[h], y[h][j], acc[j]);
        }
    };
    steps(std::integral_constant<int, STEPS>());
    if (STEPS > 4) steps(std::integral_constant<int, 4>());
    steps(std::integral_constant<int, 1>());
    if (k < k1) {
        const tg_i32x4 x = product_load(xp + k, k1 - k - q * 16);
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[j] = TileMul<int8_t>::mul(x, product_load(yp[j] + k, k1 - k - q * 16), acc[j]);
    }
    if (wave > 0) {
#pragma unroll
        for (int j = 0; j < FN; ++j) s_part[wave - 1][j][lane] = acc[j];
    }
    __syncthreads();
    if (wave > 0) return;
    const int64_t x = x0 + q * 4;
#pragma unroll
    for (int j = 0; j < FN; ++j) {
        const int64_t y = j * 16 + row;
        const tg_i32x4 sum = acc[j] + s_part[0][j][lane] + s_part[1][j][lane] + s_part[2][j][lane];
        if (y >= Y.rows) continue;
        const float s = as[y];
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool in = x + e < X.rows;
            v[e] = (float)sum[e] * s * (in ? bs[x + e] : 0.0f) + (in && bias ? bias[x + e] : 0.0f);
        }
        if (x < X.rows) tile_put(out + y * X.rows + x, v, X.rows - x);
    }
}

// Short rows, of up to STEPS x 64 bytes: the output's bytes bound the product, and a tile would be loaded, multiplied once or twice and stored,
// each after the other.  A wave keeps the rows of 16 FN tokens in registers and walks over the channels 16 CB at a time, beside the
// other waves of its workgroup, with the next ones' rows and scales on their way.  A lane's results are 16 bytes of an output row (which 16
// channels a product takes is free: for outputs of 16 bits two products share 32, in turn four by four), but a wave's are 64 bytes of each of 16
// rows, which lie far apart: so the workgroup's go through LDS, 16 KB at a time, and are stored as stretches of a row.  (203 tokens, 10^6 channels of
// 128, fp32: 243 us without, 216 with it, of which 54 are left without the stores; 4000 tokens, 30 000 channels of 200, fp32: 197 and 150.)
template <class O, int STEPS, int FN, int CB, bool BIAS>
__global__ __launch_bounds__(256, 2) void product_short_kernel(TileRows X, TileRows Y, int bytes, const float* __restrict__ as,
                                                            const float* __restrict__ bs, const float* __restrict__ bias, O* __restrict__ out)
{
    constexpr int W = 16 / (int)sizeof(O), PER = W / 4;        // neighbours of a row that a lane stores; products they come from
    static_assert(CB % PER == 0, "whole stores");
    constexpr int PIECES = 16 * CB / PER;                      // of 16 bytes, of a row of the workgroup's
    constexpr int FEW = 1024 / (16 * PIECES), TURN = FEW < FN ? FEW : FN;      // groups of 16 tokens that go through LDS at a time
    static_assert(FN % TURN == 0, "whole turns");
    constexpr int EACH = TURN * 16 * PIECES / 256;             // pieces that a lane stores of them
    typedef O vec __attribute__((ext_vector_type(W)));
    __shared__ vec s_out[2][TURN * 16 * PIECES];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = tg_lane(), row = lane & 15, q = lane >> 4;
    const int64_t chunks = (X.rows + 16 * CB - 1) / (16 * CB), groups = (chunks + 3) / 4, y0 = (int64_t)blockIdx.y * (16 * FN);
    const char* end = X.p + X.rows * X.pitch;
    tg_i32x4 y[FN][STEPS];
    float sy[FN];
#pragma unroll
    for (int j = 0; j < FN; ++j) {
        const int64_t r = y0 + j * 16 + row;
        const bool in = r < Y.rows;
        sy[j] = in ? as[r] : 0.0f;
#pragma unroll
        for (int h = 0; h < STEPS; ++h)
            y[j][h] = product_load(Y.p + (in ? r : 0) * Y.pitch + h * 64 + q * 16, bytes - h * 64 - q * 16);
    }
    tg_i32x4 x[CB][STEPS], next[CB][STEPS];
    float c[CB / PER][W], c_next[CB / PER][W];
    // (channels that are not there are read as the last chunk's first: nobody stores their sums)
    const auto load = [&](int64_t chunk) {
        if (chunk >= chunks) chunk = chunks - 1;
        const int64_t first = chunk * (16 * CB);
#pragma unroll
        for (int i = 0; i < CB; ++i) {
            const int64_t r = first + i / PER * (16 * PER) + (row >> 2) * W + i % PER * 4 + (row & 3);
            const char* p = X.p + (r < X.rows ? r : first) * X.pitch + q * 16;
#pragma unroll
            for (int h = 0; h < STEPS; ++h) next[i][h] = product_load_on(p + h * 64, end);
        }
#pragma unroll
        for (int i = 0; i < CB / PER; ++i) {
            const int64_t v = first + i * (16 * PER) + q * W;
#pragma unroll
            for (int e = 0; e < W; e += 4) {
                TgPiece<float> s;
                s.load(bs + v + e, v + e + 4 <= X.rows ? 4 : (int)(X.rows - v - e));
#pragma unroll
                for (int f = 0; f < 4; ++f) c_next[i][e + f] = s.v[f];
            }
        }
    };
    int buffer = 0;
    load((int64_t)blockIdx.x * 4 + wave);
    for (int64_t group = blockIdx.x; group < groups; group += gridDim.x) {
        const int64_t v0 = group * (64 * CB), v_wave = v0 + wave * (16 * CB);
#pragma unroll
        for (int i = 0; i < CB; ++i)
#pragma unroll
            for (int h = 0; h < STEPS; ++h) x[i][h] = next[i][h];
#pragma unroll
        for (int i = 0; i < CB / PER; ++i)
#pragma unroll
            for (int e = 0; e < W; ++e) c[i][e] = c_next[i][e];
        if (group + gridDim.x < groups) load((group + gridDim.x) * 4 + wave);
        TgPiece<float> b[CB];
        if (BIAS) {
#pragma unroll
            for (int i = 0; i < CB; ++i) {
                const int64_t v = v_wave + i / PER * (16 * PER) + q * W + i % PER * 4;
                b[i].load(bias + v, v + 4 <= X.rows ? 4 : v < X.rows ? (int)(X.rows - v) : 0);
            }
        }
#pragma unroll
        for (int j0 = 0; j0 < FN; j0 += TURN) {
            if (y0 + j0 * 16 >= Y.rows) break;
            // (piece p of token t lies at place p ^ t: the lanes that write one column of pieces at a time are in different banks)
#pragma unroll
            for (int jj = 0; jj < TURN; ++jj) {
                const int j = j0 + jj;
                tg_i32x4 acc[CB];
#pragma unroll
                for (int i = 0; i < CB; ++i) {
                    acc[i] = tg_i32x4{0, 0, 0, 0};
#pragma unroll
                    for (int h = 0; h < STEPS; ++h) acc[i] = TileMul<int8_t>::mul(x[i][h], y[j][h], acc[i]);
                }
#pragma unroll
                for (int i = 0; i < CB / PER; ++i) {
                    vec o;
#pragma unroll
                    for (int e = 0; e < W; ++e) {
                        const float v = (float)acc[i * PER + e / 4][e % 4] * sy[j] * c[i][e];
                        o[e] = (O)(BIAS ? v + b[i * PER + e / 4].v[e % 4] : v);
                    }
                    s_out[buffer][(jj * 16 + row) * PIECES + (((wave * (CB / PER) + i) * 4 + q) ^ row)] = o;
                }
            }
            // (two buffers in turn: one is written again only behind the next barrier, when all have read it)
            __syncthreads();
#pragma unroll
            for (int n = 0; n < EACH; ++n) {
                const int at = n * 256 + threadIdx.x, t = at / PIECES, p = at % PIECES;
                const vec o = s_out[buffer][t * PIECES + (p ^ (t & 15))];
                const int64_t r = y0 + j0 * 16 + t, v = v0 + p * W;
                if (r >= Y.rows || v >= X.rows) continue;
                typedef O loose __attribute__((ext_vector_type(W), aligned(sizeof(O))));
                O* to = out + r * X.rows + v;
                if (v + W <= X.rows) *reinterpret_cast<loose*>(to) = o;
                else {
#pragma unroll
                    for (int e = 0; e < W - 1; ++e)
                        if (v + e < X.rows) to[e] = o[e];
                }
            }
            buffer ^= 1;
        }
    }
}

// rows of d elements of e bytes to rows of a multiple of 16 bytes, the rest zero: 16 bytes a lane
template <class W>
__global__ __launch_bounds__(256) void pack_kernel(const W* __restrict__ p, int64_t ld, int64_t rows, int d, int per /* pieces of a row of out */,
                                                   W* __restrict__ out)
{
    constexpr int E = 16 / (int)sizeof(W);
    typedef W from __attribute__((ext_vector_type(E), aligned(sizeof(W))));
    typedef W to __attribute__((ext_vector_type(E)));
    const int64_t all = rows * per;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int64_t r = all < (1ll << 31) ? (int64_t)((uint32_t)i / (uint32_t)per) : i / per;
        const int at = (int)(i - r * per) * E;
        const W* q = p + r * ld + at;
        to x;
        if (at + E <= d) {
            const from v = *reinterpret_cast<const from*>(q);
#pragma unroll
            for (int j = 0; j < E; ++j) x[j] = v[j];
        } else {
#pragma unroll
            for (int j = 0; j < E; ++j) x[j] = at + j < d ? q[j] : (W)0;
        }
        reinterpret_cast<to*>(out)[i] = x;
    }
}
void tg_launch_pack(const void* p, int64_t ld, int64_t rows, int d, int e, void* out, hipStream_t s)
{
    if (rows == 0) return;
    const int per = (int)(tile_pitch(d, e) / 16);
    const int64_t wgs = (rows * per + 255) / 256;
    const dim3 g((unsigned)(wgs < 32768 ? wgs : 32768)), b(256);
    if (e == 1) hipLaunchKernelGGL(pack_kernel<uint8_t>, g, b, 0, s, (const uint8_t*)p, ld, rows, d, per, (uint8_t*)out);
    else if (e == 2) hipLaunchKernelGGL(pack_kernel<uint16_t>, g, b, 0, s, (const uint16_t*)p, ld, rows, d, per, (uint16_t*)out);
    else hipLaunchKernelGGL(pack_kernel<uint32_t>, g, b, 0, s, (const uint32_t*)p, ld, rows, d, per, (uint32_t*)out);
}

size_t tg_product_space(int64_t m, int64_t n, int k, bool ready)
{
    if (m == 0 || product_as_is(m, k) || (ready && (k & 15) == 0)) return 0;
    TgCarve c{nullptr, 0};
    c.take<char>((size_t)m * tile_pitch(k, 1));
    c.take<char>((size_t)n * tile_pitch(k, 1));
    return c.used;
}

template <class O, int STEPS, int FN>
static void launch_short(const TileRows& X, const TileRows& Y, int bytes, const float* as, const float* bs, const float* bias, O* out, hipStream_t s)
{
    constexpr int CB = 2;                                      // (64 channels at a time for outputs of 32 bits: 230 us where 32 take 216)
    // (groups of tokens along y: the limit on a grid's y is 65535)
    const int64_t most = 65535ll * 16 * FN, chunks = (X.rows + 16 * CB - 1) / (16 * CB);
    for (int64_t y0 = 0; y0 < Y.rows; y0 += most) {
        const TileRows part{Y.p + y0 * Y.pitch, Y.rows - y0 < most ? Y.rows - y0 : most, Y.pitch, Y.width};
        const int64_t ny = (part.rows + 16 * FN - 1) / (16 * FN);
        // two workgroups a CU, twice (256 tokens, 10^6 channels of 256, bf16: 231 us, 283 with twice as many)
        int64_t nx = (1024 + ny - 1) / ny;
        if (nx < 64) nx = 64;
        if (nx > (chunks + 3) / 4) nx = (chunks + 3) / 4;
        const dim3 grid((unsigned)nx, (unsigned)ny);
        if (bias) hipLaunchKernelGGL((product_short_kernel<O, STEPS, FN, CB, true>), grid, dim3(256), 0, s, X, part, bytes, as + y0, bs, bias, out + y0 * X.rows);
        else hipLaunchKernelGGL((product_short_kernel<O, STEPS, FN, CB, false>), grid, dim3(256), 0, s, X, part, bytes, as + y0, bs, bias, out + y0 * X.rows);
    }
}
template <class O, int BM, int BN, int WM, int WN, int NB = 2>
static void launch_tiles(const TileRows& X, const TileRows& Y, int bytes, const float* as, const float* bs, const float* bias, O* out, hipStream_t s)
{
    const uint32_t nx = (uint32_t)((X.rows + BM - 1) / BM), ny = (uint32_t)((Y.rows + BN - 1) / BN);
    const dim3 wgs(nx * ny), threads(64 * WM * WN);
    if (bias) hipLaunchKernelGGL((product_kernel<O, BM, BN, WM, WN, NB, true>), wgs, threads, 0, s, X, Y, bytes, as, bs, bias, nx, ny, 8u, out);
    else hipLaunchKernelGGL((product_kernel<O, BM, BN, WM, WN, NB, false>), wgs, threads, 0, s, X, Y, bytes, as, bs, bias, nx, ny, 8u, out);
}
template <class O>
static void launch_product(const TileRows& X, const TileRows& Y, int bytes, const float* as, const float* bs, const float* bias, O* out, hipStream_t s)
{
    if (bytes <= PRODUCT_SHORT) {
        const auto go = [&](auto steps, auto most) {
            constexpr int S = decltype(steps)::value, FN = decltype(most)::value;
            if (Y.rows <= 16) launch_short<O, S, 1>(X, Y, bytes, as, bs, bias, out, s);
            else if (Y.rows <= 32) launch_short<O, S, 2>(X, Y, bytes, as, bs, bias, out, s);
            else if (Y.rows <= 64 || FN == 4) launch_short<O, S, 4>(X, Y, bytes, as, bs, bias, out, s);
            else launch_short<O, S, FN>(X, Y, bytes, as, bs, bias, out, s);
        };
        if (bytes <= 64) go(std::integral_constant<int, 1>(), std::integral_constant<int, 8>());
        else if (bytes <= 128) go(std::integral_constant<int, 2>(), std::integral_constant<int, 8>());
        else go(std::integral_constant<int, 4>(), std::integral_constant<int, 4>());
        return;
    }
    const auto tiles = [&](int64_t bm, int64_t bn) { return ((X.rows + bm - 1) / bm) * ((Y.rows + bn - 1) / bn); };
    if (bytes > 512 && tiles(256, 256) >= 200) launch_tiles<O, 256, 256, 2, 4>(X, Y, bytes, as, bs, bias, out, s);
    else if (tiles(128, 128) >= 200) launch_tiles<O, 128, 128, 2, 2>(X, Y, bytes, as, bs, bias, out, s);
    else launch_tiles<O, 64, 64, 2, 2, 4>(X, Y, bytes, as, bs, bias, out, s);
}

void tg_launch_product(const int8_t* a, const float* as, const int8_t* b, const float* bs, const float* bias, int64_t m, int64_t n, int k,
                       void* out, int dtype, void* space, hipStream_t s)
{
    TileRows Y{(const char*)a, m, (uint32_t)k, (uint32_t)k}, X{(const char*)b, n, (uint32_t)k, (uint32_t)k};
    if (!product_as_is(m, k)) {
        // (a width of its own only for a length that is no multiple of 16, where both are copied)
        TgCarve c{(char*)space, 0};
        const auto copy = [&](TileRows& rows, const int8_t* p) {
            const bool ready = tile_ready(p, k, k, 1);
            rows.pitch = rows.width = tile_pitch(k, 1);
            char* const place = c.take<char>((size_t)rows.rows * rows.pitch);
            if (ready) return;
            tg_launch_pack(p, k, rows.rows, k, 1, place, s);
            rows.p = place;
        };
        copy(Y, a);
        copy(X, b);
    }
    const int bytes = (int)X.width;
    if (m <= PRODUCT_FEW && bytes > PRODUCT_SHORT) {
        const int64_t most = TILE_LAUNCH_ITEMS / 256 * 16;
        for (int64_t x0 = 0; x0 < n; x0 += most) {
            const dim3 g((unsigned)(((n - x0 < most ? n - x0 : most) + 15) / 16)), t(256);
            TG_WITH_TYPE(dtype, O, {
                if (m <= 16) hipLaunchKernelGGL((product_few_kernel<O, 1>), g, t, 0, s, X, Y, bytes, as, bs, bias, x0, (O*)out);
                else if (m <= 32) hipLaunchKernelGGL((product_few_kernel<O, 2>), g, t, 0, s, X, Y, bytes, as, bs, bias, x0, (O*)out);
                else hipLaunchKernelGGL((product_few_kernel<O, 4>), g, t, 0, s, X, Y, bytes, as, bs, bias, x0, (O*)out);
            });
        }
        return;
    }
    TG_WITH_TYPE(dtype, O, launch_product<O>(X, Y, bytes, as, bs, bias, (O*)out, s));
}
