// Root-mean-square norm with the residual's addition, its gradient, and rows on an 8-bit grid with a scale each.
//
// All of these are bound by the bytes of their rows: a row is read once, stays in the registers of the lanes that share it (a wave where
// it is short, a workgroup of up to 16 waves where it is long) through its sums, and is written once.  (30 011 rows of 960 bf16: 42 us there, 5.5 TB/s, 42 back; with
// the rows of the gradient asked for one by one 54.)
#include "tg_embed.h"
#include "tg_device.h"

// T lanes of a workgroup share a row; CH pieces of 16 bytes of it a lane.
template <int T> struct NormShare { static constexpr int ROWS = T < 256 ? 256 / T : 1, THREADS = T < 256 ? 256 : T; };

// What is left of a row from a lane's piece on.  Rows of whole pieces (WHOLE) have one or none: the kernels then hold no code for parts
// of a piece, which is most of it otherwise.
template <class E, bool WHOLE>
__device__ inline int norm_left(int left) { return !WHOLE ? left : left > 0 ? TgPiece<E>::E : 0; }

template <class V>
__device__ inline V wave_sum(V x)
{
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) x += __shfl_xor(x, m);
    return x;
}
// sum over the T lanes of a row, the same in all of them; `s`: a word per wave, not used by the sum before
template <int T, class V>
__device__ inline V row_sum(V x, V* s)
{
    x = wave_sum(x);
    if (T == 64) return x;
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = x;
    __syncthreads();
    V y = s[0];
#pragma unroll
    for (int i = 1; i < T / 64; ++i) y += s[i];
    return y;
}
// their maximum
template <int T>
__device__ inline double row_max64(double x, double* s)
{
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) x = fmax(x, __shfl_xor(x, m));
    if (T == 64) return x;
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = x;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < T / 64; ++i) x = fmax(x, s[i]);
    return x;
}

template <class E, int T, int CH, bool WHOLE>
__global__ __launch_bounds__(NormShare<T>::THREADS) void norm_kernel(const E* x, int64_t ld_x, const E* res, int64_t ld_res,
                                                                     const E* __restrict__ w, int64_t n, int d, float eps, E* __restrict__ y,
                                                                     E* r, float* __restrict__ rstd_out)
{
    typedef TgPiece<E> P;
    __shared__ float s_sum[16];
    __shared__ double s_sum64[16];
    const int lane = threadIdx.x % T;
    const int64_t row = (int64_t)blockIdx.x * NormShare<T>::ROWS + threadIdx.x / T;
    if (row >= n) return;                                   // (whole waves: with T > 64 a workgroup has one row)
    P p[CH];
    float sum = 0.0f;
#pragma unroll
    for (int c = 0; c < CH; ++c) p[c].load(x + row * ld_x + (lane + c * T) * P::E, norm_left<E, WHOLE>(d - (lane + c * T) * P::E));
    if (res) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int at = (lane + c * T) * P::E;
            P q;
            q.load(res + row * ld_res + at, norm_left<E, WHOLE>(d - at));
#pragma unroll
            for (int i = 0; i < P::E; ++i) p[c].v[i] += q.v[i];
            p[c].round();
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) p[c].store(r + row * d + (lane + c * T) * P::E, norm_left<E, WHOLE>(d - (lane + c * T) * P::E));
    }
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < P::E; ++i) sum = fmaf(p[c].v[i], p[c].v[i], sum);
    const float mean = row_sum<T>(sum, s_sum) / (float)d + eps;
    float rstd = 1.0f / sqrtf(mean);
    // (squares that leave fp32's range, above or below: rows beyond 1.8e19, or of less than 1e-15 under no eps to speak of)
    if (__builtin_expect(!(mean >= 0x1p-100f && mean <= 3.4028234e38f), 0)) {
        double sum64 = 0.0;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < P::E; ++i) {
                asm volatile("" : "+v"(p[c].v[i]));        // (nothing of this is made out where it is not needed)
                sum64 = fma((double)p[c].v[i], (double)p[c].v[i], sum64);
            }
        rstd = (float)(1.0 / sqrt(row_sum<T>(sum64, s_sum64) / d + (double)eps));
    }
    if (rstd_out && lane == 0) rstd_out[row] = rstd;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int at = (lane + c * T) * P::E;
        P g;
        g.load(w + at, norm_left<E, WHOLE>(d - at));
#pragma unroll
        for (int i = 0; i < P::E; ++i) g.v[i] *= p[c].v[i] * rstd;
        g.store(y + row * d + at, norm_left<E, WHOLE>(d - at));
    }
}

// 1 / sqrt(x) and 1 / x in 64 bits from the instructions' estimates, to a few units in the last place: each step of Newton's doubles the bits, of
// which the estimates have 20 or more.  (Zero and infinity give NaN.)
__device__ inline double norm_rsqrt(double x)
{
    double y = __builtin_amdgcn_rsq(x);
#pragma unroll
    for (int i = 0; i < 2; ++i) y = fma(0.5 * y, fma(-x * y, y, 1.0), y);
    return y;
}
__device__ inline double norm_rcp(double x)
{
    double y = __builtin_amdgcn_rcp(x);
#pragma unroll
    for (int i = 0; i < 2; ++i) y = fma(y, fma(-x, y, 1.0), y);
    return y;
}

// The norm in 64 bits, the normed row on its grid.  Which whole number a value next to a border becomes must not depend on how its row
// was summed, so sum, scale and quotient are taken in 64 bits; the bytes of the rows still bound the kernel.  A 16-bit value times its weight is exact in
// 32 bits while it stays within their range (a row that leaves it takes its products in 64 bits), and so is its quotient's
// rounding, except next to a border.  (16 384 rows of 4096 bf16: 100 us, 4.7 TB/s, as a copy; 109
// with the divisions and the root spelt out and code for parts of a piece.)
template <class E, int T, int CH, bool WHOLE, bool NORM>
__global__ __launch_bounds__(NormShare<T>::THREADS) void norm_q8_kernel(const E* x, int64_t ld_x, const E* res, int64_t ld_res,
                                                                        const E* __restrict__ w, int64_t n, int d, double per_d, float eps,
                                                                        int8_t* __restrict__ q_out, float* __restrict__ scale_out, E* r)
{
    typedef TgPiece<E> P;
    typedef char qvec __attribute__((ext_vector_type(P::E), aligned(1)));
    __shared__ double s_sum[16];
    __shared__ double s_max[16];
    const int lane = threadIdx.x % T;
    const int64_t row = (int64_t)blockIdx.x * NormShare<T>::ROWS + threadIdx.x / T;
    if (row >= n) return;
    P p[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) p[c].load(x + row * ld_x + (lane + c * T) * P::E, norm_left<E, WHOLE>(d - (lane + c * T) * P::E));
    double rstd = 1.0;
    if (NORM) {
        if (res) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int at = (lane + c * T) * P::E;
                P q;
                q.load(res + row * ld_res + at, norm_left<E, WHOLE>(d - at));
#pragma unroll
                for (int i = 0; i < P::E; ++i) p[c].v[i] += q.v[i];
                p[c].round();
            }
#pragma unroll
            for (int c = 0; c < CH; ++c) p[c].store(r + row * d + (lane + c * T) * P::E, norm_left<E, WHOLE>(d - (lane + c * T) * P::E));
        }
        double sum = 0.0;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < P::E; ++i) sum = fma((double)p[c].v[i], (double)p[c].v[i], sum);
        rstd = norm_rsqrt(fma(row_sum<T>(sum, s_sum), per_d, (double)eps));
    }
    // max |r w|, and whether a value is NaN (a maximum leaves it out)
    constexpr bool SHORT = sizeof(E) == 2;
    double top = 0.0;
    float top32 = 0.0f;
    bool odd = false;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int at = (lane + c * T) * P::E;
        P g;
        if (NORM) g.load(w + at, norm_left<E, WHOLE>(d - at));
#pragma unroll
        for (int i = 0; i < P::E; ++i) {
            if (SHORT) {
                if (NORM) p[c].v[i] *= g.v[i];
                odd |= !(p[c].v[i] == p[c].v[i]);
                top32 = fmaxf(top32, fabsf(p[c].v[i]));
            } else {
                const double t = NORM ? (double)p[c].v[i] * (double)g.v[i] : (double)p[c].v[i];
                odd |= !(t == t);
                top = fmax(top, fabs(t));
            }
        }
    }
    if (SHORT) top = top32 <= 3.4028234e38f ? (double)top32 : 1e300;        // (beyond fp32: to be found out)
    if (odd) top = __builtin_inf();
    top = row_max64<T>(top, s_max);
    // (only bf16 has values whose products leave fp32's range: 1e-30 is far enough above its end for what is lost there to be zero on the grid)
    const bool wide = NORM && __is_same(E, tg_bf16) && !(top >= 1e-30 && top <= 3.4028234e38) && top <= 1e300;
    const E* again = res ? r + row * d : x + row * ld_x;
    if (wide) {
        top = 0.0;
#pragma unroll 1
        for (int at = lane * P::E; at < d; at += T * P::E) {
            P z, g;
            z.load(again + at, norm_left<E, WHOLE>(d - at));
            g.load(w + at, norm_left<E, WHOLE>(d - at));
#pragma unroll
            for (int i = 0; i < P::E; ++i) top = fmax(top, fabs((double)z.v[i] * (double)g.v[i]));
        }
        top = row_max64<T>(top, s_sum);
    }
    float scale = (float)(top * rstd * (1.0 / 127.0));
    // not a number, an infinite row, or one whose norm is: no grid
    const bool none = !(top <= 1.79e308) || !(rstd <= 1.79e308) || !(scale <= 3.4028234e38f);
    if (none) scale = __builtin_nanf("");
    if (lane == 0) scale_out[row] = scale;
    const double f = none || scale == 0.0f ? 0.0 : rstd * norm_rcp((double)scale);
    const float f32 = (float)f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int at = (lane + c * T) * P::E, left = norm_left<E, WHOLE>(d - at);
        qvec q;
        // (a scale below fp32's normal numbers has few bits of its own: the quotient can pass 127)
        if (SHORT) {
            // the quotient in 32 bits is off by less than 127 x 2^-22: it decides unless it lies that near to a border, or is no finite number (a
            // factor that fp32 does not hold, of rows that stay below 127 / 3.4e38)
            bool near = false;
#pragma unroll
            for (int i = 0; i < P::E; ++i) {
                const float u = p[c].v[i] * f32, whole = rintf(u);
                q[i] = (char)(int)fminf(fmaxf(whole, -127.0f), 127.0f);
                near |= !(fabsf(u - whole) <= 0.5f - 1e-4f);
            }
            if (near) {
#pragma unroll
                for (int i = 0; i < P::E; ++i) q[i] = (char)(int)fmin(fmax(rint((double)p[c].v[i] * f), -127.0), 127.0);
            }
            if (wide) {
                P z, g;
                z.load(again + at, left);
                g.load(w + at, left);
#pragma unroll
                for (int i = 0; i < P::E; ++i) q[i] = (char)(int)fmin(fmax(rint((double)z.v[i] * (double)g.v[i] * f), -127.0), 127.0);
            }
            if (none) q = (qvec)0;
        } else {
            P g;
            if (NORM) g.load(w + at, left);
#pragma unroll
            for (int i = 0; i < P::E; ++i) {
                const double t = NORM ? (double)p[c].v[i] * (double)g.v[i] : (double)p[c].v[i];
                q[i] = (char)(int)(none ? 0.0 : fmin(fmax(rint(t * f), -127.0), 127.0));
            }
        }
        int8_t* o = q_out + row * d + at;
        if (left >= P::E) *reinterpret_cast<qvec*>(o) = q;
        else
#pragma unroll
            for (int i = 0; i < P::E; ++i)
                if (i < left) o[i] = (int8_t)q[i];
    }
}

template <class E>
__global__ __launch_bounds__(256) void dequantize_kernel(const int8_t* __restrict__ q, const float* __restrict__ scale, int64_t n, int d,
                                                         int pieces, E* __restrict__ out)
{
    typedef TgPiece<E> P;
    typedef char qvec __attribute__((ext_vector_type(P::E), aligned(1)));
    const int64_t all = n * pieces;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / pieces;
        const int at = (int)(i - row * pieces) * P::E, left = d - at;
        const float s = scale[row];
        P p;
        if (left >= P::E) {
            const qvec x = *reinterpret_cast<const qvec*>(q + row * d + at);
#pragma unroll
            for (int j = 0; j < P::E; ++j) p.v[j] = (float)(int8_t)x[j] * s;
        } else {
#pragma unroll
            for (int j = 0; j < P::E; ++j) p.v[j] = j < left ? (float)q[row * d + at + j] * s : 0.0f;
        }
        p.store(out + row * d + at, left);
    }
}

// u = dy w, c = mean(u r): dx = dr + rstd (u - r rstd^2 c), dw = sum over rows of dy r rstd.  A workgroup takes every gridDim.x-th
// group of rows and keeps its part of dw in registers; the parts are added by norm_dw_kernel in the workgroups' order.
template <class E, int T, int CH, bool WHOLE>
__global__ __launch_bounds__(NormShare<T>::THREADS) void norm_grad_kernel(const E* __restrict__ dy, int64_t ld_dy, const E* dr, int64_t ld_dr,
                                                                          const E* __restrict__ r, int64_t ld_r, const E* __restrict__ w,
                                                                          const float* __restrict__ rstd_in, int64_t n, int d, E* dx,
                                                                          float* __restrict__ parts)
{
    typedef TgPiece<E> P;
    constexpr int ROWS = NormShare<T>::ROWS;
    __shared__ float s_sum[2][16];
    const int lane = threadIdx.x % T;
    float dw[CH][P::E];
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < P::E; ++i) dw[c][i] = 0.0f;
    // the row behind is asked for while this one is summed
    typename P::vec a_dy[CH], a_r[CH], a_dr[CH], gw[CH];
    float a_rstd = 0.0f;
    const int64_t step = (int64_t)gridDim.x * ROWS;
    int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / T;
    const auto ask = [&](int64_t i) {
        a_rstd = rstd_in[i];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int at = (lane + c * T) * P::E, left = norm_left<E, WHOLE>(d - at);
            a_dy[c] = P::raw(dy + i * ld_dy + at, left);
            a_r[c] = P::raw(r + i * ld_r + at, left);
            if (dr) a_dr[c] = P::raw(dr + i * ld_dr + at, left);
        }
    };
#pragma unroll
    for (int c = 0; c < CH; ++c) gw[c] = P::raw(w + (lane + c * T) * P::E, norm_left<E, WHOLE>(d - (lane + c * T) * P::E));
    if (row < n) ask(row);
    int turn = 0;
    for (; row < n; row += step) {
        P u[CH], z[CH];
        typename P::vec b_dr[CH];
        const float rstd = a_rstd;
        float sum = 0.0f;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            b_dr[c] = a_dr[c];
#pragma unroll
            for (int i = 0; i < P::E; ++i) {
                const float v = (float)a_dy[c][i];
                z[c].v[i] = (float)a_r[c][i] * rstd;
                dw[c][i] = fmaf(v, z[c].v[i], dw[c][i]);
                u[c].v[i] = v * (float)gw[c][i];
                sum = fmaf(u[c].v[i], z[c].v[i], sum);
            }
        }
        if (row + step < n) ask(row + step);
        // (two sets of words in turn: a wave may be a row ahead of another that still reads its sum)
        const float mean = row_sum<T>(sum, s_sum[turn]) / (float)d;
        turn ^= 1;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int at = (lane + c * T) * P::E;
            P o;
#pragma unroll
            for (int i = 0; i < P::E; ++i) {
                const float v = rstd * (u[c].v[i] - z[c].v[i] * mean);
                o.v[i] = dr ? (float)b_dr[c][i] + v : v;
            }
            o.store(dx + row * d + at, norm_left<E, WHOLE>(d - at));
        }
    }
    // the rows that a workgroup had in hand at a time are added, the first with the second and so on, and leave one part
    if (ROWS > 1) {
        __shared__ float s_dw[ROWS > 1 ? ROWS - 1 : 1][CH * P::E][64];
        const int wave = threadIdx.x >> 6;
        if (wave > 0) {
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < P::E; ++i) s_dw[wave > 0 ? wave - 1 : 0][c * P::E + i][lane] = dw[c][i];
        }
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int r = 0; r < ROWS - 1; ++r)
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < P::E; ++i) dw[c][i] += s_dw[r][c * P::E + i][lane];
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int at = (lane + c * T) * P::E;
#pragma unroll
        for (int i = 0; i < P::E; ++i)
            if (at + i < d) parts[(int64_t)blockIdx.x * d + at + i] = dw[c][i];
    }
}
// 16 columns a workgroup, 64 lanes a column: lane j of a column adds the parts j, j + 64, ..., then the lanes are added as a tree
template <class E>
__global__ __launch_bounds__(1024) void norm_dw_kernel(const float* __restrict__ parts, int count, int d, E* __restrict__ dw)
{
    __shared__ float s[64][17];
    const int c = threadIdx.x & 15, j = threadIdx.x >> 4;
    const int col = blockIdx.x * 16 + c;
    float sum = 0.0f;
    if (col < d) {
#pragma unroll 8
        for (int p = j; p < count; p += 64) sum += parts[(int64_t)p * d + col];
    }
    s[j][c] = sum;
    __syncthreads();
#pragma unroll
    for (int h = 32; h >= 1; h >>= 1) {
        if (j < h) s[j][c] += s[j + h][c];
        __syncthreads();
    }
    if (j == 0 && col < d) dw[col] = (E)s[0][c];
}

// The lanes a row of `d` elements gets and the pieces a lane holds: a wave up to two pieces a lane (1024 elements of 16 bits), four
// waves up to four (8192), sixteen beyond (8192 elements of 32 bits).
#define NORM_SHAPE(pieces, WHOLE, LAUNCH)                                            \
    do {                                                                             \
        if ((pieces) <= 64) { LAUNCH(64, 1, WHOLE); }                                \
        else if ((pieces) <= 128) { LAUNCH(64, 2, WHOLE); }                          \
        else if ((pieces) <= 256) { LAUNCH(256, 1, WHOLE); }                         \
        else if ((pieces) <= 512) { LAUNCH(256, 2, WHOLE); }                         \
        else if ((pieces) <= 1024) { LAUNCH(256, 4, WHOLE); }                        \
        else { LAUNCH(1024, 2, WHOLE); }                                             \
    } while (0)
#define NORM_SHAPES(E, d, LAUNCH)                                                    \
    do {                                                                             \
        const int pieces_ = ((d) + TgPiece<E>::E - 1) / TgPiece<E>::E;               \
        if ((d) % TgPiece<E>::E == 0) { NORM_SHAPE(pieces_, true, LAUNCH); }         \
        else { NORM_SHAPE(pieces_, false, LAUNCH); }                                 \
    } while (0)

// rows of one launch: below 2^32 work-items
#define NORM_LAUNCH_ROWS (1ll << 21)

template <class F>
static void norm_chunks(int64_t n, F launch)
{
    for (int64_t r0 = 0; r0 < n; r0 += NORM_LAUNCH_ROWS) launch(r0, n - r0 < NORM_LAUNCH_ROWS ? n - r0 : NORM_LAUNCH_ROWS);
}

void tg_launch_norm(const void* x, int64_t ld_x, const void* res, int64_t ld_res, const void* w, int dtype, int64_t n, int d, float eps,
                    void* y, void* r, float* rstd, hipStream_t s)
{
    norm_chunks(n, [&](int64_t r0, int64_t nr) {
#define NORM_FWD(T, CH, W)                                                                                                                  \
    hipLaunchKernelGGL((norm_kernel<E, T, CH, W>), dim3((unsigned)((nr + NormShare<T>::ROWS - 1) / NormShare<T>::ROWS)),                     \
                       dim3(NormShare<T>::THREADS), 0, s, (const E*)x + r0 * ld_x, ld_x, res ? (const E*)res + r0 * ld_res : nullptr,     \
                       ld_res, (const E*)w, nr, d, eps, (E*)y + r0 * d, r ? (E*)r + r0 * d : nullptr, rstd ? rstd + r0 : nullptr)
        TG_WITH_TYPE(dtype, E, NORM_SHAPES(E, d, NORM_FWD));
    });
}

void tg_launch_norm_q8(const void* x, int64_t ld_x, const void* res, int64_t ld_res, const void* w, int dtype, int64_t n, int d, float eps,
                       int8_t* q, float* scale, void* r, hipStream_t s)
{
    norm_chunks(n, [&](int64_t r0, int64_t nr) {
#define NORM_Q8(T, CH, W)                                                                                                                   \
    do {                                                                                                                                 \
        const dim3 g((unsigned)((nr + NormShare<T>::ROWS - 1) / NormShare<T>::ROWS)), b(NormShare<T>::THREADS);                           \
        const E* xr = (const E*)x + r0 * ld_x;                                                                                           \
        const E* rr = res ? (const E*)res + r0 * ld_res : nullptr;                                                                       \
        if (w) hipLaunchKernelGGL((norm_q8_kernel<E, T, CH, W, true>), g, b, 0, s, xr, ld_x, rr, ld_res, (const E*)w, nr, d, 1.0 / d, eps, q + r0 * d, \
                                  scale + r0, r ? (E*)r + r0 * d : nullptr);                                                             \
        else hipLaunchKernelGGL((norm_q8_kernel<E, T, CH, W, false>), g, b, 0, s, xr, ld_x, rr, ld_res, (const E*)w, nr, d, 1.0 / d, eps, q + r0 * d,  \
                                scale + r0, (E*)nullptr);                                                                                \
    } while (0)
        TG_WITH_TYPE(dtype, E, NORM_SHAPES(E, d, NORM_Q8));
    });
}

void tg_launch_dequantize(const int8_t* q, const float* scale, int64_t n, int d, int dtype, void* out, hipStream_t s)
{
    if (n == 0) return;
    TG_WITH_TYPE(dtype, E, {
        const int pieces = (d + TgPiece<E>::E - 1) / TgPiece<E>::E;
        const int64_t wgs = (n * pieces + 255) / 256;
        hipLaunchKernelGGL(dequantize_kernel<E>, dim3((unsigned)(wgs < 16384 ? wgs : 16384)), dim3(256), 0, s, q, scale, n, d, pieces, (E*)out);
    });
}

// workgroups of the gradient: each leaves a part of dw
#define NORM_GRAD_WGS 1024
static int64_t norm_grad_wgs(int64_t n, int rows)
{
    const int64_t wgs = (n + rows - 1) / rows;
    return wgs < NORM_GRAD_WGS ? wgs : NORM_GRAD_WGS;
}
size_t tg_norm_grad_space(int64_t n, int d) { return (size_t)norm_grad_wgs(n, 1) * d * sizeof(float); }

void tg_launch_norm_grad(const void* dy, int64_t ld_dy, const void* dr, int64_t ld_dr, const void* r, int64_t ld_r, const void* w,
                         const float* rstd, int dtype, int64_t n, int d, void* dx, void* dw, void* space, hipStream_t s)
{
    float* parts = (float*)space;
    int64_t count = 0;
#define NORM_BWD(T, CH, W)                                                                                                                  \
    do {                                                                                                                                 \
        count = norm_grad_wgs(n, NormShare<T>::ROWS);                                                                                  \
        if (n > 0)                                                                                                                       \
            hipLaunchKernelGGL((norm_grad_kernel<E, T, CH, W>), dim3((unsigned)count), dim3(NormShare<T>::THREADS), 0, \
                               s, (const E*)dy, ld_dy, (const E*)dr, ld_dr, (const E*)r, ld_r, (const E*)w, rstd, n, d, (E*)dx, parts);   \
        hipLaunchKernelGGL(norm_dw_kernel<E>, dim3((unsigned)((d + 15) / 16)), dim3(1024), 0, s, parts, (int)count, d, (E*)dw);           \
    } while (0)
    TG_WITH_TYPE(dtype, E, NORM_SHAPES(E, d, NORM_BWD));
}
