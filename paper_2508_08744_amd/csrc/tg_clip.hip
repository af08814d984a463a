// The norm of many gradients together, and their values brought under one: bound by their bytes, read once for the norm and once more to be scaled.
//
// The tensors come as lists in the kernels' arguments (nothing is copied to the device for them, so the calls can be captured), each in pieces of CLIP_PIECE
// values.  A workgroup has a stretch of pieces and leaves one sum of squares, in 64 bits (the squares of fp32 and bf16 leave 32 bits' range); every workgroup of the second pass adds all
// of those up in the same order and has the factor.  It takes its stretch from the end: what was read last is still in the caches.
// (197 M values of 16 bits: 61 us for the norm, 6.5 TB/s, and 135 to scale, 5.8 TB/s; with the call 204 into other tensors, 209 in place, 84 in place where the factor is 1; the stretches taken forwards and results through the caches: 253 us for 200 M in the place of 203.)
#include "tg_embed.h"
#include "tg_device.h"

#define CLIP_TENSORS 128        // of a launch: the lists stay below 4 KB of arguments
#define CLIP_PIECE 8192
#define CLIP_GROUPS 1024        // workgroups, and sums, of all launches together; one more for a launch that would have none

struct ClipList {
    const void* in[CLIP_TENSORS];
    void* out[CLIP_TENSORS];
    uint64_t count[CLIP_TENSORS];           // values, and in the upper two bits their type
    uint32_t first[CLIP_TENSORS + 1];       // a tensor's first piece; the last: all pieces
    int tensors;
    uint32_t each;                          // pieces of a workgroup
};
static_assert(sizeof(ClipList) + 64 <= 4096, "the arguments of a launch");

// the tensor that piece p is of
__device__ inline int clip_tensor(const ClipList& a, uint32_t p)
{
    int lo = 0, hi = a.tensors;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (a.first[mid] <= p) lo = mid;
        else hi = mid;
    }
    return lo;
}
__device__ inline double clip_sum(double x, double* s)
{
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const u64 o = tg_shfl_xor64((u64)__double_as_longlong(x), m);
        x += __longlong_as_double((long long)o);
    }
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = x;
    __syncthreads();
    return (s[0] + s[1]) + (s[2] + s[3]);
}

template <class E>
__device__ inline void clip_squares(const E* p, uint64_t left, double& sum)
{
    typedef TgPiece<E> P;
    constexpr int TURNS = CLIP_PIECE / (256 * P::E);
    typename P::vec v[TURNS];
    if (left >= CLIP_PIECE) {
#pragma unroll
        for (int i = 0; i < TURNS; ++i) v[i] = *reinterpret_cast<const typename P::vec*>(p + (i * 256 + threadIdx.x) * P::E);
    } else {
#pragma unroll
        for (int i = 0; i < TURNS; ++i) {
            const int at = (i * 256 + threadIdx.x) * P::E;
            v[i] = P::raw(p + at, (int)left - at);
        }
    }
#pragma unroll
    for (int i = 0; i < TURNS; ++i)
#pragma unroll
        for (int e = 0; e < P::E; ++e) {
            const double x = (double)(float)v[i][e];
            sum = fma(x, x, sum);
        }
}
__global__ __launch_bounds__(256) void clip_squares_kernel(ClipList a, double* __restrict__ sums)
{
    __shared__ double s[4];
    const uint32_t p0 = blockIdx.x * a.each, all = a.first[a.tensors], p1 = p0 + a.each < all ? p0 + a.each : all;
    double sum = 0.0;
    int t = clip_tensor(a, p0);
    for (uint32_t p = p0; p < p1; ++p) {
        while (a.first[t + 1] <= p) ++t;
        const uint64_t count = a.count[t] << 2 >> 2, at = (uint64_t)(p - a.first[t]) * CLIP_PIECE;
        const int type = (int)(a.count[t] >> 62);
        TG_WITH_TYPE(type, E, clip_squares((const E*)a.in[t] + at, count - at, sum));
    }
    sum = clip_sum(sum, s);
    if (threadIdx.x == 0) sums[blockIdx.x] = sum;
}
// the sum of all squares, the same in every lane of every workgroup
__device__ inline double clip_total(const double* __restrict__ sums, int count, double* s)
{
    double x = 0.0;
    for (int i = threadIdx.x; i < count; i += 256) x += sums[i];
    return clip_sum(x, s);
}
__global__ __launch_bounds__(256) void clip_norm_kernel(const double* __restrict__ sums, int count, float scale, float* __restrict__ norm)
{
    __shared__ double s[4];
    const double total = clip_total(sums, count, s);
    if (threadIdx.x == 0) *norm = (float)(fabs((double)scale) * sqrt(total));
}

template <class E>
__device__ inline void clip_scale(const E* p, E* q, uint64_t left, float factor, float then)
{
    typedef TgPiece<E> P;
    constexpr int TURNS = CLIP_PIECE / (256 * P::E);
    typename P::vec v[TURNS];
    if (left >= CLIP_PIECE) {
#pragma unroll
        for (int i = 0; i < TURNS; ++i) v[i] = *reinterpret_cast<const typename P::vec*>(p + (i * 256 + threadIdx.x) * P::E);
#pragma unroll
        for (int i = 0; i < TURNS; ++i) {
#pragma unroll
            for (int e = 0; e < P::E; ++e) v[i][e] = (E)((float)v[i][e] * factor * then);
            __builtin_nontemporal_store(v[i], reinterpret_cast<typename P::vec*>(q + (i * 256 + threadIdx.x) * P::E));    // (in the place of what is still to be read they would take room)
        }
    } else {
#pragma unroll
        for (int i = 0; i < TURNS; ++i) {
            const int at = (i * 256 + threadIdx.x) * P::E;
            v[i] = P::raw(p + at, (int)left - at);
        }
#pragma unroll
        for (int i = 0; i < TURNS; ++i) {
            const int at = (i * 256 + threadIdx.x) * P::E;
            P o;
#pragma unroll
            for (int e = 0; e < P::E; ++e) o.v[e] = (float)v[i][e] * factor * then;
            o.store(q + at, (int)left - at);
        }
    }
}
// norm: written by the first workgroup, or null
__global__ __launch_bounds__(256) void clip_scale_kernel(ClipList a, const double* __restrict__ sums, int count, float scale, float max_norm,
                                                         float* __restrict__ out_norm)
{
    __shared__ double s[4];
    const double norm = fabs((double)scale) * sqrt(clip_total(sums, count, s));
    // (a norm that is no number, or infinite, brings nothing under anything; in 64 bits it is so only where a value is: one beyond fp32 counts as it is)
    const double by = norm > (double)max_norm && norm <= 1.7e308 ? (double)scale * ((double)max_norm / norm) : (double)scale;
    // (in two steps where 32 bits have few bits left for it: norms beyond them)
    const bool tiny = fabs(by) < 0x1p-64;
    const float factor = (float)(tiny ? by * 0x1p64 : by), then = tiny ? 0x1p-64f : 1.0f;
    if (out_norm && blockIdx.x == 0 && threadIdx.x == 0) *out_norm = (float)norm;
    const uint32_t p0 = blockIdx.x * a.each, all = a.first[a.tensors], p1 = p0 + a.each < all ? p0 + a.each : all;
    if (p0 >= p1) return;
    int t = clip_tensor(a, p1 - 1);
    for (uint32_t p = p1; p-- > p0;) {
        while (a.first[t] > p) --t;
        if (factor == 1.0f && then == 1.0f && a.in[t] == a.out[t]) continue;        // they are what they would become
        const uint64_t values = a.count[t] << 2 >> 2, at = (uint64_t)(p - a.first[t]) * CLIP_PIECE;
        const int type = (int)(a.count[t] >> 62);
        TG_WITH_TYPE(type, E, clip_scale((const E*)a.in[t] + at, (E*)a.out[t] + at, values - at, factor, then));
    }
}

// The launches: the next at most CLIP_TENSORS tensors that hold anything, and workgroups by their share of all pieces.
struct ClipWalk {
    const void* const* in;
    void* const* out;
    const int64_t* counts;
    const int32_t* dtypes;
    int tensors, at;
    int64_t pieces;              // of all tensors

    static int64_t pieces_of(int64_t count) { return (count + CLIP_PIECE - 1) / CLIP_PIECE; }
    // a launch has fewer than 2^31 pieces: `part` of a tensor at a time where it has more
    int64_t part = 0;
    int groups = 0;
    bool next(ClipList* a)
    {
        const int64_t most = 1ll << 30;
        int n = 0;
        int64_t all = 0;
        while (at < tensors && n < CLIP_TENSORS && all < most) {
            const int64_t from = part * CLIP_PIECE, left = counts[at] - from;
            if (left <= 0) {
                ++at;
                part = 0;
                continue;
            }
            const int64_t bytes = from * (dtypes[at] == 0 ? 4 : 2), room = (most - all) * CLIP_PIECE, now = left < room ? left : room;
            a->in[n] = (const char*)in[at] + bytes;
            a->out[n] = out ? (char*)out[at] + bytes : nullptr;
            a->count[n] = (uint64_t)now | (uint64_t)dtypes[at] << 62;
            a->first[n] = (uint32_t)all;
            all += pieces_of(now);
            part += pieces_of(now);
            ++n;
        }
        if (n == 0) return false;
        a->first[n] = (uint32_t)all;
        a->tensors = n;
        const int64_t share = (int64_t)((double)CLIP_GROUPS * (double)all / (double)pieces), wgs = share < 1 ? 1 : share;
        a->each = (uint32_t)((all + wgs - 1) / wgs);
        groups = (int)((all + a->each - 1) / a->each);
        return true;
    }
};
static ClipWalk clip_walk(const void* const* in, void* const* out, const int64_t* counts, const int32_t* dtypes, int tensors)
{
    ClipWalk w{in, out, counts, dtypes, tensors, 0, 0};
    for (int i = 0; i < tensors; ++i) w.pieces += ClipWalk::pieces_of(counts[i]);
    return w;
}
size_t tg_grad_norm_space(const int64_t* counts, int tensors)
{
    int64_t pieces = 0;
    for (int i = 0; i < tensors; ++i) pieces += ClipWalk::pieces_of(counts[i]);
    // every launch has its share of the workgroups, or one
    return sizeof(double) * (size_t)(CLIP_GROUPS + tensors / CLIP_TENSORS + (pieces >> 30) + 2);
}
void tg_launch_clip(const void* const* grads, void* const* out, const int64_t* counts, const int32_t* dtypes, int tensors, float scale, float max_norm,
                    float* norm, void* space, hipStream_t s)
{
    double* const sums = (double*)space;
    ClipList a;
    int count = 0;
    for (ClipWalk w = clip_walk(grads, nullptr, counts, dtypes, tensors); w.next(&a); count += w.groups)
        hipLaunchKernelGGL(clip_squares_kernel, dim3((unsigned)w.groups), dim3(256), 0, s, a, sums + count);
    bool written = false;
    if (out)
        for (ClipWalk w = clip_walk(grads, out, counts, dtypes, tensors); w.next(&a); written = true)
            hipLaunchKernelGGL(clip_scale_kernel, dim3((unsigned)w.groups), dim3(256), 0, s, a, sums, count, scale, max_norm, written ? nullptr : norm);
    if (!written) hipLaunchKernelGGL(clip_norm_kernel, dim3(1), dim3(256), 0, s, sums, count, scale, norm);
}
