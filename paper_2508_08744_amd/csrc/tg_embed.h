// Shared by the operators behind include/tagore_embed.h: element types, 16-byte pieces of rows, and the launchers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

typedef __bf16 tg_bf16;
typedef _Float16 tg_f16;

// 16 bytes of a row.  A row may begin at any element, so the type carries the element's alignment alone: the compiler still makes one
// 16-byte access of it (gfx950 takes any alignment), and rows that are aligned pay nothing.
template <class T> struct TgPiece {
    static constexpr int E = 16 / (int)sizeof(T);
    typedef T vec __attribute__((ext_vector_type(E), aligned(sizeof(T))));
    float v[E];
    // the 16 bytes as they are: held until they are needed they take half the registers of 16-bit values
    static __device__ inline vec raw(const T* p, int left)
    {
        if (left >= E) return *reinterpret_cast<const vec*>(p);
        vec x;
#pragma unroll
        for (int i = 0; i < E; ++i) x[i] = i < left ? p[i] : (T)0.0f;
        return x;
    }
    // `left` elements of the row from p on (E or more: a whole piece); what is not there reads as zero
    __device__ inline void load(const T* p, int left)
    {
        if (left >= E) {
            const vec x = *reinterpret_cast<const vec*>(p);
#pragma unroll
            for (int i = 0; i < E; ++i) v[i] = (float)x[i];
        } else {
#pragma unroll
            for (int i = 0; i < E; ++i) v[i] = i < left ? (float)p[i] : 0.0f;
        }
    }
    __device__ inline void store(T* p, int left) const
    {
        if (left >= E) {
            vec x;
#pragma unroll
            for (int i = 0; i < E; ++i) x[i] = (T)v[i];
            *reinterpret_cast<vec*>(p) = x;
        } else {
#pragma unroll
            for (int i = 0; i < E; ++i)
                if (i < left) p[i] = (T)v[i];
        }
    }
    // the values as a row of the type would hold them
    __device__ inline void round()
    {
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = (float)(T)v[i];
    }
};

// ids of 32 or 64 bits: the row, or -1 where there is none
__device__ inline int64_t tg_row_of(const void* ids, int ids64, int64_t t, int64_t n_rows)
{
    const int64_t v = ids64 ? reinterpret_cast<const int64_t*>(ids)[t] : (int64_t)reinterpret_cast<const int32_t*>(ids)[t];
    return v >= 0 && v < n_rows ? v : -1;
}

// one of the three types, by number (checked before)
#define TG_WITH_TYPE(dtype, T, ...)                     \
    do {                                                \
        if ((dtype) == 0) { typedef float T; __VA_ARGS__; }        \
        else if ((dtype) == 1) { typedef tg_bf16 T; __VA_ARGS__; } \
        else { typedef tg_f16 T; __VA_ARGS__; }         \
    } while (0)

static inline size_t tg_type_bytes(int dtype) { return dtype == 0 ? 4 : 2; }

// carves a workspace; with a null base it only counts
struct TgCarve {
    char* base;
    size_t used;
    template <class T> T* take(size_t count)
    {
        used = (used + 255) & ~(size_t)255;
        T* p = base ? reinterpret_cast<T*>(base + used) : nullptr;
        used += count * sizeof(T);
        return p;
    }
};

// ---- tg_lookup.hip
void tg_launch_lookup(const void* table, int64_t ld, int dtype, int64_t n_rows, int d, const void* ids, int ids64, int64_t n, float scale,
                      void* out, hipStream_t s);
size_t tg_lookup_grad_space(int64_t n, int64_t n_rows, int d);
void tg_launch_lookup_grad(const void* grad, int64_t ld, int dtype, const void* ids, int ids64, int64_t n, int64_t n_rows, int d, float scale,
                           int accumulate, void* out, int out_dtype, void* space, hipStream_t s);
// zeros into a whole number of 16-bit values
void tg_launch_zero(void* p, size_t bytes, hipStream_t s);

// ---- tg_norm.hip
void tg_launch_norm(const void* x, int64_t ld_x, const void* res, int64_t ld_res, const void* w, int dtype, int64_t n, int d, float eps,
                    void* y, void* r, float* rstd, hipStream_t s);
size_t tg_norm_grad_space(int64_t n, int d);
void tg_launch_norm_grad(const void* dy, int64_t ld_dy, const void* dr, int64_t ld_dr, const void* r, int64_t ld_r, const void* w,
                         const float* rstd, int dtype, int64_t n, int d, void* dx, void* dw, void* space, hipStream_t s);
// w null: no norm
void tg_launch_norm_q8(const void* x, int64_t ld_x, const void* res, int64_t ld_res, const void* w, int dtype, int64_t n, int d, float eps,
                       int8_t* q, float* scale, void* r, hipStream_t s);
void tg_launch_dequantize(const int8_t* q, const float* scale, int64_t n, int d, int dtype, void* out, hipStream_t s);

// ---- tg_product.hip
size_t tg_product_space(int64_t m, int64_t n, int k, bool ready);
void tg_launch_product(const int8_t* a, const float* as, const int8_t* b, const float* bs, const float* bias, int64_t m, int64_t n, int k,
                       void* out, int dtype, void* space, hipStream_t s);

// ---- tg_xent.hip
// aligned: 0, or 1 where the rows of h and w can be read where they are but for their length, 2: those of w, 3: those of h
size_t tg_xent_space(int64_t n, int64_t n_rows, int d, int dtype, int aligned);
void tg_launch_xent(const void* h, int64_t ld_h, const void* w, int64_t ld_w, int dtype, int64_t n, int64_t n_rows, int d, const void* targets,
                    int targets64, float scale, float* loss, float* lse, void* space, hipStream_t s);
size_t tg_xent_grad_space(int64_t n, int64_t n_rows, int d, int dtype, int aligned, bool least);
void tg_launch_xent_grad(const void* h, int64_t ld_h, const void* w, int64_t ld_w, int dtype, int64_t n, int64_t n_rows, int d,
                         const void* targets, int targets64, const float* lse, const float* dloss, float scale, void* dh, void* dw,
                         void* space, size_t bytes, hipStream_t s);
