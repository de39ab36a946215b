// moe_grad_norm / moe_clip_grads: the global norm of many gradients, and clipping to it.
//
// The list of tensors travels in the kernels' arguments, a table of them per launch.  A launch's tensors are cut into parts,
// which its workgroups take in turn; each leaves one sum of squares, in 64 bits, in the workspace.  Up to 2048 of them
// are added by every workgroup of the clipping launch itself, in one order: that is 16 KB of the L2 and saves a launch (157
// tensors of 2.2 M elements together 15.5 us, 17.8 with it).  More of them, from a second table on, are added once: each launch would read them
// for every part (300 tensors of 2^20 floats in place, not clipped, 248 us, 263 otherwise; 1200 tensors 976, 1436).  Squares are
// summed in 64 bits because gradients may be anything that fp32 holds: the square of 2e19 is beyond fp32, that of 1e-23
// below it.  Bound: HBM; everything is read twice and written once.  270 M floats and 130 M bfloat16: squares 276 us (4.9
// TB/s; 256 after a pause), clipping 497 (5.4).  The clipping pass has a workgroup for nearly every part: with 2048 that take parts in turn it is
// 590 us; going backwards, from what the first pass read last, gains nothing.
#include <math.h>
#include "moe_common.h"

#define GRAD_TABLE 160          // tensors per launch: 24 bytes each, inside 4 KB of arguments
#define GRAD_WGS 2048           // workgroups, and so sums, of a squares launch, at most: eight per CU
#define GRAD_CLIP_WGS 65536     // of a clipping launch
#define GRAD_SUMS 2048          // that each of a clipping launch's workgroups adds up itself, at most

struct GradTable {
    const void* in[GRAD_TABLE];
    void* out[GRAD_TABLE];
    int32_t first[GRAD_TABLE + 1];      // parts of the tensors before
    int32_t tail[GRAD_TABLE];           // elements of a tensor's last part
    uint32_t bf16[GRAD_TABLE / 32];     // a bit per tensor
    int32_t count, part;                // tensors; elements per part
};
static_assert(sizeof(GradTable) <= 4000, "kernel arguments");

struct GradPart {
    int tensor;
    int64_t begin, end;                 // elements of the tensor
    bool bf16;
};
__device__ __forceinline__ GradPart grad_part(const GradTable& t, int part) {
    int lo = 0, hi = t.count;           // first[lo] <= part < first[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (t.first[mid] <= part) lo = mid; else hi = mid;
    }
    const int64_t a = (int64_t)(part - t.first[lo]) * t.part;
    return {lo, a, a + (part + 1 == t.first[lo + 1] ? t.tail[lo] : t.part), (t.bf16[lo >> 5] >> (lo & 31) & 1u) != 0};
}

// This thread's elements of [a, b) of p: single ones up to a 16-byte boundary, vectors, the rest; four vectors are asked for
// before the first is used
template <typename T, typename F1, typename FN>
__device__ __forceinline__ void each_element(const T* __restrict__ p, int64_t a, int64_t b, F1 one, FN many) {
    constexpr int CN = Chunk<T>::N, U = 4;
    const int64_t lead = ((16 - ((uintptr_t)(p + a) & 15)) & 15) / sizeof(T);
    const int64_t v0 = a + lead < b ? a + lead : b;
    const int nv = (int)((b - v0) / CN);
    const int64_t end = v0 + (int64_t)nv * CN;
    if (a + threadIdx.x < v0) one(a + threadIdx.x, ld_f32(p + a + threadIdx.x));
    if (end + threadIdx.x < b) one(end + threadIdx.x, ld_f32(p + end + threadIdx.x));
    int i = threadIdx.x;
    for (; i + (U - 1) * 256 < nv; i += U * 256) {
        float v[U][CN];
#pragma unroll
        for (int u = 0; u < U; ++u) Chunk<T>::load(p + v0 + (int64_t)(i + u * 256) * CN, v[u]);
#pragma unroll
        for (int u = 0; u < U; ++u) many(v0 + (int64_t)(i + u * 256) * CN, v[u]);
    }
    for (; i < nv; i += 256) {
        float v[CN];
        Chunk<T>::load(p + v0 + (int64_t)i * CN, v);
        many(v0 + (int64_t)i * CN, v);
    }
}

__device__ __forceinline__ double block_sum(double s) {
    __shared__ double s_part[4];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, MOE_WAVE);
    if ((threadIdx.x & 63) == 0) s_part[threadIdx.x >> 6] = s;
    __syncthreads();
    return (s_part[0] + s_part[1]) + (s_part[2] + s_part[3]);
}

template <typename T>
__device__ __forceinline__ double part_squares(const T* p, int64_t a, int64_t b) {
    double s = 0.0;
    each_element<T>(p, a, b, [&](int64_t, float x) { s = fma((double)x, (double)x, s); },
                    [&](int64_t, const float (&v)[Chunk<T>::N]) {
#pragma unroll
                        for (int j = 0; j < Chunk<T>::N; ++j) s = fma((double)v[j], (double)v[j], s);
                    });
    return s;
}

__global__ __launch_bounds__(256) void grad_squares_kernel(const GradTable t, double* __restrict__ sums) {
    double s = 0.0;
    for (int i = blockIdx.x; i < t.first[t.count]; i += gridDim.x) {
        const GradPart g = grad_part(t, i);
        s += g.bf16 ? part_squares((const bf16_t*)t.in[g.tensor], g.begin, g.end) : part_squares((const float*)t.in[g.tensor], g.begin, g.end);
    }
    s = block_sum(s);
    if (threadIdx.x == 0) sums[blockIdx.x] = s;
}

// the norm, in every thread of the workgroup
__device__ __forceinline__ double norm_of(int n, const double* sums) {
    double s = 0.0;
#pragma unroll 8
    for (int i = threadIdx.x; i < n; i += 256) s += sums[i];
    return sqrt(block_sum(s));
}

// ... which also takes the first sum's place (every thread has read them)
__global__ __launch_bounds__(256) void grad_norm_kernel(int n, double* sums, float* __restrict__ norm) {
    const double v = norm_of(n, sums);
    if (threadIdx.x == 0) {
        norm[0] = (float)v;
        sums[0] = v;
    }
}

// The factor max_norm / norm as f 2^e: e is 0 but where the quotient is so small that fp32 would hold it with fewer bits, or as 0,
// though its products with large gradients are not
struct GradFactor {
    float f;
    int e;
};

template <typename T>
__device__ __forceinline__ void scale_part(const T* p, T* o, int64_t a, int64_t b, GradFactor by) {
    auto scaled = [by](float x) { return ldexpf(x * by.f, by.e); };
    if (((uintptr_t)p & 15) == ((uintptr_t)o & 15)) {
        each_element<T>(p, a, b, [&](int64_t i, float x) { st_f32(o + i, scaled(x)); },
                        [&](int64_t i, const float (&v)[Chunk<T>::N]) {
                            float w[Chunk<T>::N];
#pragma unroll
                            for (int j = 0; j < Chunk<T>::N; ++j) w[j] = scaled(v[j]);
                            Chunk<T>::store(o + i, w);
                        });
    } else {        // the output lies differently against 16 bytes
        for (int64_t i = a + threadIdx.x; i < b; i += 256) st_f32(o + i, scaled(ld_f32(p + i)));
    }
}

__global__ __launch_bounds__(256) void grad_scale_kernel(const GradTable t, float max_norm, int n, const double* __restrict__ sums,
                                                         float* __restrict__ norm) {
    const double wide = n ? norm_of(n, sums) : sums[0];
    const float v = (float)wide;
    if (n && blockIdx.x == 0 && threadIdx.x == 0) norm[0] = v;  // (every launch writes the same)
    const bool clip = v > max_norm && v < INFINITY;
    GradFactor by = {1.0f, 0};
    if (clip) {
        double q = max_norm / wide;
        if (q < 0x1p-100) q = frexp(q, &by.e);
        by.f = (float)q;
    }
    for (int i = blockIdx.x; i < t.first[t.count]; i += gridDim.x) {
        const GradPart g = grad_part(t, i);
        const void* in = t.in[g.tensor];
        void* out = t.out[g.tensor];
        if (!clip && in == out) continue;
        if (g.bf16) scale_part((const bf16_t*)in, (bf16_t*)out, g.begin, g.end, by);
        else scale_part((const float*)in, (float*)out, g.begin, g.end, by);
    }
}

// Elements per part: 16384, fewer where that would leave workgroups without work
static int grad_part_size(const moe_grad* g, int count) {
    int64_t n = 0;
    for (int i = 0; i < count; ++i) n += g[i].n;
    int part = 16384;
    while (part > 2048 && n / part < GRAD_WGS) part >>= 1;
    return part;
}

// Calls f(table, workgroups) for every launch's table; at most so many workgroups
template <typename F>
static void each_table(const moe_grad* g, int count, int most, F f) {
    GradTable t;
    t.part = grad_part_size(g, count);
    auto flush = [&]() {
        if (t.count) f(t, t.first[t.count] < most ? t.first[t.count] : most);
        t.count = 0;
        t.first[0] = 0;
        for (uint32_t& w : t.bf16) w = 0;
    };
    t.count = 0;
    flush();
    for (int i = 0; i < count; ++i) {
        if (g[i].n == 0) continue;
        const int64_t parts = (g[i].n + t.part - 1) / t.part;
        if (t.count == GRAD_TABLE || t.first[t.count] + parts > (1 << 30)) flush();
        t.in[t.count] = g[i].grad;
        t.out[t.count] = g[i].out;
        t.tail[t.count] = (int32_t)(g[i].n - (parts - 1) * t.part);
        if (g[i].dtype == MOE_BF16) t.bf16[t.count >> 5] |= 1u << (t.count & 31);
        t.first[t.count + 1] = t.first[t.count] + (int32_t)parts;
        ++t.count;
    }
    flush();
}

static int grad_status(const moe_grad* g, int count, bool clip) {
    if (!g && count > 0) return MOE_ERR_NULL;
    if (count < 0) return MOE_ERR_SHAPE;
    for (int i = 0; i < count; ++i) {
        if (g[i].dtype != MOE_F32 && g[i].dtype != MOE_BF16) return MOE_ERR_DTYPE;
        if (g[i].n < 0 || g[i].n > (1ll << 43)) return MOE_ERR_SHAPE;
        if (g[i].n && (!g[i].grad || (clip && !g[i].out))) return MOE_ERR_NULL;
        const uintptr_t align = elem_bytes(g[i].dtype) - 1;
        if (g[i].n && (((uintptr_t)g[i].grad & align) || (clip && ((uintptr_t)g[i].out & align)))) return MOE_ERR_SHAPE;
    }
    return MOE_OK;
}

static int grad_sums(const moe_grad* g, int count) {
    int n = 0;
    each_table(g, count, GRAD_WGS, [&](const GradTable&, int wgs) { n += wgs; });
    return n;
}
static size_t grad_ws_bytes(const moe_grad* g, int count) {
    const int n = grad_sums(g, count);
    return align_up((size_t)(n ? n : 1) * 8, 256);
}

extern "C" size_t moe_grad_workspace_bytes(const moe_grad* grads, int32_t count) {
    return grad_status(grads, count, false) == MOE_OK ? grad_ws_bytes(grads, count) : 0;
}

// the sums of squares of every launch's workgroups; returns their number
static int squares_impl(const moe_grad* grads, int count, double* sums, hipStream_t st) {
    int done = 0;
    each_table(grads, count, GRAD_WGS, [&](const GradTable& t, int wgs) {
        grad_squares_kernel<<<wgs, 256, 0, st>>>(t, sums + done);
        done += wgs;
    });
    return done;
}

extern "C" int moe_grad_norm(const moe_grad* grads, int32_t count, float* norm, void* ws, size_t ws_bytes, void* stream) {
    const int rc = begin_call(grad_status(grads, count, false));
    if (rc) return rc;
    if (!norm) return MOE_ERR_NULL;
    if (!ws_ok(ws, ws_bytes, grad_ws_bytes(grads, count))) return MOE_ERR_WORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    const int n = squares_impl(grads, count, (double*)ws, st);
    grad_norm_kernel<<<1, 256, 0, st>>>(n, (double*)ws, norm);
    return launch_status();
}

extern "C" int moe_clip_grads(const moe_grad* grads, int32_t count, float max_norm, float* norm, void* ws, size_t ws_bytes,
                              void* stream) {
    const int rc = begin_call(grad_status(grads, count, true));
    if (rc) return rc;
    if (!norm) return MOE_ERR_NULL;
    if (!(max_norm >= 0.0f) || !isfinite(max_norm)) return MOE_ERR_SHAPE;
    if (!ws_ok(ws, ws_bytes, grad_ws_bytes(grads, count))) return MOE_ERR_WORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    const int n = squares_impl(grads, count, (double*)ws, st);
    const bool apart = n == 0 || n > GRAD_SUMS;
    if (apart) grad_norm_kernel<<<1, 256, 0, st>>>(n, (double*)ws, norm);
    each_table(grads, count, GRAD_CLIP_WGS, [&](const GradTable& t, int wgs) {
        grad_scale_kernel<<<wgs, 256, 0, st>>>(t, max_norm, apart ? 0 : n, (const double*)ws, norm);
    });
    return launch_status();
}
