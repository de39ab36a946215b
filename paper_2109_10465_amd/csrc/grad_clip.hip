// moe_grad_norm / moe_clip_grads: the global norm of many gradients, and clipping to it.
//
// The list of tensors travels in the kernels' arguments, a table of them per launch.  Each workgroup of a launch takes a
// fixed part of one tensor and leaves the sum of its squares, in 64 bits, in the workspace; one workgroup adds those
// in a fixed order.  Squares are summed in 64 bits because gradients may be anything that fp32 holds: the square of 2e19 is
// beyond fp32, that of 1e-23 below it.
#include <math.h>
#include "moe_common.h"

#define GRAD_TABLE 96           // tensors per launch: 28 bytes each, inside 4 KB of arguments
#define GRAD_PART 16384         // elements per workgroup

struct GradTable {
    const void* in[GRAD_TABLE];
    void* out[GRAD_TABLE];
    int64_t n[GRAD_TABLE];
    int32_t first[GRAD_TABLE + 1];      // workgroups of the tensors before
    uint32_t bf16[GRAD_TABLE / 32];     // a bit per tensor
    int count;
};

__device__ __forceinline__ int grad_tensor(const GradTable& t, int wg) {
    int lo = 0, hi = t.count;           // first[lo] <= wg < first[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (t.first[mid] <= wg) lo = mid; else hi = mid;
    }
    return lo;
}

// f(value, index) for this thread's elements of [a, b) of p: single elements up to a 16-byte boundary, vectors, the rest
template <typename T, typename F1, typename FN>
__device__ __forceinline__ void each_element(const T* p, int64_t a, int64_t b, F1 one, FN many) {
    constexpr int CN = Chunk<T>::N;
    const int64_t lead = ((16 - ((uintptr_t)(p + a) & 15)) & 15) / sizeof(T);
    const int64_t v0 = a + lead < b ? a + lead : b, nv = (b - v0) / CN;
    for (int64_t i = a + threadIdx.x; i < v0; i += 256) one(i);
    for (int64_t i = threadIdx.x; i < nv; i += 256) many(v0 + i * CN);
    for (int64_t i = v0 + nv * CN + threadIdx.x; i < b; i += 256) one(i);
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
    each_element<T>(p, a, b,
        [&](int64_t i) { const double v = ld_f32(p + i); s = fma(v, v, s); },
        [&](int64_t i) {
            float v[Chunk<T>::N];
            Chunk<T>::load(p + i, v);
#pragma unroll
            for (int j = 0; j < Chunk<T>::N; ++j) s = fma((double)v[j], (double)v[j], s);
        });
    return s;
}

__global__ __launch_bounds__(256) void grad_squares_kernel(const GradTable t, double* __restrict__ part) {
    const int x = grad_tensor(t, blockIdx.x);
    const int64_t a = (int64_t)(blockIdx.x - t.first[x]) * GRAD_PART, b = min(a + GRAD_PART, t.n[x]);
    const bool half = t.bf16[x >> 5] >> (x & 31) & 1u;
    const double s = block_sum(half ? part_squares((const bf16_t*)t.in[x], a, b) : part_squares((const float*)t.in[x], a, b));
    if (threadIdx.x == 0) part[blockIdx.x] = s;
}

__global__ __launch_bounds__(256) void grad_norm_kernel(int n, const double* __restrict__ part, float* __restrict__ norm) {
    double s = 0.0;
    for (int i = threadIdx.x; i < n; i += 256) s += part[i];
    s = block_sum(s);
    if (threadIdx.x == 0) norm[0] = (float)sqrt(s);
}

template <typename T>
__device__ __forceinline__ void scale_part(const T* p, T* o, int64_t a, int64_t b, float f) {
    if (((uintptr_t)p & 15) == ((uintptr_t)o & 15)) {
        each_element<T>(p, a, b,
            [&](int64_t i) { st_f32(o + i, ld_f32(p + i) * f); },
            [&](int64_t i) {
                float v[Chunk<T>::N];
                Chunk<T>::load(p + i, v);
#pragma unroll
                for (int j = 0; j < Chunk<T>::N; ++j) v[j] *= f;
                Chunk<T>::store(o + i, v);
            });
    } else {
        for (int64_t i = a + threadIdx.x; i < b; i += 256) st_f32(o + i, ld_f32(p + i) * f);
    }
}

__global__ __launch_bounds__(256) void grad_scale_kernel(const GradTable t, float max_norm, const float* __restrict__ norm) {
    const float n = norm[0];
    const bool clip = n > max_norm && n < INFINITY;
    const float f = clip ? max_norm / n : 1.0f;
    const int x = grad_tensor(t, blockIdx.x);
    if (!clip && t.in[x] == t.out[x]) return;
    const int64_t a = (int64_t)(blockIdx.x - t.first[x]) * GRAD_PART, b = min(a + GRAD_PART, t.n[x]);
    if (t.bf16[x >> 5] >> (x & 31) & 1u) scale_part((const bf16_t*)t.in[x], (bf16_t*)t.out[x], a, b, f);
    else scale_part((const float*)t.in[x], (float*)t.out[x], a, b, f);
}

// Calls f(table, workgroups) for every launch's table
template <typename F>
static void each_table(const moe_grad* g, int count, F f) {
    GradTable t;
    int64_t wgs = 0;
    auto flush = [&]() {
        if (t.count) f(t, (int)wgs);
        t.count = 0;
        wgs = 0;
        for (uint32_t& w : t.bf16) w = 0;
    };
    t.count = 0;
    flush();
    for (int i = 0; i < count; ++i) {
        if (g[i].n == 0) continue;
        const int64_t need = (g[i].n + GRAD_PART - 1) / GRAD_PART;
        if (t.count == GRAD_TABLE || wgs + need >= (1ll << 31)) flush();
        t.in[t.count] = g[i].grad;
        t.out[t.count] = g[i].out;
        t.n[t.count] = g[i].n;
        t.first[t.count] = (int32_t)wgs;
        if (g[i].dtype == MOE_BF16) t.bf16[t.count >> 5] |= 1u << (t.count & 31);
        wgs += need;
        t.first[++t.count] = (int32_t)wgs;
    }
    flush();
}

static int64_t grad_parts(const moe_grad* g, int count) {
    int64_t n = 0;
    for (int i = 0; i < count; ++i) n += (g[i].n + GRAD_PART - 1) / GRAD_PART;
    return n;
}

static int grad_status(const moe_grad* g, int count, bool clip) {
    if (!g && count > 0) return MOE_ERR_NULL;
    if (count < 0) return MOE_ERR_SHAPE;
    int64_t total = 0;
    for (int i = 0; i < count; ++i) {
        if (g[i].dtype != MOE_F32 && g[i].dtype != MOE_BF16) return MOE_ERR_DTYPE;
        if (g[i].n < 0 || g[i].n > (1ll << 44)) return MOE_ERR_SHAPE;
        if (g[i].n && (!g[i].grad || (clip && !g[i].out))) return MOE_ERR_NULL;
        const uintptr_t align = elem_bytes(g[i].dtype) - 1;
        if (g[i].n && (((uintptr_t)g[i].grad & align) || (clip && ((uintptr_t)g[i].out & align)))) return MOE_ERR_SHAPE;
        total += g[i].n / GRAD_PART + 1;
    }
    return total < (1ll << 31) ? MOE_OK : MOE_ERR_SHAPE;
}

static size_t grad_ws_bytes(const moe_grad* g, int count) {
    const int64_t n = grad_parts(g, count);
    return align_up((size_t)(n ? n : 1) * 8, 256);
}

extern "C" size_t moe_grad_workspace_bytes(const moe_grad* grads, int32_t count) {
    return grad_status(grads, count, false) == MOE_OK ? grad_ws_bytes(grads, count) : 0;
}

static int norm_impl(const moe_grad* grads, int count, float* norm, void* ws, hipStream_t st) {
    double* part = (double*)ws;
    int64_t done = 0;
    each_table(grads, count, [&](const GradTable& t, int wgs) {
        grad_squares_kernel<<<wgs, 256, 0, st>>>(t, part + done);
        done += wgs;
    });
    grad_norm_kernel<<<1, 256, 0, st>>>((int)done, part, norm);
    return launch_status();
}

extern "C" int moe_grad_norm(const moe_grad* grads, int32_t count, float* norm, void* ws, size_t ws_bytes, void* stream) {
    const int rc = begin_call(grad_status(grads, count, false));
    if (rc) return rc;
    if (!norm) return MOE_ERR_NULL;
    if (!ws_ok(ws, ws_bytes, grad_ws_bytes(grads, count))) return MOE_ERR_WORKSPACE;
    return norm_impl(grads, count, norm, ws, (hipStream_t)stream);
}

extern "C" int moe_clip_grads(const moe_grad* grads, int32_t count, float max_norm, float* norm, void* ws, size_t ws_bytes,
                              void* stream) {
    int rc = begin_call(grad_status(grads, count, true));
    if (rc) return rc;
    if (!norm) return MOE_ERR_NULL;
    if (!(max_norm >= 0.0f) || !isfinite(max_norm)) return MOE_ERR_SHAPE;
    if (!ws_ok(ws, ws_bytes, grad_ws_bytes(grads, count))) return MOE_ERR_WORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    rc = norm_impl(grads, count, norm, ws, st);
    if (rc) return rc;
    each_table(grads, count, [&](const GradTable& t, int wgs) { grad_scale_kernel<<<wgs, 256, 0, st>>>(t, max_norm, norm); });
    return launch_status();
}
