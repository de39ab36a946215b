// 8-bit operands: e4m3 values with one power of two for a block of 128, made from rows or from weight
// matrices (moe_quantise_rows_fp8, moe_quantise_weights_fp8, moe_dispatch_fp8).
//
// The scale is a power of two because that is what the matrix instructions apply by themselves
// (v_mfma_scale_f32_32x32x64_f8f6f4 takes an exponent byte for 32 reduction entries of each operand's row), so a
// product of blocks needs no instruction besides.
#include "fp8.h"

// Four fp32 -> four e4m3 bytes, rounded to nearest even.  |v| <= 448 or not finite; infinities become NaN as NaN does.
__device__ __forceinline__ uint32_t pack_e4m3x4(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// ---------------------------------------------------------------------------
// rows: 16 lanes share a block of 128, 8 entries each
// ---------------------------------------------------------------------------
template <typename T> __device__ __forceinline__ void load8(const T* p, float (&v)[8]);
template <> __device__ __forceinline__ void load8<bf16_t>(const bf16_t* p, float (&v)[8]) { Chunk<bf16_t>::load(p, v); }
template <> __device__ __forceinline__ void load8<float>(const float* p, float (&v)[8]) {
    float a[4], b[4];
    Chunk<float>::load(p, a);
    Chunk<float>::load(p + 4, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
}

// The largest magnitude as bits: their order as integers is that of the values, infinities and NaN above all
__device__ __forceinline__ uint32_t top_bits(const float (&v)[8]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
    return m;
}

// TOKENS: row r of x goes to the rows row_of[r*k + j] of q (dispatch); else to row r
template <typename T, bool TOKENS>
__global__ __launch_bounds__(256) void quantise_rows_kernel(int rows, int K, int nkb, int kb_stride, int k, int R,
                                                            const T* __restrict__ x, const int32_t* __restrict__ row_of,
                                                            uint8_t* __restrict__ q, uint8_t* __restrict__ b) {
    const int l16 = threadIdx.x & 15;
    const long long blocks = (long long)rows * nkb;
    for (long long at = (long long)blockIdx.x * 16 + (threadIdx.x >> 4); at < blocks; at += (long long)gridDim.x * 16) {
        const int r = (int)(at / nkb), kb = (int)(at - (long long)r * nkb), k0 = kb * 128 + l16 * 8;
        float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (k0 < K) load8(x + (size_t)r * K + k0, v);
        uint32_t m = top_bits(v);
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, MOE_WAVE));
        const int byte = scale_byte(m);
        const float f = scale_inverse(byte);
        uint2 w;
        w.x = pack_e4m3x4(v[0] * f, v[1] * f, v[2] * f, v[3] * f);
        w.y = pack_e4m3x4(v[4] * f, v[5] * f, v[6] * f, v[7] * f);
        for (int j = 0; j < (TOKENS ? k : 1); ++j) {
            int to = r;
            if (TOKENS) {
                to = row_of[(size_t)r * k + j];
                if ((unsigned)to >= (unsigned)R) continue;
            }
            *reinterpret_cast<uint2*>(q + ((size_t)to * nkb + kb) * 128 + l16 * 8) = w;
            uint8_t* bt = b + (size_t)to * kb_stride;
            if (l16 == 0) bt[kb] = (uint8_t)byte;
            if (kb == nkb - 1 && l16 > 0 && kb + l16 < kb_stride) bt[kb + l16] = 127;
        }
    }
}

template <bool TOKENS>
static void launch_rows(int rows, int K, int dtype, int k, int R, const void* x, const int32_t* row_of, void* q, uint8_t* b,
                        hipStream_t st) {
    const int nkb = fp8_blocks(K), stride = fp8_scale_stride(K);
    const long long blocks = ((long long)rows * nkb + 15) / 16;
    const int grid = (int)(blocks < 16384 ? blocks : 16384);
    if (dtype == MOE_BF16)
        quantise_rows_kernel<bf16_t, TOKENS><<<grid, 256, 0, st>>>(rows, K, nkb, stride, k, R, (const bf16_t*)x, row_of, (uint8_t*)q, b);
    else
        quantise_rows_kernel<float, TOKENS><<<grid, 256, 0, st>>>(rows, K, nkb, stride, k, R, (const float*)x, row_of, (uint8_t*)q, b);
}

extern "C" int moe_quantise_rows_fp8(int32_t rows, int32_t K, int32_t dtype, const void* x, void* q, uint8_t* b, void* stream) {
    int rc = begin_call(fp8_extent_status(rows, 1, K, 128, dtype));
    if (rc) return rc;
    if (!x || !q || !b) return MOE_ERR_NULL;
    if (!aligned(16, x, q) || !aligned(4, b)) return MOE_ERR_SHAPE;
    launch_rows<false>(rows, K, dtype, 1, rows, x, nullptr, q, b, (hipStream_t)stream);
    return launch_status();
}

int dispatch_fp8_check(const moe_fp8_shape* s, const void* x, const int32_t* row_of, const void* xq, const uint8_t* xb) {
    const int rc = fp8_shape_status(s);
    if (rc) return rc;
    return !(x && row_of && xq && xb) ? MOE_ERR_NULL : aligned(16, x, xq) && aligned(4, xb) ? MOE_OK : MOE_ERR_SHAPE;
}

extern "C" int moe_dispatch_fp8(const moe_fp8_shape* shape, const void* x, const int32_t* row_of, void* xq, uint8_t* xb,
                                void* stream) {
    const int rc = begin_call(dispatch_fp8_check(shape, x, row_of, xq, xb));
    if (rc) return rc;
    launch_rows<true>(shape->T, shape->d_model, shape->dtype, shape->k, shape->T * shape->k, x, row_of, xq, xb, (hipStream_t)stream);
    return launch_status();
}

// ---------------------------------------------------------------------------
// weights: a workgroup per block of 128 x 128, transposed through LDS
// ---------------------------------------------------------------------------
// Thread (a, c) of 32 x 8 holds the four reduction entries 4a .. 4a+3 of the columns 4 (c + 8 j) .. +3, j < 4, so that
// four bytes that are neighbours in the output are in one thread.
template <typename T>
__global__ __launch_bounds__(256) void quantise_weights_kernel(int K, int N, int nkb, int nnb, int kb_stride,
                                                               const T* __restrict__ W, uint8_t* __restrict__ q,
                                                               uint8_t* __restrict__ b) {
    constexpr int PAD = 132;                    // bytes per output row in LDS: 33 words, so that columns hit different banks
    __shared__ __align__(16) uint8_t s_q[128 * PAD];
    __shared__ uint32_t s_top[4];
    const int kb = blockIdx.x, nb = blockIdx.y, e = blockIdx.z;
    const int c = threadIdx.x & 7, a = threadIdx.x >> 3;
    const T* w = W + (size_t)e * K * N;
    float v[4][4][4];                           // [j][k][n]
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int n = nb * 128 + 4 * (c + 8 * j);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int k = kb * 128 + 4 * a + i;
#pragma unroll
            for (int u = 0; u < 4; ++u) v[j][i][u] = 0.0f;
            if (k < K && n < N) {
                typename Vec4io<T>::raw raw = *reinterpret_cast<const typename Vec4io<T>::raw*>(w + (size_t)k * N + n);
                Vec4io<T>::unpack(raw, v[j][i]);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) m = max(m, __float_as_uint(v[j][i][u]) & 0x7fffffffu);
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, MOE_WAVE));
    if ((threadIdx.x & 63) == 0) s_top[threadIdx.x >> 6] = m;
    __syncthreads();
    m = max(max(s_top[0], s_top[1]), max(s_top[2], s_top[3]));
    const int byte = scale_byte(m);
    const float f = scale_inverse(byte);
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int u = 0; u < 4; ++u)
            *reinterpret_cast<uint32_t*>(s_q + (4 * (c + 8 * j) + u) * PAD + 4 * a) =
                pack_e4m3x4(v[j][0][u] * f, v[j][1][u] * f, v[j][2][u] * f, v[j][3][u] * f);
    __syncthreads();
    uint8_t* out = q + ((size_t)e * nnb + nb) * 128 * nkb * 128 + (size_t)kb * 128;
    for (int i = threadIdx.x; i < 128 * 8; i += 256) {
        const int n = i >> 3, u = i & 7;
        const uint32_t* p = reinterpret_cast<const uint32_t*>(s_q + n * PAD + 16 * u);
        *reinterpret_cast<uint4*>(out + (size_t)n * nkb * 128 + 16 * u) = make_uint4(p[0], p[1], p[2], p[3]);
    }
    uint8_t* bt = b + ((size_t)e * nnb + nb) * kb_stride;
    if (threadIdx.x == 0) bt[kb] = (uint8_t)byte;
    if (kb == nkb - 1 && threadIdx.x > 0 && kb + (int)threadIdx.x < kb_stride) bt[kb + threadIdx.x] = 127;
}

extern "C" int moe_quantise_weights_fp8(int32_t E, int32_t K, int32_t N, int32_t dtype, const void* W, void* q, uint8_t* b,
                                        void* stream) {
    int rc = begin_call(fp8_extent_status(1, E, K, N, dtype));
    if (rc) return rc;
    if (!W || !q || !b) return MOE_ERR_NULL;
    if (!aligned(16, W, q) || !aligned(4, b)) return MOE_ERR_SHAPE;
    const int nkb = fp8_blocks(K), nnb = fp8_blocks(N);
    const dim3 grid(nkb, nnb, E);
    hipStream_t st = (hipStream_t)stream;
    if (dtype == MOE_BF16)
        quantise_weights_kernel<bf16_t><<<grid, 256, 0, st>>>(K, N, nkb, nnb, fp8_scale_stride(K), (const bf16_t*)W, (uint8_t*)q, b);
    else
        quantise_weights_kernel<float><<<grid, 256, 0, st>>>(K, N, nkb, nnb, fp8_scale_stride(K), (const float*)W, (uint8_t*)q, b);
    return launch_status();
}
