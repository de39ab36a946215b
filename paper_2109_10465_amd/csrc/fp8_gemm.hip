// moe_expert_product_fp8 / moe_expert_ffn_fwd_fp8: the experts' products on 8-bit operands.
//
//   y[r, n] = sum over blocks b of 128 reduction entries of 2^(xe[r,b] + we[n/128,b]) sum_{k in b} xq[r,k] wq[n,k]
//
// computed as the transposed tile (weights are the instruction's first operand): a lane then holds, of one row, four
// consecutive columns out of every eight, and a wave whole blocks of 128 columns, so that the hidden activation's
// largest magnitude, its exponent and its bytes are found without leaving the wave.
#include <type_traits>
#include "fp8.h"

typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

struct Fp8Args {
    const uint8_t *xq, *xb, *wq, *wb;
    const int32_t* start;
    void* y;            // the output, or the hidden activation's bytes
    uint8_t* yb;        // and its exponents
    int rows, E, N;     // N: columns that exist
    int nkb, nnb;       // blocks of 128 along the reduction and the columns
    int xb_stride, yb_stride;       // exponent bytes per row (xb_stride: also per block row of the weights)
};

enum { OUT_BF16 = 0, OUT_RELU8 = 1, OUT_GELU8 = 2 };

// one step of 64 reduction entries with the exponents of byte S of either word
template <int S> __device__ __forceinline__ f32x16_t mma(i32x8_t w, i32x8_t x, f32x16_t c, int we, int xe) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w, x, c, 0, 0, S, we, S, xe);
}
__device__ __forceinline__ i32x8_t two16(uint4 a, uint4 b) {
    return i32x8_t{(int)a.x, (int)a.y, (int)a.z, (int)a.w, (int)b.x, (int)b.y, (int)b.z, (int)b.w};
}

// gelu(z) = z Phi(z), as the fp32 experts have it: two fits of Phi that meet at |z| = 1.0625
__device__ __forceinline__ float gelu(float z) {
    constexpr float CENTRE[6] = {0.39894229f, -0.066490486f, 0.0099737411f, -0.0011868734f, 0.00011374246f, -7.6692668e-06f};
    constexpr float MILLS_NUM[4] = {1.2527357f, 1.0029950f, 0.36051896f, 0.061547495f};
    constexpr float MILLS_DEN[5] = {1.0f, 1.5959138f, 1.0661000f, 0.36044064f, 0.061549164f};
    constexpr float LH = -0.72134751f, PHI0 = 0.39894228f, PHI0_LN2 = 0.27652571f;
    const float t = fminf(fabsf(z), 16.0f), s = t * t, e = s * LH, rest = fmaf(s, LH, -e);
    const float pdf = __builtin_amdgcn_exp2f(e) * fmaf(rest, PHI0_LN2, PHI0);
    float c = CENTRE[5], num = MILLS_NUM[3], den = MILLS_DEN[4];
#pragma unroll
    for (int i = 4; i >= 0; --i) c = fmaf(c, s, CENTRE[i]);
#pragma unroll
    for (int i = 2; i >= 0; --i) num = fmaf(num, t, MILLS_NUM[i]);
#pragma unroll
    for (int i = 3; i >= 0; --i) den = fmaf(den, t, MILLS_DEN[i]);
    const float q = num * pdf * __builtin_amdgcn_rcpf(den);
    return z * (t < 1.0625f ? fmaf(z, c, 0.5f) : (z >= 0.0f ? 1.0f - q : q));
}

// lanes 0..31 end with a = (own a, partner's a), lanes 32..63 with (partner's b, own b)
__device__ __forceinline__ void swap_halves(uint32_t& a, uint32_t& b) {
    const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
    a = r[0];
    b = r[1];
}

// The wave's tile of 128 columns (block nb) and 32 rows: acc[f][4 q + i] is column 32 f + 8 q + 4 half + i of row r
template <int OUT>
__device__ __forceinline__ void store_tile(const Fp8Args& p, f32x16_t (&acc)[4], int nb, int r, bool live, int half) {
    if constexpr (OUT == OUT_RELU8 || OUT == OUT_GELU8) {
        uint32_t top = 0;
#pragma unroll
        for (int f = 0; f < 4; ++f)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float z = acc[f][i], h = OUT == OUT_GELU8 ? gelu(z) : (z > 0.0f || z != z ? z : 0.0f);
                acc[f][i] = h;
                top = max(top, __float_as_uint(h) & 0x7fffffffu);
            }
        top = max(top, (uint32_t)__shfl_xor((int)top, 32, MOE_WAVE));
        const int byte = scale_byte(top);
        const float g = scale_inverse(byte);
        uint8_t* row = (uint8_t*)p.y + ((size_t)r * p.nnb + nb) * 128;
#pragma unroll
        for (int f = 0; f < 4; ++f) {
            uint32_t d[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                int w = __builtin_amdgcn_cvt_pk_fp8_f32(acc[f][4 * q] * g, acc[f][4 * q + 1] * g, 0, false);
                d[q] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(acc[f][4 * q + 2] * g, acc[f][4 * q + 3] * g, w, true);
            }
            swap_halves(d[0], d[2]);
            swap_halves(d[1], d[3]);
            if (live) *reinterpret_cast<uint4*>(row + 32 * f + 16 * half) = make_uint4(d[0], d[2], d[1], d[3]);
        }
        if (live) {
            uint8_t* bt = p.yb + (size_t)r * p.yb_stride;
            if (half == 0) bt[nb] = (uint8_t)byte;
            else if (nb == p.nnb - 1)
                for (int i = p.nnb; i < p.yb_stride; ++i) bt[i] = 127;
        }
    } else {
        bf16_t* row = (bf16_t*)p.y + (size_t)r * p.N;
#pragma unroll
        for (int f = 0; f < 4; ++f) {
            uint32_t d[4][2];
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int i = 0; i < 2; ++i) d[q][i] = pack_bf16x2(acc[f][4 * q + 2 * i], acc[f][4 * q + 2 * i + 1]);
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                swap_halves(d[q][0], d[q + 2][0]);
                swap_halves(d[q][1], d[q + 2][1]);
                const int n = nb * 128 + 32 * f + 16 * half + 8 * q;
                if (live && n < p.N) *reinterpret_cast<uint4*>(row + n) = make_uint4(d[q][0], d[q][1], d[q + 2][0], d[q + 2][1]);
            }
        }
    }
}

// Which expert and rows the row tile `at` has, tiles of TR rows, expert by expert: found by a wave, four experts a lane
struct RowTile { int e, row, end; };     // e < 0: no such tile
template <int TR>
__device__ __forceinline__ RowTile find_tile(const int32_t* __restrict__ start, int E, int rows, int at, int lane) {
    int s[5], n = 0, t[4];
#pragma unroll
    for (int q = 0; q < 5; ++q) s[q] = min(max(start[min(4 * lane + q, E)], 0), rows);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        t[q] = 4 * lane + q < E ? (max(s[q + 1] - s[q], 0) + TR - 1) / TR : 0;
        n += t[q];
    }
    int run = n;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(run, o, MOE_WAVE);
        if (lane >= o) run += u;
    }
    run -= n;                       // tiles of the lanes before
    RowTile r = {-1, 0, 0};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if (at >= run && at < run + t[q]) r = {4 * lane + q, s[q] + (at - run) * TR, s[q + 1]};
        run += t[q];
    }
    const unsigned long long owner = __ballot(r.e >= 0);
    if (!owner) return {-1, 0, 0};
    const int src = __ffsll((long long)owner) - 1;
    return {__shfl(r.e, src, MOE_WAVE), __shfl(r.row, src, MOE_WAVE), __shfl(r.end, src, MOE_WAVE)};
}

// one wave: 128 columns and 32 rows, operands straight from memory
template <int OUT>
__global__ __launch_bounds__(64) void fp8_gemm_kernel(const Fp8Args p) {
    const int lane = threadIdx.x, l32 = lane & 31, half = lane >> 5, nb = blockIdx.x % p.nnb;
    const RowTile t = find_tile<32>(p.start, p.E, p.rows, blockIdx.x / p.nnb, lane);
    if (t.e < 0) return;
    const int r = t.row + l32;
    const bool live = r < t.end;
    const size_t kbytes = (size_t)p.nkb * 128;
    const uint8_t* x = p.xq + (size_t)(live ? r : t.row) * kbytes + 16 * half;
    const uint8_t* w = p.wq + ((size_t)t.e * p.nnb + nb) * 128 * kbytes + (size_t)l32 * kbytes + 16 * half;
    const int* xe = reinterpret_cast<const int*>(p.xb + (size_t)(live ? r : t.row) * p.xb_stride);
    const int* we = reinterpret_cast<const int*>(p.wb + ((size_t)t.e * p.nnb + nb) * p.xb_stride);
    f32x16_t acc[4];
#pragma unroll
    for (int f = 0; f < 4; ++f)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[f][i] = 0.0f;
    auto block = [&](int kb, auto byte, int we4, int xe4) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const size_t at = (size_t)kb * 128 + 64 * s;
            const i32x8_t b = two16(*reinterpret_cast<const uint4*>(x + at), *reinterpret_cast<const uint4*>(x + at + 32));
#pragma unroll
            for (int f = 0; f < 4; ++f) {
                const uint8_t* wf = w + (size_t)(32 * f) * kbytes + at;
                const i32x8_t a = two16(*reinterpret_cast<const uint4*>(wf), *reinterpret_cast<const uint4*>(wf + 32));
                acc[f] = mma<decltype(byte)::value>(a, b, acc[f], we4, xe4);
            }
        }
    };
    for (int kb = 0; kb < p.nkb; kb += 4) {
        const int we4 = we[kb >> 2], xe4 = xe[kb >> 2];
        block(kb, std::integral_constant<int, 0>(), we4, xe4);
        if (kb + 1 < p.nkb) block(kb + 1, std::integral_constant<int, 1>(), we4, xe4);
        if (kb + 2 < p.nkb) block(kb + 2, std::integral_constant<int, 2>(), we4, xe4);
        if (kb + 3 < p.nkb) block(kb + 3, std::integral_constant<int, 3>(), we4, xe4);
    }
    store_tile<OUT>(p, acc, nb, r, live, half);
}

template <int OUT>
static void launch_fp8(const Fp8Args& p, hipStream_t st) {
    const long long most = (long long)p.rows / 32 + (p.E < p.rows ? p.E : p.rows);     // row tiles, at most
    fp8_gemm_kernel<OUT><<<(unsigned)(most * p.nnb), 64, 0, st>>>(p);
}

static Fp8Args fp8_args(int rows, int E, int K, int N, const void* xq, const uint8_t* xb, const int32_t* start, const void* wq,
                        const uint8_t* wb, void* y, uint8_t* yb) {
    Fp8Args p;
    p.xq = (const uint8_t*)xq; p.xb = xb; p.wq = (const uint8_t*)wq; p.wb = wb;
    p.start = start; p.y = y; p.yb = yb;
    p.rows = rows; p.E = E; p.N = N;
    p.nkb = fp8_blocks(K); p.nnb = fp8_blocks(N);
    p.xb_stride = fp8_scale_stride(K); p.yb_stride = fp8_scale_stride(N);
    return p;
}

extern "C" int moe_expert_product_fp8(int32_t rows, int32_t E, int32_t K, int32_t N, const void* xq, const uint8_t* xb,
                                      const int32_t* expert_start, const void* Wq, const uint8_t* Wb, void* y,
                                      void* stream) {
    const int rc = begin_call(fp8_extent_status(rows, E, K, N, MOE_BF16));
    if (rc) return rc;
    if (!xq || !xb || !expert_start || !Wq || !Wb || !y) return MOE_ERR_NULL;
    launch_fp8<OUT_BF16>(fp8_args(rows, E, K, N, xq, xb, expert_start, Wq, Wb, y, nullptr), (hipStream_t)stream);
    return launch_status();
}

int fp8_shape_status(const moe_fp8_shape* s) {
    if (!s) return MOE_ERR_NULL;
    if (s->dtype != MOE_BF16 || (s->act != MOE_RELU && s->act != MOE_GELU)) return MOE_ERR_DTYPE;
    if (s->T < 1 || s->k < 1 || s->k > 8 || (int64_t)s->T * s->k >= (1 << 30)) return MOE_ERR_SHAPE;
    return fp8_extent_status(s->T * s->k, s->E, s->d_model, s->d_ff, s->dtype);
}

int ffn_fp8_check(const moe_fp8_shape* s, const void* xq, const uint8_t* xb, const int32_t* expert_start, const void* W1q,
                  const uint8_t* W1b, const void* W2q, const uint8_t* W2b, const void* hq, const uint8_t* hb, const void* yd) {
    const int rc = fp8_shape_status(s);
    return rc ? rc : xq && xb && expert_start && W1q && W1b && W2q && W2b && hq && hb && yd ? MOE_OK : MOE_ERR_NULL;
}

extern "C" int moe_expert_ffn_fwd_fp8(const moe_fp8_shape* shape, const void* xq, const uint8_t* xb,
                                      const int32_t* expert_start, const void* W1q, const uint8_t* W1b, const void* W2q,
                                      const uint8_t* W2b, void* hq, uint8_t* hb, void* yd, void* stream) {
    const int rc = begin_call(ffn_fp8_check(shape, xq, xb, expert_start, W1q, W1b, W2q, W2b, hq, hb, yd));
    if (rc) return rc;
    const int R = shape->T * shape->k;
    hipStream_t st = (hipStream_t)stream;
    const Fp8Args p1 = fp8_args(R, shape->E, shape->d_model, shape->d_ff, xq, xb, expert_start, W1q, W1b, hq, hb);
    if (shape->act == MOE_GELU) launch_fp8<OUT_GELU8>(p1, st);
    else launch_fp8<OUT_RELU8>(p1, st);
    const Fp8Args p2 = fp8_args(R, shape->E, shape->d_ff, shape->d_model, hq, hb, expert_start, W2q, W2b, yd, nullptr);
    launch_fp8<OUT_BF16>(p2, st);
    return launch_status();
}

// ---------------------------------------------------------------------------
// one pass as one call (host code)
// ---------------------------------------------------------------------------
extern "C" int moe_layer_fwd_fp8(const moe_fp8_shape* s, const moe_router* r, int32_t logits_given, const moe_fp8_buffers* b,
                                 const void* x, const float* Wg, const float* select_bias_or_null,
                                 const uint8_t* token_mask_or_null, const void* W1q, const uint8_t* W1b, const void* W2q,
                                 const uint8_t* W2b, void* stream) {
    if (!s || !r || !b) return MOE_ERR_NULL;
    // everything that a step could refuse, before the first one is issued
    moe_shape gate = {s->T, s->d_model, s->d_ff, s->E, 1, 1, s->dtype, s->act};
    int rc = fp8_shape_status(s);
    if (!rc && (r->T != s->T || r->E != s->E || r->k != s->k)) rc = MOE_ERR_SHAPE;
    if (!rc && !logits_given) rc = gate_logits_check(&gate, x, Wg, b->logits, 0.0f);
    if (!rc) rc = router_fwd_check(r, b->logits, b->expert_idx, b->gate_w);
    if (!rc) rc = sort_check(r, b->expert_idx, b->row_of, b->expert_start, b->ws, b->ws_bytes);
    if (!rc) rc = dispatch_fp8_check(s, x, b->row_of, b->xq, b->xb);
    if (!rc) rc = ffn_fp8_check(s, b->xq, b->xb, b->expert_start, W1q, W1b, W2q, W2b, b->hq, b->hb, b->yd);
    if (!rc) rc = combine_rows_check(s, b->yd, b->row_of, b->gate_w, b->y);
    if (!rc && !logits_given) rc = moe_gate_logits(&gate, x, Wg, nullptr, b->logits, stream);
    if (!rc) rc = moe_router_fwd(r, b->logits, select_bias_or_null, token_mask_or_null, b->expert_idx, b->gate_w, stream);
    if (!rc) rc = moe_sort_choices(r, b->expert_idx, b->row_of, b->expert_start, b->ws, b->ws_bytes, stream);
    if (!rc) rc = moe_dispatch_fp8(s, x, b->row_of, b->xq, b->xb, stream);
    if (!rc) rc = moe_expert_ffn_fwd_fp8(s, b->xq, b->xb, b->expert_start, W1q, W1b, W2q, W2b, b->hq, b->hb, b->yd, stream);
    if (!rc) rc = moe_combine_rows(s, b->yd, b->row_of, b->gate_w, b->y, stream);
    return rc;
}
