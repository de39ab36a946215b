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
typedef short i16x2_t __attribute__((ext_vector_type(2)));

struct Fp8Args {
    const uint8_t *xq, *xb, *wq, *wb;
    const int32_t* start;
    void* y;            // the output, or the hidden activation's bytes
    uint8_t* yb;        // and its exponents
    int rows, E, N;     // N: columns that exist
    int nkb, nnb;       // blocks of 128 along the reduction and the columns
    int xb_stride, yb_stride;       // exponent bytes per row (xb_stride: also per block row of the weights)
};

enum { OUT_BF16 = 0, OUT_F32 = 1, OUT_RELU8 = 2, OUT_GELU8 = 3 };

// one step of 64 reduction entries with the exponents of byte S of either word
template <int S> __device__ __forceinline__ f32x16_t mma(i32x8_t w, i32x8_t x, f32x16_t c, int we, int xe) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w, x, c, 0, 0, S, we, S, xe);
}
__device__ __forceinline__ i32x8_t two16(u32x4_buf_t a, u32x4_buf_t b) {
    return i32x8_t{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
}
__device__ __forceinline__ i32x8_t two16(uint4 a, uint4 b) {
    return i32x8_t{(int)a.x, (int)a.y, (int)a.z, (int)a.w, (int)b.x, (int)b.y, (int)b.z, (int)b.w};
}

// gelu(z) = max(z, 0) - t Phi(-t) with t = |z|, and Phi(-t) = exp(-t^2 / 2) erfcx(t / sqrt 2) / 2, whose second factor is a
// polynomial in u = 1 / (1 + 0.2975 t): seven coefficients, fitted to 64 bits on t <= 13.5 with equal relative errors, leave
// 1.5e-6 of it.  So the error is a share of the value on the left too, where values fall to nothing: a block of 128 of
// nothing but such values has an exponent of its own, and holds them as exactly as any other.  Below -13.2 the exponential is under
// what fp32 holds, and gelu 0.  Rounded to 8 bits, less would do, but an error e of a value moves a share e / step of
// the roundings, and their effect on the output goes with the root of that: 1e-5 would be seen beside bfloat16's rounding.
// 21 instruction slots (exponential and reciprocal four each) instead of the 33 of the two fits that the fp32 experts use: the
// epilogue of the first product is bound by vector instructions.
__device__ __forceinline__ float gelu(float z) {
    constexpr float TAIL[7] = {-0.00011587030167f, 0.12084179371595f, 0.10217944532633f, 0.17530386149883f, -0.06812294572592f,
                               0.25719109177589f, -0.08727779239416f};
    constexpr float TAIL_AT = 0.2975f, LOG2E_HALF = -0.72134752044f;
    const float t = __builtin_amdgcn_fmed3f(fabsf(z), 0.0f, 16.0f);    // (an infinite z: the tail is 0, not infinity times 0)
    const float u = __builtin_amdgcn_rcpf(fmaf(TAIL_AT, t, 1.0f));
    float r = TAIL[6];
#pragma unroll
    for (int i = 5; i >= 0; --i) r = fmaf(r, u, TAIL[i]);
    return fmaf(-t, r * __builtin_amdgcn_exp2f(t * LOG2E_HALF * t), __builtin_elementwise_maximum(z, 0.0f));     // (keeps NaN)
}

// lanes 0..31 end with a = (own a, partner's a), lanes 32..63 with (partner's b, own b)
__device__ __forceinline__ void swap_halves(uint32_t& a, uint32_t& b) {
    const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
    a = r[0];
    b = r[1];
}

// Values of one matrix tile (columns 32 f + 8 q + 4 half + i of the block nb in v[4 q + i]) of row r: the activation and its
// largest magnitude so far, and the tile in the output's type.
template <int OUT>
__device__ __forceinline__ float activate(f32x16_t& v, float top) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float z = v[i], h = OUT == OUT_GELU8 ? gelu(z) : (z <= 0.0f ? 0.0f : z);
        v[i] = h;
        top = fmaxf(top, fabsf(h));         // (NaN are passed over: they become NaN, whatever the exponent)
    }
    return top;
}
// unit: the block's, a power of two (8-bit output); the conversion divides by it
template <int OUT>
__device__ __forceinline__ void store_tile(const Fp8Args& p, const f32x16_t& v, int nb, int f, int r, bool live, int half, float unit) {
    if constexpr (OUT == OUT_RELU8 || OUT == OUT_GELU8) {
        uint32_t d[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            i16x2_t w = {0, 0};
            w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, v[4 * q], v[4 * q + 1], unit, false);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, v[4 * q + 2], v[4 * q + 3], unit, true);
            d[q] = __builtin_bit_cast(uint32_t, w);
        }
        swap_halves(d[0], d[2]);
        swap_halves(d[1], d[3]);
        if (live)
            *reinterpret_cast<uint4*>((uint8_t*)p.y + ((size_t)r * p.nnb + nb) * 128 + 32 * f + 16 * half) = make_uint4(d[0], d[2], d[1], d[3]);
    } else if constexpr (OUT == OUT_F32) {
        float* row = (float*)p.y + (size_t)r * p.N;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int n = nb * 128 + 32 * f + 8 * q + 4 * half;
            if (live && n < p.N) *reinterpret_cast<float4*>(row + n) = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
        }
    } else {
        bf16_t* row = (bf16_t*)p.y + (size_t)r * p.N;
        uint32_t d[4][2];
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int i = 0; i < 2; ++i) d[q][i] = pack_bf16x2(v[4 * q + 2 * i], v[4 * q + 2 * i + 1]);
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            swap_halves(d[q][0], d[q + 2][0]);
            swap_halves(d[q][1], d[q + 2][1]);
            const int n = nb * 128 + 32 * f + 16 * half + 8 * q;
            if (live && n < p.N) *reinterpret_cast<uint4*>(row + n) = make_uint4(d[q][0], d[q][1], d[q + 2][0], d[q + 2][1]);
        }
    }
}
// the exponent byte of block nb of row r, and behind the last block the bytes that fill up
__device__ __forceinline__ void store_byte(const Fp8Args& p, int byte, int nb, int r, int half) {
    uint8_t* bt = p.yb + (size_t)r * p.yb_stride;
    if (half == 0) bt[nb] = (uint8_t)byte;
    else if (nb == p.nnb - 1)
        for (int i = p.nnb; i < p.yb_stride; ++i) bt[i] = 127;
}
// a hidden block's exponent byte, of a unit that fp32 holds as a normal number: 2^-126 at least
__device__ __forceinline__ int block_byte(float top) { return max(1, scale_byte(__float_as_uint(top))); }
__device__ __forceinline__ float block_unit(int byte) { return __uint_as_float((uint32_t)byte << 23); }
// all four tiles of a block in one wave
template <int OUT>
__device__ __forceinline__ void store_block(const Fp8Args& p, f32x16_t (&acc)[4], int nb, int r, bool live, int half) {
    float unit = 1.0f;
    if constexpr (OUT == OUT_RELU8 || OUT == OUT_GELU8) {
        float top = 0.0f;
#pragma unroll
        for (int f = 0; f < 4; ++f) top = activate<OUT>(acc[f], top);
        const int byte = block_byte(fmaxf(top, __shfl_xor(top, 32, MOE_WAVE)));
        unit = block_unit(byte);
        if (live) store_byte(p, byte, nb, r, half);
    }
#pragma unroll
    for (int f = 0; f < 4; ++f) store_tile<OUT>(p, acc[f], nb, f, r, live, half, unit);
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

// ---------------------------------------------------------------------------
// few rows and few columns: a product whose tiles would leave most of the chip idle (the second product of a token or two)
// ---------------------------------------------------------------------------
// A workgroup has 32 columns and 32 rows; its eight waves take an eighth of the reduction each, with the operands
// straight from memory in registers, four blocks of 128 on their way at a time, and nothing shared before the
// partial sums meet in LDS.
#define THIN8_WAVES 8
struct Fp8Slab {            // 128 reduction entries
    u32x4_buf_t w[4], x[4];         // 16-byte chunks 2 j + half
    int we, xe;
};

template <int OUT>
__global__ __launch_bounds__(64 * THIN8_WAVES, 2) void fp8_thin_kernel(const Fp8Args p) {
    static_assert(OUT == OUT_BF16 || OUT == OUT_F32, "a block's largest magnitude would need four such tiles");
    __shared__ float4 s_part[THIN8_WAVES][4][64];       // [wave][q][lane]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, half = lane >> 5, ct = blockIdx.x % (4 * p.nnb), nb = ct >> 2;
    const RowTile t = find_tile<32>(p.start, p.E, p.rows, blockIdx.x / (4 * p.nnb), lane);
    if (t.e < 0) return;
    // rows behind the expert's last one, and entries behind the wave's part, are beyond the buffers: zeros
    const uint32_t kbytes = (uint32_t)p.nkb * 128;
    const size_t left = t.end - t.row;
    const auto wr = buf_rsrc(p.wq + (((size_t)t.e * p.nnb + nb) * 128 + 32 * (ct & 3)) * kbytes, (size_t)32 * kbytes);
    const auto xr = buf_rsrc(p.xq + (size_t)t.row * kbytes, left * kbytes);
    const auto wer = buf_rsrc(p.wb + ((size_t)t.e * p.nnb + nb) * p.xb_stride, p.xb_stride);
    const auto xer = buf_rsrc(p.xb + (size_t)t.row * p.xb_stride, left * p.xb_stride);
    const uint32_t off = l32 * kbytes + 16 * half, xoff = l32 * p.xb_stride;
    f32x16_t acc;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0.0f;
    const int per = (p.nkb + THIN8_WAVES - 1) / THIN8_WAVES, k0 = wave * per, k1 = min(k0 + per, p.nkb);
    auto load = [&](Fp8Slab& s, int kb) {
        const bool in = kb < k1;
        const uint32_t o = in ? off + kb * 128 : BUF_OOB;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            s.w[j] = __builtin_amdgcn_raw_buffer_load_b128(wr, o + 32 * j, 0, 0);
            s.x[j] = __builtin_amdgcn_raw_buffer_load_b128(xr, o + 32 * j, 0, 0);
        }
        s.we = __builtin_amdgcn_raw_buffer_load_b8(wer, in ? kb : BUF_OOB, 0, 0);
        s.xe = __builtin_amdgcn_raw_buffer_load_b8(xer, in ? xoff + kb : BUF_OOB, 0, 0);
    };
    Fp8Slab s[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) load(s[i], k0 + i);
    __builtin_amdgcn_sched_barrier(0);
    for (int kb = k0; kb < k1; kb += 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
                acc = mma<0>(two16(s[i].w[2 * h], s[i].w[2 * h + 1]), two16(s[i].x[2 * h], s[i].x[2 * h + 1]), acc, s[i].we, s[i].xe);
            load(s[i], kb + 4 + i);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) s_part[wave][q][lane] = make_float4(acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]);
    __syncthreads();
    if (wave >= 4) return;
    // wave q finishes columns 8 q + 4 half .. +3 of the tile; the sums are added in the waves' order
    float4 v = s_part[0][wave][lane];
#pragma unroll
    for (int u = 1; u < THIN8_WAVES; ++u) {
        const float4 o = s_part[u][wave][lane];
        v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
    }
    const int r = t.row + l32, n = 32 * ct + 8 * wave + 4 * half;
    if (r >= t.end || n >= p.N) return;
    if constexpr (OUT == OUT_F32) *reinterpret_cast<float4*>((float*)p.y + (size_t)r * p.N + n) = v;
    else *reinterpret_cast<uint2*>((bf16_t*)p.y + (size_t)r * p.N + n) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
}

// ---------------------------------------------------------------------------
// tiles staged through LDS
// ---------------------------------------------------------------------------
// WF x WT waves; a wave has 128 columns and 32 TT rows, four by TT matrix tiles of 32 x 32.  A tile has BT rows: those of all
// waves, or only the first one's (then the others help to load).  A slab is 128 reduction entries of the tile's columns and
// rows; NS slabs have a place in LDS, one is worked on, the others are being filled by loads that write LDS themselves.  A
// workgroup walks its tiles and treats their slabs as one stream, so the next tile's first slabs are on their way during a
// tile's epilogue.
// Bound of the large tile, 131072 rows, 2048 x 8192, 16 experts: second product 1.82 ms (2420 TFLOP/s), where its matrix
// instructions without the loads take 1.21 (3650 TFLOP/s: power holds the clock at 1.8 GHz of 2.4) and its loads without the
// instructions 1.37 to 1.70, from the L2; 56 % of the matrix pipes' cycles are busy, no bank conflicts.  The first product, 2.47
// with gelu and 2.03 with relu, adds its epilogue, which the one workgroup of a CU has nothing to overlap with but the
// next tile's loads.  Neither fragments read ahead, a ring of four slabs of 64, nor loads that warm the L2 gained anything.
template <int WF, int WT, int TT, int BT_, int NS_>
struct Fp8Tile {
    static constexpr int NW = WF * WT, NT = 64 * NW, NS = NS_;
    static constexpr int BF = 128 * WF, BT = BT_;                   // columns and rows
    static constexpr int STAGE = (BF + BT) * 128;
    static constexpr int WL = BF / 8 / NW, XL = BT / 8 / NW;        // loads of a slab per wave: 8 rows of 128 bytes each
    static constexpr int TABLE = NS * STAGE;                        // running tile counts and starts behind the stages
    static constexpr int EXPS = TABLE + (260 + 260) * 4;            // then, per wave, two buffers of exponent words:
    static constexpr int XW = (TT + 1) / 2;                         // XW loads of 64 rows' ones and one of the columns'
    static constexpr int BYTES = EXPS + NW * 2 * (XW + 1) * 256;
    static_assert(BF % (8 * NW) == 0 && BT % (8 * NW) == 0 && NW % 2 == 0, "whole loads per wave");
    static_assert((NS - 2) * (WL + XL) < 64, "vmcnt is a 6-bit counter");
    static_assert(NS == 2 || NS == 3, "two buffers of exponents");
};

#define FP8_BAND 4      // row tiles per band of the walk inside an expert: an XCD's workgroups share 4 row panels at a time

struct Fp8Place { int e, row, end, col; };      // a tile: expert, first row, the expert's end, first block of 128 columns

// eight e4m3 values as fp16, which holds them all
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
__device__ __forceinline__ f16x8_t to_f16(uint32_t lo, uint32_t hi) {
    const f16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true);
    const f16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true);
    return f16x8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// which tile is number `at` (found by the whole wave)
template <int BT, int WF>
__device__ __forceinline__ Fp8Place fp8_place(const int* tiles, const int* start, int at, int ctiles, int lane) {
    const int4 t = *reinterpret_cast<const int4*>(tiles + 4 * lane);        // running counts in front of four experts
    const int next = tiles[4 * lane + 4];
    int q = -1;
    if (at >= t.x && at < t.y) q = 0;
    else if (at >= t.y && at < t.z) q = 1;
    else if (at >= t.z && at < t.w) q = 2;
    else if (at >= t.w && at < next) q = 3;
    const int src = __ffsll((long long)__ballot(q >= 0)) - 1;
    const int e = __builtin_amdgcn_readfirstlane(__shfl(4 * lane + q, src, MOE_WAVE));
    const int in = at - __builtin_amdgcn_readfirstlane(tiles[e]);
    const int s0 = __builtin_amdgcn_readfirstlane(start[e]), s1 = __builtin_amdgcn_readfirstlane(start[e + 1]);
    const int rt = (s1 - s0 + BT - 1) / BT, band = in / (FP8_BAND * ctiles), high = min(FP8_BAND, rt - FP8_BAND * band);
    const int within = in - band * FP8_BAND * ctiles, col = within / high;
    return {e, __builtin_amdgcn_readfirstlane(s0 + (FP8_BAND * band + within - col * high) * BT), s1,
            __builtin_amdgcn_readfirstlane(col * WF)};
}

// FINE: the products are formed of fp16 operands and added in fp32, slab by slab, so that they are as exact as fp32 sums;
// the four waves have 32 columns of all rows each, and share the conversion of the columns.  For hidden activations of few
// rows: they are rounded to 4 bits, where a sum that is 2^-14 off falls to the other side of a tie in 1 of 900 entries, and
// such steps of 6 % show where few rows are summed (48 rows of 376: outputs 0.3 % off, bf16's rounding 0.17).  The matrix
// instructions take twice as long, which the weights' bytes hide.
// TURNS: the tiles begin their reduction at different slabs and come round.  Workgroups that walk rows of a multiple of 4096
// bytes in step ask the same memory channels: second product of 122 rows, 32 experts, 1024 x 4096, weights from memory,
// 34.3 us in step, 28.1 like this; with rows of 2048, 3968 or 4224 bytes 26 either way.  (Its instructions cost a token's
// product 0.7 us: not where nothing is gained.)
template <int WF, int WT, int TT, int BT, int NS, int OUT, bool FINE, bool TURNS>
__global__ __launch_bounds__(64 * WF * WT, 2) void fp8_tile_kernel(const Fp8Args p) {
    typedef Fp8Tile<WF, WT, TT, BT, NS> G;
    extern __shared__ __align__(1024) uint8_t smem[];
    int* tiles = reinterpret_cast<int*>(smem + G::TABLE);
    int* start = tiles + 260;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, half = lane >> 5, wf = wave % WF, wt = FINE ? 0 : wave / WF;     // (waves without rows are then spread over the SIMDs)
    const int ctiles = (p.nnb + WF - 1) / WF;
    if (wave == 0) {
        int s[5], t[4], n = 0;
#pragma unroll
        for (int q = 0; q < 5; ++q) s[q] = min(max(p.start[min(4 * lane + q, p.E)], 0), p.rows);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            t[q] = 4 * lane + q < p.E ? (max(s[q + 1] - s[q], 0) + G::BT - 1) / G::BT * ctiles : 0;
            n += t[q];
        }
        int run = n;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int u = __shfl_up(run, o, MOE_WAVE);
            if (lane >= o) run += u;
        }
        if (lane == 63) { tiles[256] = run; start[256] = s[4]; }
        run -= n;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            tiles[4 * lane + q] = run;
            start[4 * lane + q] = s[q];
            run += t[q];
        }
    }
    __syncthreads();
    const int total = __builtin_amdgcn_readfirstlane(tiles[256]);
    // workgroup w is on XCD w % 8; an XCD takes as many consecutive tiles at a time as it has workgroups, or an eighth of
    // them where there are fewer: the grid holds for any distribution of the rows
    const int per = min((int)gridDim.x >> 3, (total + 7) >> 3), xcd = blockIdx.x & 7;
    int at = xcd * per + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per || at >= total) return;
    const int stride = per * 8;
    const uint32_t kbytes = (uint32_t)p.nkb * 128;
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)smem;

    // loads of a slab: lane l fills 16 bytes of row 8 m + l / 8; the chunks of a row are permuted by bits 1..3 of the row, so
    // that 16 rows' reads of one chunk hit all 64 banks
    const int lrow = lane >> 3, chunk = (lane & 7) ^ (((lrow >> 1) + 4 * (wave & 1)) & 7);
    uint32_t voff[G::WL > G::XL ? G::WL : G::XL];
#pragma unroll
    for (int i = 0; i < (G::WL > G::XL ? G::WL : G::XL); ++i)
        voff[i] = (uint32_t)((i * G::NW + wave) * 8 + lrow) * kbytes + 16 * chunk;
    // fragment reads
    uint32_t frag[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) frag[c] = l32 * 128 + (((4 * (c >> 1) + 2 * half + (c & 1)) ^ ((l32 >> 1) & 7)) << 4);
    const uint32_t wbase = wf * 128 * 128, xbase = G::BF * 128 + wt * TT * 32 * 128;

    auto scalar = [](uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); };
    auto desc = [&](uint64_t base, uint64_t n) {
        return u32x4_buf_t{scalar((uint32_t)base), scalar((uint32_t)(base >> 32) & 0xffffu), scalar(n < 0x7fffffffull ? (uint32_t)n : 0x7fffffffu), 0x00020000u};
    };
    auto load_word = [](u32x4_buf_t d, uint32_t off, uint32_t to) {         // 64 lanes' words, one after the other
        asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dword %1, %2, 0 offen lds" :: "s"(to), "v"(off), "s"(d) : "memory");
    };
    // the cursor of the loads, NS - 1 slabs ahead of the products: the tile, its slab, and what is left of its operands
    Fp8Place next = fp8_place<G::BT, WF>(tiles, start, at, ctiles, lane);
    auto begin = [&](const Fp8Place& t) { return TURNS ? ((t.e * p.nnb + t.col) & 7) * 4 : 0; };
    int nkb = begin(next), done = 0;    // the slab, and how many of the tile's went before
    int group = 0;                      // which buffer takes the exponents of the next four slabs
    bool more = true;
    u32x4_buf_t wd, xd;
    auto aim = [&]() {
        const uint32_t k = (uint32_t)nkb * 128;
        wd = desc((uint64_t)(p.wq + ((size_t)next.e * p.nnb + next.col) * 128 * kbytes + k), (uint64_t)(p.nnb - next.col) * 128 * kbytes - k);
        xd = desc((uint64_t)(p.xq + (size_t)next.row * kbytes + k), (uint64_t)(next.end - next.row) * kbytes - k);
    };
    auto step = [&](u32x4_buf_t& d) {   // 128 bytes further, and as much less to the end
        const uint32_t lo = d[0] + 128;
        d[1] = scalar(d[1] + (lo < 128 ? 1 : 0));
        d[0] = scalar(lo);
        d[2] = scalar(d[2] > 128 ? d[2] - 128 : 0);
    };
    const uint32_t exps = lds + G::EXPS + wave * 2 * (G::XW + 1) * 256;
    // Past the last tile the requests go on, for nothing (an empty range), so that a wait can count on their number.
    auto fetch = [&](int stage) {
        if ((nkb & 3) == 0) {
            const int nb = min(next.col + wf, p.nnb - 1);
            const uint32_t to = scalar(exps + group * (G::XW + 1) * 256);
            group ^= 1;
            const u32x4_buf_t ed = desc((uint64_t)(p.xb + (size_t)next.row * p.xb_stride + nkb),
                                        more ? (uint64_t)min(next.end - next.row, G::BT) * p.xb_stride - nkb : 0);
#pragma unroll
            for (int i = 0; i < G::XW; ++i) load_word(ed, (uint32_t)(wt * TT * 32 + 64 * i + lane) * p.xb_stride, to + 256 * i);
            load_word(desc((uint64_t)(p.wb + ((size_t)next.e * p.nnb + nb) * p.xb_stride + nkb), more ? 4 : 0), 0, to + 256 * G::XW);
        }
        const uint32_t to = scalar(lds + stage * G::STAGE);
#pragma unroll
        for (int i = 0; i < G::WL; ++i) load_to_lds(wd, voff[i], to + (i * G::NW + wave) * 1024);
#pragma unroll
        for (int i = 0; i < G::XL; ++i) load_to_lds(xd, voff[i], to + G::BF * 128 + (i * G::NW + wave) * 1024);
        ++nkb;
        if (++done < p.nkb) {
            if (TURNS && nkb == p.nkb) {
                nkb = 0;
                if (more) aim();
            } else {
                step(wd);
                step(xd);
            }
        } else {
            nkb = 0;
            done = 0;
            at += stride;
            more = more && at < total;
            if (more) {
                next = fp8_place<G::BT, WF>(tiles, start, at, ctiles, lane);
                nkb = begin(next);
                aim();
            } else {
                wd[2] = xd[2] = 0;
            }
        }
    };
    aim();
    Fp8Place cur = next;
    int cat = at;                       // the products' tile
#pragma unroll
    for (int s = 0; s < NS - 1; ++s) fetch(s);
    int stage = 0, have = 0;
    for (;;) {
        constexpr int FT = FINE ? 1 : 4;        // matrix tiles side by side
        f32x16_t acc[TT][FT];
#pragma unroll
        for (int t = 0; t < TT; ++t)
#pragma unroll
            for (int f = 0; f < FT; ++f)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[t][f][i] = 0.0f;
        int we = 0, xe[TT] = {};
        // a wave without rows (or columns) only helps to load: its products would cost the time of the others' and power, which
        // is what limits the clock
        const bool live = wt * TT * 32 < G::BT && cur.row + wt * TT * 32 < cur.end && cur.col + wf < p.nnb;
        int kb = begin(cur);
        for (int n = 0; n < p.nkb; ++n) {
            // this slab has arrived once at most the NS - 2 younger ones are outstanding, and every wave is done with the one
            // before, whose place is filled again
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"((NS - 2) * (G::WL + G::XL)) : "memory");
            if ((kb & 3) == 0) {
                const int* e = reinterpret_cast<const int*>(smem + G::EXPS + (wave * 2 + have) * (G::XW + 1) * 256);
                have ^= 1;
#pragma unroll
                for (int t = 0; t < TT; ++t) xe[t] = e[32 * t + l32];
                we = e[64 * G::XW];
                // with three slabs in flight and a reduction of one, the next request is for this very buffer
                if constexpr (NS > 2) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            }
            fetch(stage == 0 ? NS - 1 : stage - 1);
            if constexpr (FINE) {
                const uint8_t* w = smem + stage * G::STAGE + wave * 4096;
                const uint8_t* x = smem + stage * G::STAGE + G::BF * 128;
                f16x8_t a[8];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const uint4 v = *reinterpret_cast<const uint4*>(w + frag[c]);
                    a[2 * c] = to_f16(v.x, v.y);
                    a[2 * c + 1] = to_f16(v.z, v.w);
                }
#pragma unroll
                for (int t = 0; t < TT; ++t) {
                    if (cur.row + 32 * t >= cur.end) break;
                    f32x16_t part;
#pragma unroll
                    for (int i = 0; i < 16; ++i) part[i] = 0.0f;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const uint4 v = *reinterpret_cast<const uint4*>(x + t * 4096 + frag[c]);
                        part = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[2 * c], to_f16(v.x, v.y), part, 0, 0, 0);
                        part = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[2 * c + 1], to_f16(v.z, v.w), part, 0, 0, 0);
                    }
                    const int e = (we & 255) + (xe[t] & 255) - 254;
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[t][0][i] += ldexpf(part[i], e);
                }
            } else if (live) {
                const uint8_t* w = smem + stage * G::STAGE + wbase;
                const uint8_t* x = smem + stage * G::STAGE + xbase;
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    i32x8_t b[TT];
#pragma unroll
                    for (int t = 0; t < TT; ++t)
                        b[t] = two16(*reinterpret_cast<const uint4*>(x + t * 4096 + frag[2 * s]), *reinterpret_cast<const uint4*>(x + t * 4096 + frag[2 * s + 1]));
#pragma unroll
                    for (int f = 0; f < 4; ++f) {
                        const i32x8_t a = two16(*reinterpret_cast<const uint4*>(w + f * 4096 + frag[2 * s]), *reinterpret_cast<const uint4*>(w + f * 4096 + frag[2 * s + 1]));
#pragma unroll
                        for (int t = 0; t < TT; ++t) acc[t][f] = mma<0>(a, b[t], acc[t][f], we, xe[t]);
                    }
                }
            }
            we = (int)((uint32_t)we >> 8);
#pragma unroll
            for (int t = 0; t < TT; ++t) xe[t] = (int)((uint32_t)xe[t] >> 8);
            stage = stage == NS - 1 ? 0 : stage + 1;
            ++kb;
            if (TURNS && kb == p.nkb) kb = 0;
        }
        if constexpr (FINE) {
            static_assert(OUT == OUT_RELU8 || OUT == OUT_GELU8, "a block's largest magnitude is what the waves share");
            float* tops = reinterpret_cast<float*>(smem + G::BYTES);        // [wave][row]
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                const float top = activate<OUT>(acc[t][0], 0.0f), other = __shfl_xor(top, 32, MOE_WAVE);
                if (half == 0) tops[wave * BT + 32 * t + l32] = fmaxf(top, other);
            }
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");       // (the loads stay under way)
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                float top = 0.0f;
#pragma unroll
                for (int u = 0; u < G::NW; ++u) top = fmaxf(top, tops[u * BT + 32 * t + l32]);
                const int byte = block_byte(top), r = cur.row + 32 * t + l32;
                if (wave == 0 && r < cur.end) store_byte(p, byte, cur.col, r, half);
                store_tile<OUT>(p, acc[t][0], cur.col, wave, r, r < cur.end, half, block_unit(byte));
            }
        } else if (live) {
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                const int r = cur.row + (wt * TT + t) * 32 + l32;
                store_block<OUT>(p, acc[t], cur.col + wf, r, r < cur.end, half);
            }
        }
        cat += stride;
        if (cat >= total) break;
        cur = fp8_place<G::BT, WF>(tiles, start, cat, ctiles, lane);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // the last requests write this workgroup's LDS
}

// compute units of the current device (looked up once per device)
static int compute_units() {
    static int cached[64];
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 256;
    int n = __atomic_load_n(&cached[dev], __ATOMIC_RELAXED);
    if (n == 0) {
        int v = 0;
        n = (hipDeviceGetAttribute(&v, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess && v > 0) ? v : 256;
        __atomic_store_n(&cached[dev], n, __ATOMIC_RELAXED);
    }
    return n;
}

template <int WF, int WT, int TT, int BT, int NS, int OUT, bool FINE = false, bool TURNS = false>
static int launch_tiles(const Fp8Args& p, int per_cu, hipStream_t st) {
    typedef Fp8Tile<WF, WT, TT, BT, NS> G;
    static unsigned long long opted;
    const auto kern = fp8_tile_kernel<WF, WT, TT, BT, NS, OUT, FINE, TURNS>;
    constexpr size_t lds = G::BYTES + (FINE ? G::NW * BT * 4 : 0);
    if (!lds_opt_in((const void*)kern, lds, &opted)) return MOE_ERR_LAUNCH;
    const long long most = ((long long)p.rows / G::BT + (p.E < p.rows ? p.E : p.rows)) * ((p.nnb + WF - 1) / WF);
    long long wgs = (long long)compute_units() * per_cu / 8 * 8;
    if (wgs < 8) wgs = 8;
    if (wgs > (most + 7) / 8 * 8) wgs = (most + 7) / 8 * 8;
    kern<<<(unsigned)wgs, G::NT, lds, st>>>(p);
    return MOE_OK;
}

// Which kernel?  Estimated from the mean rows of the experts that can have any.
enum { FP8_LARGE = 0, FP8_SMALL = 1, FP8_THIN = 2, FP8_NARROW = 3 };
// 256 x 256 or 128 x 128: a CU holds one workgroup of the large tile, which works off its area a fifth faster (half the
// operands per product), or two of the small one; either way the launch takes whole rounds of tiles.  Measured, large against
// small, us, first product with gelu, second with bf16 output, with fp32 output: 131072 rows, 2048 x 8192, 16 experts: 2470,
// 2950; 1815, 2255; 1895, 2370.  29500 rows, 1024 x 4096, 64 experts: 207, 247; 140, 171; 152, 190.  10006 rows, 776 x 3080, 6
// experts with a Zipf gate: 67, 54 (three rounds against four halves); 45, 53; 47, 55.  4096 rows, 1024 x 4096, 16 experts: 29,
// 30; (64 tiles) 50, 30; 55, 31.
// 128 columns x 64 rows, three slabs in flight instead of two: where an expert's rows fit one tile either way, the weights'
// bytes are the time, and more of them are on their way.  Narrow against small, us, both products of 32 experts, 1024 x 4096
// (268 MB of weights): 122 rows 51.7, 60.0; 1024 rows 52.4, 61.9; 1536 rows 59.4, 65.3; beyond, a second row tile for some of
// the experts costs more than that (4096 rows 100, 77.6).
// 32 x 32 with an eight-way split reduction: where there are so few tiles that one tile's reduction is the launch's
// time, 0.6 us for each of its 128 entries, against 0.084 us for each tile's worth of thin ones.  Second products: 8 rows of
// 8 experts, 1024 x 4096: 23.1 us with the small tile, 10.4 thin; 2048 x 2048: 12.8 with the narrow tile, 15.7 thin; 122 rows
// of 32 experts, 1024 x 4096: 23, 41.
static int fp8_kernel(int rows, int experts, int nkb, int nnb, bool hidden) {
    const long long E = experts < rows ? experts : rows, per = (rows + E - 1) / E, cus = compute_units();
    const long long large = E * ((per + 255) / 256) * ((nnb + 1) / 2), small = E * ((per + 127) / 128) * nnb;
    if (!hidden && per <= 32 && 7 * (long long)nkb > 15 + small) return FP8_THIN;
    if (per <= 48) return FP8_NARROW;
    return 40 * ((large + cus - 1) / cus) < 24 * ((small + 2 * cus - 1) / (2 * cus)) ? FP8_LARGE : FP8_SMALL;
}

template <int OUT>
static int launch_fp8(const Fp8Args& p, hipStream_t st) {
    constexpr bool HIDDEN = OUT == OUT_RELU8 || OUT == OUT_GELU8;
    const int kind = fp8_kernel(p.rows, p.E, p.nkb, p.nnb, HIDDEN);
    if constexpr (!HIDDEN) {
        if (kind == FP8_THIN) {
            const long long most = (long long)p.rows / 32 + (p.E < p.rows ? p.E : p.rows);     // row tiles, at most
            fp8_thin_kernel<OUT><<<(unsigned)(most * p.nnb * 4), 64 * THIN8_WAVES, 0, st>>>(p);
            return MOE_OK;
        }
    }
    if (kind == FP8_NARROW) {
        constexpr int TT = HIDDEN ? 2 : 1;
        return p.nkb % 32 ? launch_tiles<1, 4, TT, 64, 3, OUT, HIDDEN>(p, 2, st) : launch_tiles<1, 4, TT, 64, 3, OUT, HIDDEN, true>(p, 2, st);
    }
    return kind == FP8_LARGE ? launch_tiles<2, 4, 2, 256, 2, OUT>(p, 1, st) : launch_tiles<1, 4, 1, 128, 2, OUT>(p, 2, st);
}

// measurement aid: the kernels of the block's two products
extern "C" int moe_fp8_kernels(const moe_fp8_shape* shape, int32_t* first, int32_t* second) {
    const int rc = fp8_shape_status(shape);
    if (rc) return rc;
    if (!first || !second) return MOE_ERR_NULL;
    const int R = shape->T * shape->k, d = fp8_blocks(shape->d_model), f = fp8_blocks(shape->d_ff);
    *first = fp8_kernel(R, shape->E, d, f, true);
    *second = fp8_kernel(R, shape->E, f, d, false);
    return MOE_OK;
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
                                      const int32_t* expert_start, const void* Wq, const uint8_t* Wb, int32_t y_dtype,
                                      void* y, void* stream) {
    int rc = begin_call(fp8_extent_status(rows, E, K, N, y_dtype));
    if (rc) return rc;
    if (!xq || !xb || !expert_start || !Wq || !Wb || !y) return MOE_ERR_NULL;
    if (!aligned(16, xq, Wq, y) || !aligned(4, xb, Wb)) return MOE_ERR_SHAPE;
    const Fp8Args p = fp8_args(rows, E, K, N, xq, xb, expert_start, Wq, Wb, y, nullptr);
    rc = y_dtype == MOE_BF16 ? launch_fp8<OUT_BF16>(p, (hipStream_t)stream) : launch_fp8<OUT_F32>(p, (hipStream_t)stream);
    return rc ? rc : launch_status();
}

int fp8_shape_status(const moe_fp8_shape* s) {
    if (!s) return MOE_ERR_NULL;
    if (s->dtype != MOE_BF16 || (s->act != MOE_RELU && s->act != MOE_GELU)) return MOE_ERR_DTYPE;
    if (s->T < 1 || s->k < 1 || s->k > 8 || (int64_t)s->T * s->k >= (1 << 30)) return MOE_ERR_SHAPE;
    return fp8_extent_status(s->T * s->k, s->E, s->d_model, s->d_ff, s->dtype);
}

int ffn_fp8_check(const moe_fp8_shape* s, const void* xq, const uint8_t* xb, const int32_t* expert_start, const void* W1q,
                  const uint8_t* W1b, const void* W2q, const uint8_t* W2b, const void* hq, const uint8_t* hb, int yd_dtype,
                  const void* yd) {
    const int rc = fp8_shape_status(s);
    if (rc) return rc;
    if (yd_dtype != MOE_F32 && yd_dtype != MOE_BF16) return MOE_ERR_DTYPE;
    if (!(xq && xb && expert_start && W1q && W1b && W2q && W2b && hq && hb && yd)) return MOE_ERR_NULL;
    return aligned(16, xq, W1q, W2q, hq, yd) && aligned(4, xb, W1b, W2b, hb) ? MOE_OK : MOE_ERR_SHAPE;
}

extern "C" int moe_expert_ffn_fwd_fp8(const moe_fp8_shape* shape, const void* xq, const uint8_t* xb,
                                      const int32_t* expert_start, const void* W1q, const uint8_t* W1b, const void* W2q,
                                      const uint8_t* W2b, void* hq, uint8_t* hb, int32_t yd_dtype, void* yd,
                                      void* stream) {
    int rc = begin_call(ffn_fp8_check(shape, xq, xb, expert_start, W1q, W1b, W2q, W2b, hq, hb, yd_dtype, yd));
    if (rc) return rc;
    const int R = shape->T * shape->k;
    hipStream_t st = (hipStream_t)stream;
    const Fp8Args p1 = fp8_args(R, shape->E, shape->d_model, shape->d_ff, xq, xb, expert_start, W1q, W1b, hq, hb);
    rc = shape->act == MOE_GELU ? launch_fp8<OUT_GELU8>(p1, st) : launch_fp8<OUT_RELU8>(p1, st);
    if (rc) return rc;
    const Fp8Args p2 = fp8_args(R, shape->E, shape->d_ff, shape->d_model, hq, hb, expert_start, W2q, W2b, yd, nullptr);
    rc = yd_dtype == MOE_BF16 ? launch_fp8<OUT_BF16>(p2, st) : launch_fp8<OUT_F32>(p2, st);
    return rc ? rc : launch_status();
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
    if (!rc) rc = ffn_fp8_check(s, b->xq, b->xb, b->expert_start, W1q, W1b, W2q, W2b, b->hq, b->hb, MOE_F32, b->yd);
    if (!rc) rc = combine_rows_check(s, MOE_F32, b->yd, b->row_of, b->gate_w, b->y);
    if (!rc && !logits_given) rc = moe_gate_logits(&gate, x, Wg, nullptr, b->logits, stream);
    if (!rc) rc = moe_router_fwd(r, b->logits, select_bias_or_null, token_mask_or_null, b->expert_idx, b->gate_w, stream);
    if (!rc) rc = moe_sort_choices(r, b->expert_idx, b->row_of, b->expert_start, b->ws, b->ws_bytes, stream);
    if (!rc) rc = moe_dispatch_fp8(s, x, b->row_of, b->xq, b->xb, stream);
    if (!rc) rc = moe_expert_ffn_fwd_fp8(s, b->xq, b->xb, b->expert_start, W1q, W1b, W2q, W2b, b->hq, b->hb, MOE_F32, b->yd, stream);
    if (!rc) rc = moe_combine_rows(s, MOE_F32, b->yd, b->row_of, b->gate_w, b->y, stream);
    return rc;
}
