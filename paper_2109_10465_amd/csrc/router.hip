// moe_router_fwd / moe_router_bwd: choice and weights of 1..8 experts per token out of at most 256,
// within groups of experts; moe_sort_choices: rows of the choices, expert by expert; moe_combine_rows:
// the mixture of such rows.
#include <math.h>
#include "moe_common.h"

#define ROUTER_MAX_K 8
#define LOGISTIC_ZERO -690.0f    // logits below have a logistic score under 1e-299, which counts as 0 (as exp overflows it does in 64 bits)

// ---------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------
// LPT lanes share a token and hold Q consecutive experts of one group each: group g has the Lg lanes from
// g * Lg on, so the order of (lane, entry) is the order of the ids, whatever the groups' size.
struct RouterArgs {
    int T, E, k, score, n_groups, group, top_groups, group_best, renormalise;   // group = experts per group
    float scale;
    int lg_log2, lpt_log2;          // lanes per group and per token
};

__device__ __forceinline__ double score64(double l, bool sigmoid, double top, double total) {
    return sigmoid ? 1.0 / (1.0 + exp(-l)) : exp(l - top) / total;
}

template <typename V> __device__ __forceinline__ bool ahead(V va, int ia, V vb, int ib) {
    return va > vb || (va == vb && ia < ib);
}

// V: what the choice compares - the logits themselves (float), or score + bias (double)
template <int Q, typename V>
__global__ __launch_bounds__(256) void router_fwd_kernel(const RouterArgs a, const float* __restrict__ logits,
                                                         const float* __restrict__ bias, const uint8_t* __restrict__ mask,
                                                         int32_t* __restrict__ expert_idx, float* __restrict__ gate_w) {
    constexpr bool BIAS = sizeof(V) == 8;
    const int lpt = 1 << a.lpt_log2, lg = 1 << a.lg_log2;
    const int sub = threadIdx.x & (lpt - 1), t = blockIdx.x * (256 >> a.lpt_log2) + (threadIdx.x >> a.lpt_log2);
    const int g = sub >> a.lg_log2, first = (sub & (lg - 1)) * Q, e0 = g * a.group + first;
    const int here = g < a.n_groups ? min(max(a.group - first, 0), Q) : 0;
    const bool in = t < a.T, valid = in && (!mask || mask[t] != 0);
    const bool sigmoid = a.score == MOE_SIGMOID;
    const float* row = logits + (size_t)(in ? t : 0) * a.E;
    float l[Q];
#pragma unroll
    for (int i = 0; i < Q; ++i) {
        l[i] = valid && i < here ? row[e0 + i] : -INFINITY;
        if (!(l[i] == l[i])) l[i] = -INFINITY;
    }
    // the softmax's largest logit and sum, where scores are compared or not divided by the chosen ones' sum
    float top = 0.0f;
    double total = 1.0;
    if (!sigmoid) {
        top = l[0];
#pragma unroll
        for (int i = 1; i < Q; ++i) top = fmaxf(top, l[i]);
        for (int o = lpt >> 1; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, MOE_WAVE));
        if (top == -INFINITY) top = 0.0f;
        total = 0.0;
#pragma unroll
        for (int i = 0; i < Q; ++i) total += exp((double)l[i] - (double)top);
        for (int o = lpt >> 1; o > 0; o >>= 1) total += __shfl_xor(total, o, MOE_WAVE);
        if (!(total > 0.0)) total = 1.0;
    }
    V v[Q];
    unsigned left = (1u << here) - 1u;          // experts that can still be chosen
#pragma unroll
    for (int i = 0; i < Q; ++i) {
        if constexpr (BIAS) {
            v[i] = -INFINITY;
            if (valid && i < here && l[i] > -INFINITY) {
                const double w = score64(l[i], sigmoid, top, total) + (double)bias[e0 + i];
                if (w == w) v[i] = w;
            }
        } else {
            v[i] = l[i];
        }
    }
    if (a.n_groups > 1) {
        V b0 = -INFINITY, b1 = -INFINITY;
#pragma unroll
        for (int i = 0; i < Q; ++i) {
            if (v[i] > b0) { b1 = b0; b0 = v[i]; } else if (v[i] > b1) b1 = v[i];
        }
        for (int o = lg >> 1; o > 0; o >>= 1) {
            const V c0 = __shfl_xor(b0, o, MOE_WAVE), c1 = __shfl_xor(b1, o, MOE_WAVE);
            const V lo = b0 < c0 ? b0 : c0;
            b0 = b0 < c0 ? c0 : b0;
            b1 = b1 < c1 ? c1 : b1;
            b1 = b1 < lo ? lo : b1;
        }
        double gv = (double)b0;
        if (a.group_best == 2) {
            if constexpr (BIAS) gv = b0 + b1;
            else gv = b1 == -INFINITY ? -INFINITY
                                      : score64(b0, sigmoid, top, total) + score64(b1, sigmoid, top, total);
        }
        if (!(gv == gv) || g >= a.n_groups) gv = -INFINITY;
        int before = 0;                         // groups in front of this one
        for (int o = 1; o < lpt >> a.lg_log2; ++o) {
            const double w = __shfl_xor(gv, o << a.lg_log2, MOE_WAVE);
            before += (g ^ o) < a.n_groups && ahead(w, g ^ o, gv, g);
        }
        if (before >= a.top_groups) left = 0;
    }
    int choice[ROUTER_MAX_K];
#pragma unroll
    for (int j = 0; j < ROUTER_MAX_K; ++j) {
        choice[j] = 0;
        if (j >= a.k) continue;
        V best = -INFINITY;
        int id = 0x7fffffff;
#pragma unroll
        for (int i = 0; i < Q; ++i)
            if ((left >> i & 1u) && ahead(v[i], e0 + i, best, id)) { best = v[i]; id = e0 + i; }
        for (int o = lpt >> 1; o > 0; o >>= 1) {
            const V w = __shfl_xor(best, o, MOE_WAVE);
            const int wi = __shfl_xor(id, o, MOE_WAVE);
            if (ahead(w, wi, best, id)) { best = w; id = wi; }
        }
        choice[j] = id;
        if (id >= e0 && id < e0 + here) left &= ~(1u << (id - e0));
    }
    if (!in || sub != 0) return;
    if (!valid) {
        for (int j = 0; j < a.k; ++j) {
            expert_idx[(size_t)t * a.k + j] = -1;
            gate_w[(size_t)t * a.k + j] = 0.0f;
        }
        return;
    }
    float cl[ROUTER_MAX_K], most = -INFINITY;
#pragma unroll
    for (int j = 0; j < ROUTER_MAX_K; ++j) {
        cl[j] = j < a.k ? row[choice[j]] : -INFINITY;
        most = fmaxf(most, cl[j]);
    }
    // renormalised scores, scaled so that the largest is near 1: exp(l - most), or 1 / (e^-M + e^(-l - M)) with M = max(0, -most)
    float s[ROUTER_MAX_K], sum = 0.0f;
    const float m = a.renormalise ? fmaxf(0.0f, -most) : 0.0f, em = expf(-m);
#pragma unroll
    for (int j = 0; j < ROUTER_MAX_K; ++j) {
        if (cl[j] == -INFINITY || (sigmoid && cl[j] < LOGISTIC_ZERO)) s[j] = 0.0f;
        else if (sigmoid) s[j] = 1.0f / (em + expf(-cl[j] - m));
        else s[j] = a.renormalise ? expf(cl[j] - most) : (float)(exp((double)cl[j] - (double)top) / total);
        sum += s[j];
    }
    const float c = !a.renormalise ? a.scale : sum == 0.0f ? 0.0f : a.scale / sum;
#pragma unroll
    for (int j = 0; j < ROUTER_MAX_K; ++j) {
        if (j < a.k) {
            expert_idx[(size_t)t * a.k + j] = choice[j];
            gate_w[(size_t)t * a.k + j] = s[j] * c;
        }
    }
}

// ---------------------------------------------------------------------------
// backward: a wave per token, four consecutive experts per lane
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(256) void router_bwd_kernel(const RouterArgs a, const float* __restrict__ logits,
                                                         const int32_t* __restrict__ expert_idx,
                                                         const float* __restrict__ dgate_w, float* __restrict__ dlogits) {
    const int lane = threadIdx.x & 63, t = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (t >= a.T) return;
    const bool sigmoid = a.score == MOE_SIGMOID;
    const float* row = logits + (size_t)t * a.E;
    int id[ROUTER_MAX_K];
    float cl[ROUTER_MAX_K], dw[ROUTER_MAX_K], most = -INFINITY;
    bool any = false;
#pragma unroll
    for (int j = 0; j < ROUTER_MAX_K; ++j) {
        id[j] = j < a.k ? expert_idx[(size_t)t * a.k + j] : -1;
        const bool ok = (unsigned)id[j] < (unsigned)a.E;
        any |= ok;
        cl[j] = ok ? row[id[j]] : -INFINITY;
        dw[j] = ok ? dgate_w[(size_t)t * a.k + j] : 0.0f;
        most = fmaxf(most, cl[j]);
    }
    float out[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (any) {
        float r[ROUTER_MAX_K], q[ROUTER_MAX_K], sum = 0.0f, all = 0.0f, top = 0.0f, inv = 1.0f;
        float l[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        const bool dense = !sigmoid && !a.renormalise;
        if (dense) {
            top = -INFINITY;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (4 * lane + i < a.E) l[i] = row[4 * lane + i];
                top = fmaxf(top, l[i]);
            }
            top = wave_max(top);
            if (top == -INFINITY) top = 0.0f;
            float total = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) total += expf(l[i] - top);
            total = wave_sum(total);
            inv = total > 0.0f ? 1.0f / total : 0.0f;
        }
        const float m = a.renormalise ? fmaxf(0.0f, -most) : 0.0f, em = expf(-m);
#pragma unroll
        for (int j = 0; j < ROUTER_MAX_K; ++j) {
            if (cl[j] == -INFINITY || (sigmoid && cl[j] < LOGISTIC_ZERO)) r[j] = 0.0f;
            else if (sigmoid) r[j] = 1.0f / (em + expf(-cl[j] - m));
            else r[j] = a.renormalise ? expf(cl[j] - most) : expf(cl[j] - top) * inv;
            sum += r[j];
        }
        float mean = 0.0f;
        if (a.renormalise) {
            const float c = sum > 0.0f ? 1.0f / sum : 0.0f;
#pragma unroll
            for (int j = 0; j < ROUTER_MAX_K; ++j) {
                r[j] *= c;
                mean = fmaf(dw[j], r[j], mean);
            }
        }
#pragma unroll
        for (int j = 0; j < ROUTER_MAX_K; ++j) {
            q[j] = a.scale * r[j] * (dw[j] - mean);
            all += q[j];
            if (sigmoid) q[j] *= 1.0f / (1.0f + expf(cl[j]));
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (id[j] == 4 * lane + i) out[i] += q[j];
        }
        if (dense) {
#pragma unroll
            for (int i = 0; i < 4; ++i) out[i] -= expf(l[i] - top) * inv * all;
        }
    }
    float* o = dlogits + (size_t)t * a.E;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (4 * lane + i < a.E) o[4 * lane + i] = out[i];
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
int router_status(const moe_router* r) {
    if (!r) return MOE_ERR_NULL;
    if (r->score != MOE_SOFTMAX && r->score != MOE_SIGMOID) return MOE_ERR_DTYPE;
    if (r->T < 1 || r->k < 1 || r->k > ROUTER_MAX_K || r->E < r->k || r->E > 256) return MOE_ERR_SHAPE;
    if ((int64_t)r->T * r->k >= (1 << 30)) return MOE_ERR_SHAPE;
    if (r->n_groups < 1 || r->n_groups > 64 || r->E % r->n_groups) return MOE_ERR_SHAPE;
    const int group = r->E / r->n_groups;
    if (r->top_groups < 1 || r->top_groups > r->n_groups || r->group_best < 1 || r->group_best > 2) return MOE_ERR_SHAPE;
    if (r->group_best > group || r->top_groups * group < r->k) return MOE_ERR_SHAPE;
    return isfinite(r->scale) ? MOE_OK : MOE_ERR_SHAPE;
}

static int log2_up(int n) {
    int b = 0;
    while ((1 << b) < n) ++b;
    return b;
}

int router_fwd_check(const moe_router* r, const float* logits, const int32_t* expert_idx, const float* gate_w) {
    const int rc = router_status(r);
    return rc ? rc : logits && expert_idx && gate_w ? MOE_OK : MOE_ERR_NULL;
}

extern "C" int moe_router_fwd(const moe_router* router, const float* logits, const float* select_bias_or_null,
                              const uint8_t* token_mask_or_null, int32_t* expert_idx, float* gate_w, void* stream) {
    const int rc = begin_call(router_fwd_check(router, logits, expert_idx, gate_w));
    if (rc) return rc;
    const moe_router& r = *router;
    RouterArgs a = {r.T, r.E, r.k, r.score, r.n_groups, r.E / r.n_groups, r.top_groups, r.group_best, r.renormalise != 0,
                    r.scale, 0, 0};
    // four experts per lane where the groups' lanes, rounded up to powers of two, then fit in a wave; else eight, which
    // always do (a group of S > 8 experts takes fewer than S / 4 lanes)
    int Q = 4;
    for (;; Q = 8) {
        a.lg_log2 = log2_up(ceil_div(a.group, Q));
        a.lpt_log2 = a.lg_log2 + log2_up(a.n_groups);
        if (a.lpt_log2 <= 6 || Q == 8) break;
    }
    const int grid = ceil_div(r.T, 256 >> a.lpt_log2);
    hipStream_t st = (hipStream_t)stream;
#define FWD(Q, V) router_fwd_kernel<Q, V><<<grid, 256, 0, st>>>(a, logits, select_bias_or_null, token_mask_or_null, expert_idx, gate_w)
    if (Q == 4) { if (select_bias_or_null) FWD(4, double); else FWD(4, float); }
    else { if (select_bias_or_null) FWD(8, double); else FWD(8, float); }
#undef FWD
    return launch_status();
}

extern "C" int moe_router_bwd(const moe_router* router, const float* logits, const int32_t* expert_idx,
                              const float* dgate_w, float* dlogits, void* stream) {
    const int rc = begin_call(router_status(router));
    if (rc) return rc;
    if (!logits || !expert_idx || !dgate_w || !dlogits) return MOE_ERR_NULL;
    const moe_router& r = *router;
    const RouterArgs a = {r.T, r.E, r.k, r.score, r.n_groups, r.E / r.n_groups, r.top_groups, r.group_best, r.renormalise != 0,
                          r.scale, 0, 0};
    router_bwd_kernel<<<ceil_div(r.T, 4), 256, 0, (hipStream_t)stream>>>(a, logits, expert_idx, dgate_w, dlogits);
    return launch_status();
}

// ---------------------------------------------------------------------------
// rows of the choices: a stable counting sort
// ---------------------------------------------------------------------------
#define SORT_CHUNK 1024     // choices per workgroup

struct SortWs {
    int32_t* hist;          // [chunks][E] choices per chunk, then those of the chunks before
    int32_t* total;         // [E]
};
static inline int sort_chunks(const moe_router* r) { return ceil_div(r->T * r->k, SORT_CHUNK); }
size_t sort_ws_bytes(const moe_router* r) {
    return align_up((size_t)sort_chunks(r) * r->E * 4, 256) + align_up((size_t)r->E * 4, 256);
}

__global__ __launch_bounds__(SORT_CHUNK) void sort_count_kernel(int n, int E, const int32_t* __restrict__ expert_idx,
                                                                int32_t* __restrict__ hist) {
    __shared__ int s_n[256];
    if (threadIdx.x < 256) s_n[threadIdx.x] = 0;
    __syncthreads();
    const int i = blockIdx.x * SORT_CHUNK + threadIdx.x;
    const int e = i < n ? expert_idx[i] : -1;
    if ((unsigned)e < (unsigned)E) atomicAdd(&s_n[e], 1);
    __syncthreads();
    if (threadIdx.x < E) hist[(size_t)blockIdx.x * E + threadIdx.x] = s_n[threadIdx.x];
}

__device__ __forceinline__ int scan_up(int v, int lane) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(v, o, MOE_WAVE);
        if (lane >= o) v += u;
    }
    return v;
}

// one wave per expert: running sums over the chunks
__global__ __launch_bounds__(64) void sort_scan_kernel(int chunks, int E, int32_t* __restrict__ hist, int32_t* __restrict__ total) {
    const int e = blockIdx.x, lane = threadIdx.x;
    int run = 0;
    for (int c0 = 0; c0 < chunks; c0 += 64) {
        const int c = c0 + lane;
        const int n = c < chunks ? hist[(size_t)c * E + e] : 0;
        const int incl = scan_up(n, lane);
        if (c < chunks) hist[(size_t)c * E + e] = run + incl - n;
        run += __shfl(incl, 63, MOE_WAVE);
    }
    if (lane == 0) total[e] = run;
}

__global__ __launch_bounds__(SORT_CHUNK) void sort_place_kernel(int n, int E, const int32_t* __restrict__ expert_idx,
                                                                const int32_t* __restrict__ hist,
                                                                const int32_t* __restrict__ total,
                                                                int32_t* __restrict__ row_of,
                                                                int32_t* __restrict__ expert_start) {
    constexpr int WAVES = SORT_CHUNK / 64;
    __shared__ int s_base[256];                 // first row of this chunk's choices of an expert
    __shared__ int16_t s_cnt[WAVES][256];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int i = blockIdx.x * SORT_CHUNK + threadIdx.x;
    const int e = i < n ? expert_idx[i] : -1;
    const bool ok = (unsigned)e < (unsigned)E;
    for (int x = threadIdx.x; x < WAVES * 256 / 2; x += SORT_CHUNK) reinterpret_cast<int*>(s_cnt)[x] = 0;
    if (wave == 0) {                            // four experts per lane
        int v[4], sum = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            v[q] = 4 * lane + q < E ? total[4 * lane + q] : 0;
            sum += v[q];
        }
        int run = scan_up(sum, lane) - sum;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int x = 4 * lane + q;
            if (x < E) {
                s_base[x] = run + hist[(size_t)blockIdx.x * E + x];
                if (blockIdx.x == 0) expert_start[x] = run;
            }
            run += v[q];
            if (blockIdx.x == 0 && x == E - 1) expert_start[E] = run;
        }
    }
    __syncthreads();
    // the lanes of this wave with the same expert
    unsigned long long same = __ballot(ok);
#pragma unroll
    for (int b = 0; b < 8; ++b) {
        const bool bit = e >> b & 1;
        const unsigned long long m = __ballot(ok && bit);
        same &= bit ? m : ~m;
    }
    const int rank = __popcll(same & ((1ull << lane) - 1ull));
    if (ok && rank == 0) s_cnt[wave][e] = (int16_t)__popcll(same);
    __syncthreads();
    if (i >= n) return;
    int row = -1;
    if (ok) {
        row = s_base[e] + rank;
        for (int w = 0; w < wave; ++w) row += s_cnt[w][e];
    }
    row_of[i] = row;
}

int sort_check(const moe_router* r, const int32_t* expert_idx, const int32_t* row_of, const int32_t* expert_start,
               const void* ws, size_t ws_bytes) {
    const int rc = router_status(r);
    if (rc) return rc;
    if (!expert_idx || !row_of || !expert_start) return MOE_ERR_NULL;
    return ws_ok(ws, ws_bytes, sort_ws_bytes(r)) ? MOE_OK : MOE_ERR_WORKSPACE;
}

extern "C" size_t moe_sort_workspace_bytes(const moe_router* router) {
    return router_status(router) == MOE_OK ? sort_ws_bytes(router) : 0;
}

extern "C" int moe_sort_choices(const moe_router* router, const int32_t* expert_idx, int32_t* row_of,
                                int32_t* expert_start, void* ws, size_t ws_bytes, void* stream) {
    const int rc = begin_call(sort_check(router, expert_idx, row_of, expert_start, ws, ws_bytes));
    if (rc) return rc;
    const int n = router->T * router->k, E = router->E, chunks = sort_chunks(router);
    int32_t* hist = (int32_t*)ws;
    int32_t* total = (int32_t*)((char*)ws + align_up((size_t)chunks * E * 4, 256));
    hipStream_t st = (hipStream_t)stream;
    sort_count_kernel<<<chunks, SORT_CHUNK, 0, st>>>(n, E, expert_idx, hist);
    sort_scan_kernel<<<E, 64, 0, st>>>(chunks, E, hist, total);
    sort_place_kernel<<<chunks, SORT_CHUNK, 0, st>>>(n, E, expert_idx, hist, total, row_of, expert_start);
    return launch_status();
}

__global__ __launch_bounds__(256) void router_bias_kernel(int E, const int32_t* __restrict__ start, float rate,
                                                          float* __restrict__ bias) {
    const int e = threadIdx.x;
    if (e >= E) return;
    const long long mine = (long long)(start[e + 1] - start[e]) * E, mean = start[E];
    if (mine != mean) bias[e] += mine < mean ? rate : -rate;
}

extern "C" int moe_router_bias_update(const moe_router* router, const int32_t* expert_start, float rate,
                                      float* select_bias, void* stream) {
    const int rc = begin_call(router_status(router));
    if (rc) return rc;
    if (!expert_start || !select_bias) return MOE_ERR_NULL;
    if (!isfinite(rate)) return MOE_ERR_SHAPE;
    router_bias_kernel<<<1, 256, 0, (hipStream_t)stream>>>(router->E, expert_start, rate, select_bias);
    return launch_status();
}

// ---------------------------------------------------------------------------
// mixture of a token's rows: one wave per token, 16-byte vectors
// ---------------------------------------------------------------------------
// 8 entries of a row of yd
__device__ __forceinline__ void row8(const bf16_t* p, float (&v)[8]) { Chunk<bf16_t>::load(p, v); }
__device__ __forceinline__ void row8(const float* p, float (&v)[8]) {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}

template <typename T>
__global__ __launch_bounds__(256) void combine_rows_kernel(int Tn, int d, int k, int R, const T* __restrict__ yd,
                                                           const int32_t* __restrict__ row_of,
                                                           const float* __restrict__ gate_w, bf16_t* __restrict__ y) {
    const int lane = threadIdx.x & 63, t = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (t >= Tn) return;
    int row[ROUTER_MAX_K];
    float w[ROUTER_MAX_K];
#pragma unroll
    for (int j = 0; j < ROUTER_MAX_K; ++j) {
        const int r = j < k ? row_of[(size_t)t * k + j] : -1;
        row[j] = (unsigned)r < (unsigned)R ? r : -1;
        w[j] = row[j] >= 0 ? gate_w[(size_t)t * k + j] : 0.0f;
    }
    for (int v = lane; v < d / 8; v += 64) {
        float acc[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] = 0.0f;
#pragma unroll
        for (int j = 0; j < ROUTER_MAX_K; ++j) {
            if (row[j] < 0) continue;
            float b[8];
            row8(yd + (size_t)row[j] * d + (size_t)v * 8, b);
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[i] = fmaf(w[j], b[i], acc[i]);
        }
        Chunk<bf16_t>::store(y + (size_t)t * d + (size_t)v * 8, acc);
    }
}

int combine_rows_check(const moe_fp8_shape* s, int yd_dtype, const void* yd, const int32_t* row_of, const float* gate_w,
                       const void* y) {
    const int rc = fp8_shape_status(s);
    if (rc) return rc;
    if (yd_dtype != MOE_F32 && yd_dtype != MOE_BF16) return MOE_ERR_DTYPE;
    return yd && row_of && gate_w && y ? MOE_OK : MOE_ERR_NULL;
}

extern "C" int moe_combine_rows(const moe_fp8_shape* shape, int32_t yd_dtype, const void* yd, const int32_t* row_of,
                                const float* gate_w, void* y, void* stream) {
    const int rc = begin_call(combine_rows_check(shape, yd_dtype, yd, row_of, gate_w, y));
    if (rc) return rc;
    const int grid = ceil_div(shape->T, 4), R = shape->T * shape->k;
    hipStream_t st = (hipStream_t)stream;
    if (yd_dtype == MOE_BF16)
        combine_rows_kernel<bf16_t><<<grid, 256, 0, st>>>(shape->T, shape->d_model, shape->k, R, (const bf16_t*)yd, row_of, gate_w, (bf16_t*)y);
    else
        combine_rows_kernel<float><<<grid, 256, 0, st>>>(shape->T, shape->d_model, shape->k, R, (const float*)yd, row_of, gate_w, (bf16_t*)y);
    return launch_status();
}
