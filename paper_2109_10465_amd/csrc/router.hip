// moe_router_fwd / moe_router_bwd: choice and weights of 1..8 experts per token out of at most 256,
// within groups of experts; moe_sort_choices: rows of the choices, expert by expert; moe_combine_rows:
// the mixture of such rows.
#include <math.h>
#include "moe_common.h"

#define ROUTER_MAX_K 8
#define ROUTER_TOKENS (1 << 25)  // of a launch: 64 threads for each, and a grid has fewer than 2^32
#define LOGISTIC_ZERO -690.0f    // logits below have a logistic score under 1e-299, which counts as 0 (as exp overflows it does in 64 bits)

// ---------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------
// LPT lanes share a token and hold eight consecutive experts of one group each: group g has the 2^lg_log2 lanes from
// there on, so the order of (lane, entry) is the order of the ids, whatever the groups' size.
//
// The choice is one of values in 64 bits.  It is made on keys of 32 bits, whose last three bits name the lane's entry:
// a lane sorts its eight keys, and a round takes the largest head of the token's lanes, whose owner notes the expert
// and moves on to its next key.  Where two values that matter - a choice and the next one, any two groups - lie nearer
// together than keys and fp32 scores can be off, the wave makes its choices again in 64 bits.  With 256 experts that is about 1 in
// 100 tokens of logistic scores in 8 groups, and more the more pairs of groups there are, most with softmax scores, whose sums
// are small beside the errors allowed for; equal logits are always decided so, and tokens of two or more groups of masked
// experts.  What bounds it is the number of vector instructions: 65536 tokens of 256 experts, top 8, 4 of 8 groups, take 49 us, 37
// without groups and 30 without a bias too; the logits' read takes 14.  Softmax scores without a bias: 8 groups 46, 16 58, 32 93,
// 64 284; two groups masked 118; all logits equal 116.
struct RouterArgs {
    int T, E, k, score, n_groups, group, top_groups, group_best, renormalise;   // group = experts per group
    float scale;
    int lg_log2;                    // lanes per group
    int vec;                        // a lane's experts start on 16 bytes and are eight (backward: are four)
};

__device__ __forceinline__ double score64(double l, bool sigmoid, double top, double total) {
    return sigmoid ? 1.0 / (1.0 + exp(-l)) : exp(l - top) / total;
}

template <typename V> __device__ __forceinline__ bool ahead(V va, int ia, V vb, int ib) {
    return va > vb || (va == vb && ia < ib);
}

#define KEY_DEAD -3.0e38f       // an expert whose logit is -inf or NaN: after every other one (also without a finite value)
#define KEY_OUT -3.3e38f        // one that cannot be chosen
#define KEY_LEAST -2.9e38f      // the least of all others, and a group that has not as many experts as its value needs
#define LEAST64 -1.7976931348623157e308     // the same among 64-bit values, where dead ones are -inf

template <int CTRL> __device__ __forceinline__ float dpp(float v) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), CTRL, 0xf, 0xf, true));
}
// the largest value (sum) of the LPT lanes of a token, in all of them
template <int LPT, typename F> __device__ __forceinline__ float token_reduce(float v, F f) {
    v = f(v, dpp<0xB1>(v));                         // lanes 1 apart, 2 apart
    v = f(v, dpp<0x4E>(v));
    v = f(v, dpp<0x141>(v));                        // halves of eight mirrored, then of sixteen
    if constexpr (LPT >= 16) v = f(v, dpp<0x140>(v));
    if constexpr (LPT >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    if constexpr (LPT >= 64) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    return v;
}
template <int LPT> __device__ __forceinline__ float token_max(float v) { return token_reduce<LPT>(v, [](float a, float b) { return fmaxf(a, b); }); }
template <int LPT> __device__ __forceinline__ float token_sum(float v) { return token_reduce<LPT>(v, [](float a, float b) { return a + b; }); }

// The choices of the wave's tokens in 64 bits, into s_choice.  (The logits are read again: nothing is kept for this.)
template <int LPT, bool BIAS>
__device__ __forceinline__ void choose64(const RouterArgs& a, const float* __restrict__ row, const float* __restrict__ bias,
                                         bool valid, int here, int e0, int g, int sub, int32_t* s_choice) {
    float l[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        l[i] = valid && i < here ? row[e0 + i] : -INFINITY;
        l[i] = l[i] == l[i] ? l[i] : -INFINITY;
    }
    const bool sigmoid = a.score == MOE_SIGMOID;
    const int lg = 1 << a.lg_log2;
    double top = 0.0, total = 1.0;
    if (!sigmoid) {
        float m = l[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) m = fmaxf(m, l[i]);
        m = token_max<LPT>(m);
        top = m == -INFINITY ? 0.0 : (double)m;
        total = 0.0;
#pragma unroll
        for (int i = 0; i < 8; ++i) total += exp((double)l[i] - top);
        for (int o = LPT >> 1; o > 0; o >>= 1) total += __shfl_xor(total, o, MOE_WAVE);
        if (!(total > 0.0)) total = 1.0;
    }
    double v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        v[i] = l[i];
        if constexpr (BIAS) {
            const double w = score64(l[i], sigmoid, top, total) + (i < here ? (double)bias[e0 + i] : 0.0);
            v[i] = l[i] > -INFINITY ? (w > LEAST64 ? w : LEAST64) : -INFINITY;      // (a bias of -inf does not make it a dead one)
        }
    }
    unsigned left = (1u << here) - 1u;          // experts that can still be chosen
    if (a.n_groups > 1) {
        double b0 = -INFINITY, b1 = -INFINITY;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (v[i] > b0) { b1 = b0; b0 = v[i]; } else if (v[i] > b1) b1 = v[i];
        }
        for (int o = lg >> 1; o > 0; o >>= 1) {
            const double c0 = __shfl_xor(b0, o, MOE_WAVE), c1 = __shfl_xor(b1, o, MOE_WAVE);
            const double lo = b0 < c0 ? b0 : c0;
            b0 = b0 < c0 ? c0 : b0;
            b1 = b1 < c1 ? c1 : b1;
            b1 = b1 < lo ? lo : b1;
        }
        double gv = b0;
        if (a.group_best == 2) {
            if constexpr (BIAS) gv = b0 + b1;
            else gv = b1 == -INFINITY ? -INFINITY : score64(b0, sigmoid, top, total) + score64(b1, sigmoid, top, total);
        }
        if (b0 > -INFINITY && !(gv > LEAST64)) gv = LEAST64;    // one expert is more than none
        int before = 0;                         // groups in front of this one
        for (int o = 1; o < LPT >> a.lg_log2; ++o) {
            const double w = __shfl_xor(gv, o << a.lg_log2, MOE_WAVE);
            before += (g ^ o) < a.n_groups && ahead(w, g ^ o, gv, g);
        }
        if (before >= a.top_groups) left = 0;
    }
    for (int j = 0; j < a.k; ++j) {
        double best = -INFINITY;
        int id = 0x7fffffff;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if ((left >> i & 1u) && ahead(v[i], e0 + i, best, id)) { best = v[i]; id = e0 + i; }
        for (int o = LPT >> 1; o > 0; o >>= 1) {
            const double w = __shfl_xor(best, o, MOE_WAVE);
            const int wi = __shfl_xor(id, o, MOE_WAVE);
            if (ahead(w, wi, best, id)) { best = w; id = wi; }
        }
        if (sub == 0) s_choice[j] = id;
        if (id >= e0 && id < e0 + here) left &= ~(1u << (id - e0));
    }
}

template <int LPT, bool BIAS>
__global__ __launch_bounds__(256) void router_fwd_kernel(const RouterArgs a, const float* __restrict__ logits,
                                                         const float* __restrict__ bias, const uint8_t* __restrict__ mask,
                                                         int32_t* __restrict__ expert_idx, float* __restrict__ gate_w) {
    static_assert(LPT >= ROUTER_MAX_K, "a lane for every choice");
    __shared__ int32_t s_all[256 / LPT][ROUTER_MAX_K];
    const int lg = 1 << a.lg_log2;
    const int sub = threadIdx.x & (LPT - 1), t = blockIdx.x * (256 / LPT) + threadIdx.x / LPT;
    const int g = sub >> a.lg_log2, first = (sub & (lg - 1)) * 8, e0 = g * a.group + first;
    const int here = g < a.n_groups ? min(max(a.group - first, 0), 8) : 0;
    const bool in = t < a.T, valid = in && (!mask || mask[t] != 0);
    const bool sigmoid = a.score == MOE_SIGMOID;
    const float* row = logits + (size_t)(in ? t : 0) * a.E;
    int32_t* s_choice = s_all[threadIdx.x / LPT];
    float l[8], b[8];
    if (a.vec) {
        float4 p = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY), q = p;
        if (valid && here) {
            p = *reinterpret_cast<const float4*>(row + e0);
            q = *reinterpret_cast<const float4*>(row + e0 + 4);
        }
        l[0] = p.x; l[1] = p.y; l[2] = p.z; l[3] = p.w; l[4] = q.x; l[5] = q.y; l[6] = q.z; l[7] = q.w;
        p = q = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (BIAS && here) {
            p = *reinterpret_cast<const float4*>(bias + e0);
            q = *reinterpret_cast<const float4*>(bias + e0 + 4);
        }
        b[0] = p.x; b[1] = p.y; b[2] = p.z; b[3] = p.w; b[4] = q.x; b[5] = q.y; b[6] = q.z; b[7] = q.w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            l[i] = valid && i < here ? row[e0 + i] : -INFINITY;
            b[i] = BIAS && i < here ? bias[e0 + i] : 0.0f;
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) l[i] = l[i] == l[i] ? l[i] : -INFINITY;     // a NaN would make the softmax's sum one
    // the softmax's largest logit and sum, where scores are compared or not divided by the chosen ones' sum
    const bool sums = a.n_groups > 1 && a.group_best == 2;
    float top = 0.0f, total = 1.0f;
    if (!sigmoid && (BIAS || sums || !a.renormalise)) {
        top = l[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) top = fmaxf(top, l[i]);
        top = token_max<LPT>(top);
        if (top == -INFINITY) top = 0.0f;
        total = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) total += __expf(l[i] - top);
        total = token_sum<LPT>(total);
        if (!(total > 0.0f)) total = 1.0f;
    }
    const float inv = 1.0f / total;
    auto score = [&](float x) { return sigmoid ? __builtin_amdgcn_rcpf(1.0f + __expf(-x)) : __expf(x - top) * inv; };
    // The keys, sorted (Batcher's network of 19 comparisons).  An entry without an expert has a dead one's key: where such a
    // key is chosen there are others like it, and the choice is made again in 64 bits.
    float key[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float v = BIAS ? score(l[i]) + b[i] : l[i];
        v = __builtin_amdgcn_fmed3f(v, KEY_LEAST, -KEY_LEAST);
        v = l[i] > -INFINITY ? v : KEY_DEAD;
        key[i] = __uint_as_float((__float_as_uint(v) & ~7u) | (uint32_t)i);
    }
    auto order = [&](int i, int j) {
        const float hi = fmaxf(key[i], key[j]), lo = fminf(key[i], key[j]);
        key[i] = hi;
        key[j] = lo;
    };
    order(0, 1); order(2, 3); order(4, 5); order(6, 7);
    order(0, 2); order(1, 3); order(4, 6); order(5, 7);
    order(1, 2); order(5, 6); order(0, 4); order(3, 7);
    order(1, 5); order(2, 6);
    order(1, 4); order(3, 6);
    order(2, 4); order(3, 5);
    order(3, 4);
    // How far apart two choices have to be: a key drops three bits (2^-20 of its size), a score is off by less than 5e-7
    // (exponential, reciprocal and their argument), the sum with the bias by 2^-24: twice that, and a half more.
    auto near = [](float hi, float lo) { return hi - lo <= fmaf(fabsf(hi) + fabsf(lo), 1.6e-6f, 1.6e-6f); };
    bool again = false;
    if (a.n_groups > 1) {
        float b0 = key[0], b1 = key[1];
        for (int o = lg >> 1; o > 0; o >>= 1) {
            const float c0 = __shfl_xor(b0, o, MOE_WAVE), c1 = __shfl_xor(b1, o, MOE_WAVE);
            b1 = fmaxf(fmaxf(b1, c1), fminf(b0, c0));
            b0 = fmaxf(b0, c0);
        }
        float gv = b0;
        const bool dead = b0 < -2.95e38f, whole = a.group_best == 1 ? !dead : !(b1 < -2.95e38f);
        if (a.group_best == 2) gv = whole ? fmaxf(BIAS ? b0 + b1 : score(b0) + score(b1), KEY_LEAST) : dead ? KEY_DEAD : KEY_LEAST;
        if (g >= a.n_groups) gv = KEY_OUT;
        // A group's value is off by its keys' and scores' errors; where a score is made of a key, by that score's share of the
        // logit's (a softmax does not mind how large logits are, a key does).  The token's largest such error, twice, is near.
        float off = fmaf(fabsf(b0) + (a.group_best == 2 ? fabsf(b1) : 0.0f), 1.6e-6f, 1.6e-6f);
        if (!BIAS && a.group_best == 2) off = fmaf(fabsf(b0) + fabsf(b1), gv * 1.6e-6f, 1.6e-6f);
        off = 2.0f * token_max<LPT>(whole ? off : 0.0f);
        int before = 0;
        for (int o = 1; o < LPT >> a.lg_log2; ++o) {
            const float w = __shfl_xor(gv, o << a.lg_log2, MOE_WAVE);
            before += w > gv;
            again |= (g ^ o) < a.n_groups && g < a.n_groups && fabsf(w - gv) <= off;
        }
        if (before >= a.top_groups) {
#pragma unroll
            for (int i = 0; i < 8; ++i) key[i] = KEY_OUT;
        }
    }
    float mine = 0.0f, behind = 0.0f;       // lane j: the j-th choice and the one after it
    // Two lanes can have the same key, which would then both move on, and one choice be lost: a round has one owner per token.
    const unsigned long long live = __ballot(valid);
    const int tokens = __popcll(live) / LPT;
    bool shared = false;
    for (int j = 0; j <= a.k; ++j) {        // one more than are chosen
        const float w = token_max<LPT>(key[0]);
        mine = sub == j ? w : mine;
        behind = sub + 1 == j ? w : behind;
        if (j == a.k) break;
        shared |= __popcll(__ballot(key[0] == w) & live) != tokens;
        if (key[0] == w) {
            s_choice[j] = e0 + (int)(__float_as_uint(w) & 7u);
#pragma unroll
            for (int i = 0; i < 7; ++i) key[i] = key[i + 1];
            key[7] = KEY_OUT;
        }
    }
    again |= sub < a.k && near(mine, behind);
    if (shared || __any(valid && again)) choose64<LPT, BIAS>(a, row, bias, valid, here, e0, g, sub, s_choice);
    __builtin_amdgcn_wave_barrier();
    // the token's choices and weights: lane j has the j-th
    const int id = sub < a.k && valid ? s_choice[sub] : -1;
    const float x = id >= 0 ? row[id] : -INFINITY;
    // renormalised scores, scaled so that the largest is near 1: exp(x - most), or 1 / (e^-M + e^(-x - M)) with M = max(0, -most)
    float s = 0.0f, c = a.scale;
    if (a.renormalise) {
        const float most = token_max<LPT>(x), m = fmaxf(0.0f, -most);
        if (!(x == -INFINITY || (sigmoid && x < LOGISTIC_ZERO)))
            s = sigmoid ? __builtin_amdgcn_rcpf(__expf(-m) + __expf(-x - m)) : __expf(x - most);
        const float sum = token_sum<LPT>(s);
        c = sum == 0.0f ? 0.0f : a.scale * __builtin_amdgcn_rcpf(sum);
    } else if (!(x == -INFINITY || (sigmoid && x < LOGISTIC_ZERO))) {
        s = score(x);
    }
    if (in && sub < a.k) {
        expert_idx[(size_t)t * a.k + sub] = id;
        gate_w[(size_t)t * a.k + sub] = s * c;
    }
}

// ---------------------------------------------------------------------------
// backward: LPT lanes per token, four consecutive experts each; lane j < k works out q_j
// ---------------------------------------------------------------------------
template <int LPT>
__global__ __launch_bounds__(256) void router_bwd_kernel(const RouterArgs a, const float* __restrict__ logits,
                                                         const int32_t* __restrict__ expert_idx,
                                                         const float* __restrict__ dgate_w, float* __restrict__ dlogits) {
    const int lane = threadIdx.x & 63, sub = threadIdx.x & (LPT - 1), base = lane & ~(LPT - 1);
    const int t = blockIdx.x * (256 / LPT) + threadIdx.x / LPT, e4 = 4 * sub;
    const bool in = t < a.T, sigmoid = a.score == MOE_SIGMOID;
    const float* row = logits + (size_t)(in ? t : 0) * a.E;
    int id = in && sub < a.k ? expert_idx[(size_t)t * a.k + sub] : -1;
    if ((unsigned)id >= (unsigned)a.E) id = -1;
    float x = -INFINITY, dw = 0.0f;
    if (id >= 0) {
        x = row[id];
        dw = dgate_w[(size_t)t * a.k + sub];
    }
    float out[4] = {0.0f, 0.0f, 0.0f, 0.0f}, l[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    const bool dense = !sigmoid && !a.renormalise;    // (the renormalised softmax's q sum to 0)
    const bool none = x == -INFINITY || (sigmoid && x < LOGISTIC_ZERO);
    float r = 0.0f, top = 0.0f, inv = 1.0f, mean = 0.0f;
    if (dense) {
        if (in) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (e4 + i < a.E) l[i] = row[e4 + i];
                l[i] = l[i] == l[i] ? l[i] : -INFINITY;     // as the forward pass takes it
            }
        }
        top = token_max<LPT>(fmaxf(fmaxf(l[0], l[1]), fmaxf(l[2], l[3])));
        if (top == -INFINITY) top = 0.0f;
        float total = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) total += __expf(l[i] - top);
        total = token_sum<LPT>(total);
        inv = total > 0.0f ? 1.0f / total : 0.0f;
        if (!none) r = __expf(x - top) * inv;
    } else if (a.renormalise) {
        const float most = token_max<LPT>(x), m = fmaxf(0.0f, -most);
        if (!none) r = sigmoid ? __builtin_amdgcn_rcpf(__expf(-m) + __expf(-x - m)) : __expf(x - most);
        const float sum = token_sum<LPT>(r);
        r *= sum > 0.0f ? __builtin_amdgcn_rcpf(sum) : 0.0f;
        mean = token_sum<LPT>(dw * r);
    } else if (!none) {
        r = __builtin_amdgcn_rcpf(1.0f + __expf(-x));
    }
    float q = none ? 0.0f : a.scale * r * (dw - mean);
    const float all = dense ? token_sum<LPT>(q) : 0.0f;
    if (sigmoid && !none) q *= __builtin_amdgcn_rcpf(1.0f + __expf(x));
    for (int j = 0; j < a.k; ++j) {
        const int ij = __shfl(id, base + j, MOE_WAVE) - e4;
        const float qj = __shfl(q, base + j, MOE_WAVE);
#pragma unroll
        for (int i = 0; i < 4; ++i) out[i] += ij == i ? qj : 0.0f;
    }
    if (dense && all != 0.0f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) out[i] -= __expf(l[i] - top) * inv * all;
    }
    if (!in) return;
    float* o = dlogits + (size_t)t * a.E;
    if (a.vec) {
        if (e4 < a.E) *reinterpret_cast<float4*>(o + e4) = make_float4(out[0], out[1], out[2], out[3]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (e4 + i < a.E) o[e4 + i] = out[i];
    }
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
    // the groups' lanes, rounded up to powers of two, always fit in a wave: of at most 256 experts, a group of S > 8 has fewer
    // than S / 4 lanes
    a.lg_log2 = log2_up(ceil_div(a.group, 8));
    a.vec = a.group % 8 == 0 && (((uintptr_t)logits | (uintptr_t)select_bias_or_null) & 15) == 0;
    const int lanes = a.lg_log2 + log2_up(r.n_groups);
    hipStream_t st = (hipStream_t)stream;
    for (int t = 0; t < r.T; t += ROUTER_TOKENS) {
        a.T = r.T - t < ROUTER_TOKENS ? r.T - t : ROUTER_TOKENS;
        const float* l = logits + (size_t)t * r.E;
        const uint8_t* m = token_mask_or_null ? token_mask_or_null + t : nullptr;
        int32_t* id = expert_idx + (size_t)t * r.k;
        float* w = gate_w + (size_t)t * r.k;
#define FWD(LPT) (select_bias_or_null ? router_fwd_kernel<LPT, true> : router_fwd_kernel<LPT, false>)<<<ceil_div(a.T, 256 / LPT), 256, 0, st>>>( \
    a, l, select_bias_or_null, m, id, w)
        if (lanes <= 3) FWD(8); else if (lanes == 4) FWD(16); else if (lanes == 5) FWD(32); else FWD(64);
#undef FWD
    }
    return launch_status();
}

extern "C" int moe_router_bwd(const moe_router* router, const float* logits, const int32_t* expert_idx,
                              const float* dgate_w, float* dlogits, void* stream) {
    const int rc = begin_call(router_status(router));
    if (rc) return rc;
    if (!logits || !expert_idx || !dgate_w || !dlogits) return MOE_ERR_NULL;
    const moe_router& r = *router;
    RouterArgs a = {r.T, r.E, r.k, r.score, r.n_groups, r.E / r.n_groups, r.top_groups, r.group_best, r.renormalise != 0,
                    r.scale, 0, 0};
    a.vec = r.E % 4 == 0 && ((uintptr_t)dlogits & 15) == 0;
    const int lanes = log2_up(ceil_div(r.E, 4));
    hipStream_t st = (hipStream_t)stream;
    for (int t = 0; t < r.T; t += ROUTER_TOKENS) {
        a.T = r.T - t < ROUTER_TOKENS ? r.T - t : ROUTER_TOKENS;
        const size_t l = (size_t)t * r.E, c = (size_t)t * r.k;
#define BWD(LPT) router_bwd_kernel<LPT><<<ceil_div(a.T, 256 / LPT), 256, 0, st>>>(a, logits + l, expert_idx + c, dgate_w + c, dlogits + l)
        if (lanes <= 3) BWD(8); else if (lanes == 4) BWD(16); else if (lanes == 5) BWD(32); else BWD(64);
#undef BWD
    }
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

// All of it in one workgroup, for few choices: three dependent launches of which none has work for the chip.  The choices
// are counted, then placed in rounds of one per thread.
#define SORT_SMALL 8192
__global__ __launch_bounds__(SORT_CHUNK) void sort_small_kernel(int n, int E, const int32_t* __restrict__ expert_idx,
                                                                int32_t* __restrict__ row_of,
                                                                int32_t* __restrict__ expert_start) {
    constexpr int WAVES = SORT_CHUNK / 64, ROUNDS = SORT_SMALL / SORT_CHUNK;
    __shared__ int s_next[256];                 // the next choice's row of an expert
    __shared__ int16_t s_cnt[WAVES][256];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int e[ROUNDS];
    if (threadIdx.x < 256) s_next[threadIdx.x] = 0;
    for (int x = threadIdx.x; x < WAVES * 256 / 2; x += SORT_CHUNK) reinterpret_cast<int*>(s_cnt)[x] = 0;
#pragma unroll
    for (int u = 0; u < ROUNDS; ++u) {
        const int i = u * SORT_CHUNK + threadIdx.x;
        e[u] = i < n ? expert_idx[i] : -1;
        if ((unsigned)e[u] >= (unsigned)E) e[u] = -1;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < ROUNDS; ++u)
        if (e[u] >= 0) atomicAdd(&s_next[e[u]], 1);
    __syncthreads();
    if (wave == 0) {                            // four experts per lane
        int v[4], sum = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            v[q] = s_next[4 * lane + q];
            sum += v[q];
        }
        int run = scan_up(sum, lane) - sum;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int x = 4 * lane + q;
            s_next[x] = run;
            if (x < E) expert_start[x] = run;
            run += v[q];
            if (x == E - 1) expert_start[E] = run;
        }
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < ROUNDS; ++u) {
        if (u * SORT_CHUNK >= n) break;         // uniform
        const int i = u * SORT_CHUNK + threadIdx.x;
        const bool ok = e[u] >= 0;
        unsigned long long same = __ballot(ok);
#pragma unroll
        for (int b = 0; b < 8; ++b) {
            const bool bit = e[u] >> b & 1;
            const unsigned long long m = __ballot(ok && bit);
            same &= bit ? m : ~m;
        }
        const int rank = __popcll(same & ((1ull << lane) - 1ull));
        if (ok && rank == 0) s_cnt[wave][e[u]] = (int16_t)__popcll(same);
        __syncthreads();
        int row = -1;
        if (ok) {
            row = s_next[e[u]] + rank;
            for (int w = 0; w < wave; ++w) row += s_cnt[w][e[u]];
        }
        if (i < n) row_of[i] = row;
        if ((u + 1) * SORT_CHUNK >= n) break;   // uniform
        __syncthreads();
        if (threadIdx.x < 256) {                // the round's counts move on, and are cleared
            int sum = 0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                sum += s_cnt[w][threadIdx.x];
                s_cnt[w][threadIdx.x] = 0;
            }
            s_next[threadIdx.x] += sum;
        }
        __syncthreads();
    }
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
    if (n <= SORT_SMALL) {
        sort_small_kernel<<<1, SORT_CHUNK, 0, st>>>(n, E, expert_idx, row_of, expert_start);
        return launch_status();
    }
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
    const int lane = threadIdx.x & 63;
    for (int t = blockIdx.x * 4 + (threadIdx.x >> 6); t < Tn; t += gridDim.x * 4) {
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
}

int combine_rows_check(const moe_fp8_shape* s, int yd_dtype, const void* yd, const int32_t* row_of, const float* gate_w,
                       const void* y) {
    const int rc = fp8_shape_status(s);
    if (rc) return rc;
    if (yd_dtype != MOE_F32 && yd_dtype != MOE_BF16) return MOE_ERR_DTYPE;
    return !(yd && row_of && gate_w && y) ? MOE_ERR_NULL : aligned(16, yd, y) ? MOE_OK : MOE_ERR_SHAPE;
}

extern "C" int moe_combine_rows(const moe_fp8_shape* shape, int32_t yd_dtype, const void* yd, const int32_t* row_of,
                                const float* gate_w, void* y, void* stream) {
    const int rc = begin_call(combine_rows_check(shape, yd_dtype, yd, row_of, gate_w, y));
    if (rc) return rc;
    const int tokens = ceil_div(shape->T, 4), grid = tokens < ROUTER_TOKENS / 4 ? tokens : ROUTER_TOKENS / 4, R = shape->T * shape->k;
    hipStream_t st = (hipStream_t)stream;
    if (yd_dtype == MOE_BF16)
        combine_rows_kernel<bf16_t><<<grid, 256, 0, st>>>(shape->T, shape->d_model, shape->k, R, (const bf16_t*)yd, row_of, gate_w, (bf16_t*)y);
    else
        combine_rows_kernel<float><<<grid, 256, 0, st>>>(shape->T, shape->d_model, shape->k, R, (const float*)yd, row_of, gate_w, (bf16_t*)y);
    return launch_status();
}
