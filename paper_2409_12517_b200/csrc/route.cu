// Expert routing: scores, choice of the experts (groups, bias, top-k), their weights; its gradient; the balance bias.
//
// One token is a row of n_experts logits.  LANES lanes of a warp own it, lane l the V neighbouring experts from l * V, so
// a row is read once into registers and everything up to the weights happens there: the softmax's maximum and sum, the
// groups' values and the choice are reductions over the token's lanes.  Short rows share a warp (32 / LANES tokens).
#include <math_constants.h>

#include "common.cuh"

namespace fp8mlp {

namespace {

constexpr int kRouteThreads = 128;
constexpr uint32_t kAll = 0xffffffffu;

struct RouteArgs {
    const void* logits; const float* bias; int32_t* experts; float* weights;
    const float* d_weights; void* d_logits;
    int64_t T, ld, ld_d;
    int E, k, score, G, per, top_groups, group_top, renorm;
    float scale;
    int wide, wide_b, wide_d;      // rows of logits, the bias, rows of d_logits start on a vector boundary
    int lane_groups;       // a group is a power-of-two number of whole lanes
};

template <typename SRC> __device__ __forceinline__ float load1(const SRC* p);
template <> __device__ __forceinline__ float load1<float>(const float* p) { return __ldg(p); }
template <> __device__ __forceinline__ float load1<uint16_t>(const uint16_t* p) { return __uint_as_float(static_cast<uint32_t>(__ldg(p)) << 16); }

// 8 neighbouring elements on a vector boundary (32 bytes fp32, 16 bytes bf16)
template <typename SRC> __device__ __forceinline__ void load8(const SRC* p, float* v);
template <> __device__ __forceinline__ void load8<float>(const float* p, float* v) {
    uint32_t w[8];
    ld_global_nc_v8(p, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
}
template <> __device__ __forceinline__ void load8<uint16_t>(const uint16_t* p, float* v) {
    const uint4 w = ld_global_nc_v4(p);
    v[0] = bf16_lo(w.x); v[1] = bf16_hi(w.x); v[2] = bf16_lo(w.y); v[3] = bf16_hi(w.y);
    v[4] = bf16_lo(w.z); v[5] = bf16_hi(w.z); v[6] = bf16_lo(w.w); v[7] = bf16_hi(w.w);
}
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(uint16_t* p, float v) { *p = static_cast<uint16_t>(cvt_bf16x2(v, 0.0f) & 0xffffu); }
__device__ __forceinline__ void store8(float* p, const float* v) {
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(v[i]);
    st_global_v8(p, w);
}
__device__ __forceinline__ void store8(uint16_t* p, const float* v) {
    st_global_v4(p, cvt_bf16x2(v[0], v[1]), cvt_bf16x2(v[2], v[3]), cvt_bf16x2(v[4], v[5]), cvt_bf16x2(v[6], v[7]));
}

// this lane's V logits of one row; experts beyond E read as -inf
template <int V, typename SRC>
__device__ __forceinline__ void load_row(const SRC* row, int e0, int E, bool wide, float (&x)[V]) {
#pragma unroll
    for (int b = 0; b < V; b += 8) {
        if (wide && e0 + b + 8 <= E) {
            load8<SRC>(row + e0 + b, &x[b]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[b + i] = e0 + b + i < E ? load1<SRC>(row + e0 + b + i) : -CUDART_INF_F;
        }
    }
}

// Unsigned key that orders like the float; 0 (no float's key) stands for "cannot be chosen".
__device__ __forceinline__ uint32_t order_key(float c) {
    const uint32_t u = __float_as_uint(c);
    return u ^ ((static_cast<uint32_t>(static_cast<int32_t>(u) >> 31)) | 0x80000000u);
}

template <int LANES> __device__ __forceinline__ uint32_t seg_max(uint32_t v) {
    if constexpr (LANES == 32) {
        return __reduce_max_sync(kAll, v);
    } else {
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(kAll, v, o));
        return v;
    }
}
template <int LANES> __device__ __forceinline__ float seg_sum(float v) {
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
    return v;
}
template <int LANES> __device__ __forceinline__ float seg_maxf(float v) {
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(kAll, v, o));
    return v;
}

// sigma(x) = 1 / (1 + e^-x), written with e^-|x| so that neither end overflows and small values keep their digits; the
// reciprocal is of a number in [1, 2], where the special-function unit's is within one unit of the last place.
__device__ __forceinline__ float sigmoid_exact(float x) {
    const float e = expf(-fabsf(x));
    const float r = rcp_approx(1.0f + e);
    return x >= 0.0f ? r : e * r;          // NaN takes the second branch and stays NaN
}
// 1 - sigma(x) = sigma(-x)

// softmax of the token's row, in place; a row without a finite maximum comes out as NaN
template <int LANES, int V>
__device__ __forceinline__ void softmax_row(float (&x)[V]) {
    float m = x[0];
#pragma unroll
    for (int j = 1; j < V; ++j) m = fmaxf(m, x[j]);
    m = seg_maxf<LANES>(m);
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < V; ++j) { x[j] = expf(x[j] - m); sum += x[j]; }
    sum = seg_sum<LANES>(sum);
    const float inv = __fdiv_rn(1.0f, sum);
#pragma unroll
    for (int j = 0; j < V; ++j) x[j] *= inv;
}

// the larger two of (a1 >= a2) and (b1 >= b2)
__device__ __forceinline__ void merge_top2(uint32_t& a1, uint32_t& a2, uint32_t b1, uint32_t b2) {
    a2 = max(min(a1, b1), max(a2, b2));
    a1 = max(a1, b1);
}
__device__ __forceinline__ float key_value(uint32_t k) {      // the float of a key; a missing expert adds nothing
    return k == 0u ? 0.0f : __uint_as_float(k ^ ((k & 0x80000000u) ? 0x80000000u : 0xffffffffu));
}
// a group's value as a key (0: nothing to choose in it)
__device__ __forceinline__ uint32_t group_key(uint32_t k1, uint32_t k2, int group_top) {
    if (k1 == 0u) return 0u;
    const float v = group_top == 2 ? key_value(k1) + key_value(k2) : key_value(k1);
    return order_key(v + 0.0f);            // + 0: one zero only
}

// 8 keys into falling order (19 exchanges)
__device__ __forceinline__ void exchange(uint32_t& a, uint32_t& b) {
    const uint32_t hi = max(a, b);
    b = min(a, b);
    a = hi;
}
__device__ __forceinline__ void sort8(uint32_t (&k)[8]) {
    exchange(k[0], k[2]); exchange(k[1], k[3]); exchange(k[4], k[6]); exchange(k[5], k[7]);
    exchange(k[0], k[4]); exchange(k[1], k[5]); exchange(k[2], k[6]); exchange(k[3], k[7]);
    exchange(k[0], k[1]); exchange(k[2], k[3]); exchange(k[4], k[5]); exchange(k[6], k[7]);
    exchange(k[2], k[4]); exchange(k[3], k[5]);
    exchange(k[1], k[4]); exchange(k[3], k[6]);
    exchange(k[1], k[2]); exchange(k[3], k[4]); exchange(k[5], k[6]);
}

// The choice: every lane sorts its keys, eight at a time, and the token's lanes take the largest head k times.  What a
// round costs decides the kernel's time (it is bound by instructions, not by memory), so a round moves keys only; which
// expert a key belongs to is looked up once at the end, by k lanes side by side, in the unsorted keys in shared memory.
template <int LANES, int V, typename SRC>
__global__ void __launch_bounds__(kRouteThreads) route_kernel(const RouteArgs a) {
    extern __shared__ __align__(16) uint32_t smem[];
    constexpr int kTokens = kRouteThreads / LANES;
    constexpr int kRow = LANES * V + 4;                   // + 4: rows of neighbouring tokens start in other banks
    constexpr int kLists = V / 8;
    const int lane = threadIdx.x % LANES, tok = threadIdx.x / LANES;
    const int seg_base = (threadIdx.x & 31) - lane;
    uint32_t* row_key = smem + tok * kRow;                                          // this token's keys ...
    float* row_s = reinterpret_cast<float*>(smem + kTokens * kRow) + tok * kRow;    // ... and scores
    uint32_t* sel_key = smem + 2 * kTokens * kRow + 2 * tok * a.k;                  // a round's key, then its lane and count
    uint32_t* group_keys = smem + 2 * kTokens * (kRow + a.k) + tok * a.G;
    const int64_t t = static_cast<int64_t>(blockIdx.x) * kTokens + tok;
    const bool live = t < a.T;
    const int e0 = lane * V;
    grid_dependency_wait();
    grid_launch_dependents();

    float s[V];
    uint32_t key[kLists][8];
    if (live) {
        load_row<V, SRC>(static_cast<const SRC*>(a.logits) + t * a.ld, e0, a.E, a.wide != 0, s);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) s[j] = -CUDART_INF_F;
    }
    uint32_t masked = 0;
#pragma unroll
    for (int j = 0; j < V; ++j) masked |= (s[j] == -CUDART_INF_F ? 1u : 0u) << j;
    if (a.score == FP8MLP_SCORE_SOFTMAX) {
        softmax_row<LANES, V>(s);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) s[j] = sigmoid_exact(s[j]);
    }
    if (a.bias != nullptr) {
        float b[V];
        load_row<V, float>(a.bias, e0, a.E, a.wide_b != 0, b);      // past the last expert: -inf
#pragma unroll
        for (int j = 0; j < V; ++j) {
            row_s[e0 + j] = s[j];
            s[j] += b[j];
        }
    }
#pragma unroll
    for (int j = 0; j < V; ++j) key[j / 8][j % 8] = (masked >> j & 1u) != 0u || !(s[j] > -CUDART_INF_F) ? 0u : order_key(s[j]);

    if (a.G > 1 && !a.lane_groups) {                      // groups that do not fall on lanes: through shared memory
#pragma unroll
        for (int j = 0; j < V; ++j) row_key[e0 + j] = key[j / 8][j % 8];
        __syncwarp();
        for (int g = lane; g < a.G; g += LANES) {
            uint32_t k1 = 0, k2 = 0;
            for (int i = 0; i < a.per; ++i) {
                const uint32_t v = row_key[g * a.per + i];
                k2 = max(k2, min(k1, v));
                k1 = max(k1, v);
            }
            group_keys[g] = group_key(k1, k2, a.group_top);
        }
        __syncwarp();
        int last = -1;
        bool keep = false;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int g = (e0 + j) / a.per;
            if (g != last && e0 + j < a.E) {
                last = g;
                const uint32_t gk = group_keys[g];
                int rank = 0;
                for (int i = 0; i < a.G; ++i) {
                    const uint32_t other = group_keys[i];
                    rank += (other > gk || (other == gk && i < g)) ? 1 : 0;
                }
                keep = rank < a.top_groups;
            }
            if (!keep) key[j / 8][j % 8] = 0u;
        }
    }
#pragma unroll
    for (int j = 0; j < V; j += 4)
        *reinterpret_cast<uint4*>(row_key + e0 + j) = make_uint4(key[j / 8][j % 8], key[j / 8][j % 8 + 1], key[j / 8][j % 8 + 2], key[j / 8][j % 8 + 3]);
#pragma unroll
    for (int l = 0; l < kLists; ++l) sort8(key[l]);

    if (a.G > 1 && a.lane_groups) {
        const int width = a.per / V;                     // lanes of a group
        uint32_t k1 = key[0][0], k2 = key[0][1];
#pragma unroll
        for (int l = 1; l < kLists; ++l) merge_top2(k1, k2, key[l][0], key[l][1]);
        for (int o = 1; o < width; o <<= 1) {
            const uint32_t b1 = __shfl_xor_sync(kAll, k1, o), b2 = __shfl_xor_sync(kAll, k2, o);
            merge_top2(k1, k2, b1, b2);
        }
        const uint32_t gk = group_key(k1, k2, a.group_top);
        const int mine = lane / width;
        int rank = 0;
        for (int g = 0; g < a.G; ++g) {
            const uint32_t other = __shfl_sync(kAll, gk, seg_base + g * width);
            rank += (other > gk || (other == gk && g < mine)) ? 1 : 0;
        }
        if (rank >= a.top_groups) {
#pragma unroll
            for (int l = 0; l < kLists; ++l)
#pragma unroll
                for (int j = 0; j < 8; ++j) key[l][j] = 0u;
        }
    }

    uint32_t best = key[0][0];
#pragma unroll
    for (int l = 1; l < kLists; ++l) best = max(best, key[l][0]);
    uint32_t prev = 0, count = 0;
    for (int r = 0; r < a.k; ++r) {
        const uint32_t top = seg_max<LANES>(best);
        // the lowest lane among equals holds the lowest expert; how often it gave this key before tells which of its equals
        const uint32_t holders = (__ballot_sync(kAll, best == top) >> seg_base) & (LANES == 32 ? kAll : (1u << (LANES & 31)) - 1u);
        if (lane == __ffs(holders) - 1) {
            count = top == prev ? count + 1u : 0u;
            prev = top;
            sel_key[2 * r] = top;
            sel_key[2 * r + 1] = static_cast<uint32_t>(lane) | count << 8;
            bool taken = false;
            best = 0;
#pragma unroll
            for (int l = 0; l < kLists; ++l) {
                if (!taken && key[l][0] == top) {
                    taken = true;
#pragma unroll
                    for (int j = 0; j < 7; ++j) key[l][j] = key[l][j + 1];
                    key[l][7] = 0u;
                }
                best = max(best, key[l][0]);
            }
        }
    }
    __syncwarp();
    float D = 0.0f;
    constexpr int kMine = LANES >= 4 ? (FP8MLP_MAX_TOP_K + LANES - 1) / LANES : 8;      // k <= LANES * 8 where LANES < 4
    float score[kMine];
    int32_t expert[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int r = lane + i * LANES;
        score[i] = 0.0f;
        expert[i] = -1;
        if (r < a.k && sel_key[2 * r] != 0u) {
            const uint32_t want = sel_key[2 * r], who = sel_key[2 * r + 1];
            const int from = static_cast<int>(who & 255u) * V;
            uint32_t skip = who >> 8;
#pragma unroll
            for (int j = 0; j < V; j += 4) {
                const uint4 q = *reinterpret_cast<const uint4*>(row_key + from + j);
                const uint32_t four[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    if (four[m] == want) {
                        if (skip == 0u) expert[i] = from + j + m;
                        --skip;
                    }
                }
            }
            score[i] = a.bias != nullptr ? row_s[expert[i]] : key_value(want);
        }
        D += score[i];
    }
    D = seg_sum<LANES>(D);
    if (live) {
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int r = lane + i * LANES;
            if (r < a.k) {
                const float w = a.renorm ? (D == 0.0f ? 0.0f : __fdiv_rn(score[i], D)) : score[i];
                a.experts[t * a.k + r] = expert[i];
                a.weights[t * a.k + r] = w * a.scale;
            }
        }
    }
}

// one zero after the other: this token's lanes clear its row of the gradient
template <int LANES, typename SRC>
__device__ __forceinline__ void clear_row(SRC* dst, int E, bool wide, int lane) {
    int done = 0;
    if (wide) {
        const float zero[8] = {};
        for (int e = lane * 8; e + 8 <= E; e += LANES * 8) store8(dst + e, zero);
        done = E & ~7;
    }
    for (int e = done + lane; e < E; e += LANES) store1(dst + e, 0.0f);
}

// Gradient where only the chosen experts have one: with r_j = s_j / D the softmax's own normaliser cancels, and a
// sigmoid's score depends on its logit alone.  So k logits are read, not the row; the row is cleared while they are on
// their way and the k values follow.  One lane per slot, 32 / LANES tokens per warp.
template <int LANES, typename SRC>
__global__ void __launch_bounds__(kRouteThreads) route_backward_sparse_kernel(const RouteArgs a) {
    constexpr int kTokens = kRouteThreads / LANES;
    const int lane = threadIdx.x % LANES, tok = threadIdx.x / LANES;
    const int64_t t = static_cast<int64_t>(blockIdx.x) * kTokens + tok;
    const bool live = t < a.T;
    grid_dependency_wait();
    grid_launch_dependents();
    const bool slot = live && lane < a.k;
    int e = slot ? __ldg(a.experts + t * a.k + lane) : -1;
    const float dw_raw = slot ? __ldg(a.d_weights + t * a.k + lane) : 0.0f;
    if (e < 0 || e >= a.E) e = -1;
    const float dw = e < 0 ? 0.0f : dw_raw;
    const float x = e < 0 ? -CUDART_INF_F : load1<SRC>(static_cast<const SRC*>(a.logits) + t * a.ld + e);
    SRC* dst = static_cast<SRC*>(a.d_logits) + (live ? t : 0) * a.ld_d;
    if (live) clear_row<LANES, SRC>(dst, a.E, a.wide_d != 0, lane);
    float s;
    if (a.score == FP8MLP_SCORE_SOFTMAX) {
        const float m = seg_maxf<LANES>(x);
        s = e < 0 ? 0.0f : expf(x - m);
    } else {
        s = e < 0 ? 0.0f : sigmoid_exact(x);
    }
    float g = s * dw;
    if (a.renorm) {
        const float D = seg_sum<LANES>(s);
        const float r = D == 0.0f ? 0.0f : __fdiv_rn(s, D);
        g = r * (dw - seg_sum<LANES>(r * dw));
    }
    if (a.score == FP8MLP_SCORE_SIGMOID) g *= sigmoid_exact(-x);      // 1 - s
    __syncwarp();                                                      // the row is clear before its k values are written
    if (e >= 0) store1(dst + e, a.scale * g);
}

// Gradient of softmax weights that are not renormalised: every expert of the row has one.
template <int LANES, int V, typename SRC>
__global__ void __launch_bounds__(kRouteThreads) route_backward_dense_kernel(const RouteArgs a) {
    extern __shared__ __align__(16) uint32_t smem[];
    constexpr int kTokens = kRouteThreads / LANES;
    constexpr int kRow = LANES * V + 4;
    const int lane = threadIdx.x % LANES, tok = threadIdx.x / LANES;
    float* row = reinterpret_cast<float*>(smem) + tok * kRow;         // gradient of the row's scores, then of its logits
    const int64_t t = static_cast<int64_t>(blockIdx.x) * kTokens + tok;
    const bool live = t < a.T;
    const int e0 = lane * V;
    grid_dependency_wait();
    grid_launch_dependents();
    float s[V];
    if (live) {
        load_row<V, SRC>(static_cast<const SRC*>(a.logits) + t * a.ld, e0, a.E, a.wide != 0, s);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) s[j] = -CUDART_INF_F;
    }
#pragma unroll
    for (int j = 0; j < V; j += 4) *reinterpret_cast<float4*>(row + e0 + j) = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    __syncwarp();
    bool any = false;
    if (live) {
        for (int r = lane; r < a.k; r += LANES) {
            const int e = __ldg(a.experts + t * a.k + r);
            if (e >= 0 && e < a.E) {
                row[e] = a.scale * __ldg(a.d_weights + t * a.k + r);
                any = true;
            }
        }
    }
    any = seg_max<LANES>(any ? 1u : 0u) != 0u;
    softmax_row<LANES, V>(s);
    __syncwarp();
    float ds[V], dot = 0.0f;
#pragma unroll
    for (int j = 0; j < V; j += 4) *reinterpret_cast<float4*>(&ds[j]) = *reinterpret_cast<const float4*>(row + e0 + j);
#pragma unroll
    for (int j = 0; j < V; ++j) dot += s[j] * ds[j];
    dot = seg_sum<LANES>(dot);
#pragma unroll
    for (int j = 0; j < V; ++j) s[j] = any ? s[j] * (ds[j] - dot) : 0.0f;
    SRC* dst = static_cast<SRC*>(a.d_logits) + t * a.ld_d;
    if (a.wide_d) {
        if (!live) return;
#pragma unroll
        for (int b = 0; b < V; b += 8) {
            if (e0 + b + 8 <= a.E) {
                store8(dst + e0 + b, &s[b]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (e0 + b + i < a.E) store1(dst + e0 + b + i, s[b + i]);
            }
        }
    } else {                       // through shared memory: neighbouring lanes write neighbouring elements
#pragma unroll
        for (int j = 0; j < V; j += 4) *reinterpret_cast<float4*>(row + e0 + j) = make_float4(s[j], s[j + 1], s[j + 2], s[j + 3]);
        __syncwarp();
        if (!live) return;
        for (int e = lane; e < a.E; e += LANES) store1(dst + e, row[e]);
    }
}

__global__ void route_bias_kernel(int E, const int32_t* counts, float rate, float* bias) {
    __shared__ long long part[FP8MLP_MAX_EXPERTS / 32];
    grid_dependency_wait();
    grid_launch_dependents();
    const int e = threadIdx.x;
    const long long mine = e < E ? counts[e] : 0;
    long long v = mine;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
    if ((e & 31) == 0) part[e >> 5] = v;
    __syncthreads();
    long long sum = 0;
    for (int w = 0; w < FP8MLP_MAX_EXPERTS / 32; ++w) sum += part[w];
    const long long scaled = mine * E;                   // mean < count without a rounding
    if (e < E && scaled != sum) bias[e] += scaled < sum ? rate : -rate;
}

int check_router(const fp8mlp_router* r) {
    if (r == nullptr) return FP8MLP_ERR_ARG;
    if (r->score != FP8MLP_SCORE_SOFTMAX && r->score != FP8MLP_SCORE_SIGMOID) return FP8MLP_ERR_ARG;
    if (r->group_top != 1 && r->group_top != 2) return FP8MLP_ERR_ARG;
    if (r->n_experts < 1 || r->n_experts > FP8MLP_MAX_EXPERTS || r->top_k < 1 || r->top_k > FP8MLP_MAX_TOP_K ||
        r->top_k > r->n_experts)
        return FP8MLP_ERR_SHAPE;
    if (r->n_groups < 1 || r->n_experts % r->n_groups != 0 || r->top_groups < 1 || r->top_groups > r->n_groups ||
        r->top_k > r->top_groups * (r->n_experts / r->n_groups))
        return FP8MLP_ERR_SHAPE;
    return FP8MLP_OK;
}

bool multiple_of(const void* p, int64_t n) { return reinterpret_cast<uintptr_t>(p) % static_cast<uintptr_t>(n) == 0; }

RouteArgs route_args(const fp8mlp_router* r, int64_t T, const void* logits, int64_t ld, int esize) {
    RouteArgs a{};
    a.logits = logits;
    a.T = T; a.ld = ld;
    a.E = r->n_experts; a.k = r->top_k; a.score = r->score;
    a.G = r->n_groups; a.per = r->n_experts / r->n_groups; a.top_groups = r->top_groups; a.group_top = r->group_top;
    a.renorm = r->renormalise != 0; a.scale = r->scale;
    a.wide = multiple_of(logits, 8 * esize) && ld % 8 == 0;
    return a;
}

template <int LANES>
int launch_tokens(void (*kernel)(const RouteArgs), const RouteArgs& a, size_t smem, cudaStream_t st) {
    constexpr int kTokens = kRouteThreads / LANES;
    const int64_t blocks = (a.T + kTokens - 1) / kTokens;
    if (blocks > 0x7fffffff) return FP8MLP_ERR_SHAPE;
    if (smem > 48 * 1024) FP8MLP_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 64 * 1024));
    FP8MLP_CUDA_CHECK(launch_chained(kernel, dim3(static_cast<unsigned>(blocks)), kRouteThreads, smem, st, a));
    FP8MLP_LAUNCH_CHECK();
    return FP8MLP_OK;
}

template <int LANES, int V>
int launch_route(RouteArgs a, int dtype, cudaStream_t st) {
    constexpr int kTokens = kRouteThreads / LANES;
    a.lane_groups = a.G > 1 && a.per % V == 0 && ((a.per / V) & (a.per / V - 1)) == 0;
    size_t words = static_cast<size_t>(kTokens) * (2 * a.k + 2 * (LANES * V + 4));
    if (a.G > 1 && !a.lane_groups) words += static_cast<size_t>(kTokens) * a.G;
    // below 26 KiB up to 512 experts, 50 KiB for 1024 in 1024 groups
    return launch_tokens<LANES>(dtype == FP8MLP_F32 ? route_kernel<LANES, V, float> : route_kernel<LANES, V, uint16_t>, a,
                                words * sizeof(float), st);
}
template <int LANES, int V>
int launch_backward_dense(const RouteArgs& a, int dtype, cudaStream_t st) {
    return launch_tokens<LANES>(dtype == FP8MLP_F32 ? route_backward_dense_kernel<LANES, V, float>
                                                    : route_backward_dense_kernel<LANES, V, uint16_t>,
                                a, (kRouteThreads / LANES) * (LANES * V + 4) * sizeof(float), st);
}
template <int LANES>
int launch_backward_sparse(const RouteArgs& a, int dtype, cudaStream_t st) {
    return launch_tokens<LANES>(dtype == FP8MLP_F32 ? route_backward_sparse_kernel<LANES, float>
                                                    : route_backward_sparse_kernel<LANES, uint16_t>, a, 0, st);
}

// LANES x V covers the row with the fewest lanes that keep V at 8; beyond 256 experts V grows.
int run_route(const RouteArgs& a, int dtype, cudaStream_t st) {
    if (a.E <= 8) return launch_route<1, 8>(a, dtype, st);
    if (a.E <= 16) return launch_route<2, 8>(a, dtype, st);
    if (a.E <= 32) return launch_route<4, 8>(a, dtype, st);
    if (a.E <= 64) return launch_route<8, 8>(a, dtype, st);
    if (a.E <= 128) return launch_route<16, 8>(a, dtype, st);
    if (a.E <= 256) return launch_route<32, 8>(a, dtype, st);
    if (a.E <= 512) return launch_route<32, 16>(a, dtype, st);
    return launch_route<32, 32>(a, dtype, st);
}
int run_route_backward(const RouteArgs& a, int dtype, cudaStream_t st) {
    if (a.score == FP8MLP_SCORE_SIGMOID || a.renorm) {
        if (a.k <= 4) return launch_backward_sparse<4>(a, dtype, st);
        if (a.k <= 8) return launch_backward_sparse<8>(a, dtype, st);
        if (a.k <= 16) return launch_backward_sparse<16>(a, dtype, st);
        return launch_backward_sparse<32>(a, dtype, st);
    }
    if (a.E <= 8) return launch_backward_dense<1, 8>(a, dtype, st);
    if (a.E <= 16) return launch_backward_dense<2, 8>(a, dtype, st);
    if (a.E <= 32) return launch_backward_dense<4, 8>(a, dtype, st);
    if (a.E <= 64) return launch_backward_dense<8, 8>(a, dtype, st);
    if (a.E <= 128) return launch_backward_dense<16, 8>(a, dtype, st);
    if (a.E <= 256) return launch_backward_dense<32, 8>(a, dtype, st);
    if (a.E <= 512) return launch_backward_dense<32, 16>(a, dtype, st);
    return launch_backward_dense<32, 32>(a, dtype, st);
}

}  // namespace

}  // namespace fp8mlp

using namespace fp8mlp;

extern "C" int fp8mlp_route(const fp8mlp_router* r, int64_t T, const void* logits, int dtype, int64_t ld, const float* bias,
                            int32_t* experts, float* weights, void* stream) {
    const int rc = check_router(r);
    if (rc != FP8MLP_OK) return rc;
    if (dtype != FP8MLP_BF16 && dtype != FP8MLP_F32) return FP8MLP_ERR_ARG;
    if (T < 0 || (T > 0 && ld < r->n_experts)) return FP8MLP_ERR_SHAPE;
    if (T == 0) return FP8MLP_OK;
    if (logits == nullptr || experts == nullptr || weights == nullptr) return FP8MLP_ERR_ARG;
    const int esize = dtype == FP8MLP_F32 ? 4 : 2;
    if (!multiple_of(logits, esize) || !multiple_of(bias, 4) || !multiple_of(experts, 4) || !multiple_of(weights, 4))
        return FP8MLP_ERR_ALIGN;
    RouteArgs a = route_args(r, T, logits, ld, esize);
    a.bias = bias; a.experts = experts; a.weights = weights;
    a.wide_b = multiple_of(bias, 32);
    return run_route(a, dtype, static_cast<cudaStream_t>(stream));
}

extern "C" int fp8mlp_route_backward(const fp8mlp_router* r, int64_t T, const void* logits, int dtype, int64_t ld,
                                     const int32_t* experts, const float* d_weights, void* d_logits, int64_t ld_d,
                                     void* stream) {
    const int rc = check_router(r);
    if (rc != FP8MLP_OK) return rc;
    if (dtype != FP8MLP_BF16 && dtype != FP8MLP_F32) return FP8MLP_ERR_ARG;
    if (T < 0 || (T > 0 && (ld < r->n_experts || ld_d < r->n_experts))) return FP8MLP_ERR_SHAPE;
    if (T == 0) return FP8MLP_OK;
    if (logits == nullptr || experts == nullptr || d_weights == nullptr || d_logits == nullptr) return FP8MLP_ERR_ARG;
    const int esize = dtype == FP8MLP_F32 ? 4 : 2;
    if (!multiple_of(logits, esize) || !multiple_of(d_logits, esize) || !multiple_of(experts, 4) || !multiple_of(d_weights, 4))
        return FP8MLP_ERR_ALIGN;
    RouteArgs a = route_args(r, T, logits, ld, esize);
    a.experts = const_cast<int32_t*>(experts); a.d_weights = d_weights; a.d_logits = d_logits; a.ld_d = ld_d;
    a.wide_d = multiple_of(d_logits, 8 * esize) && ld_d % 8 == 0;
    return run_route_backward(a, dtype, static_cast<cudaStream_t>(stream));
}

extern "C" int fp8mlp_route_update_bias(int n_experts, const int32_t* counts, float rate, float* bias, void* stream) {
    if (n_experts < 1 || n_experts > FP8MLP_MAX_EXPERTS) return FP8MLP_ERR_SHAPE;
    if (counts == nullptr || bias == nullptr) return FP8MLP_ERR_ARG;
    if (!multiple_of(counts, 4) || !multiple_of(bias, 4)) return FP8MLP_ERR_ALIGN;
    FP8MLP_CUDA_CHECK(launch_chained(route_bias_kernel, 1, FP8MLP_MAX_EXPERTS, 0, static_cast<cudaStream_t>(stream), n_experts,
                                     counts, rate, bias));
    FP8MLP_LAUNCH_CHECK();
    return FP8MLP_OK;
}
