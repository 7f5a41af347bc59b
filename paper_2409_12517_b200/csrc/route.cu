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
    int can_lose;                  // renormalised softmax whose choice may pass over the row's largest logits
    int wide, wide_b, wide_d;      // rows of logits, the bias, rows of d_logits start on a vector boundary
    // How a row lies on its lanes: blocks of lay_per experts on 2^lane_shift lanes each, per_lane to a lane.  A block is a group
    // where the groups fall on lanes (on_lanes), else the row; then 2^sub_shift lanes work on a group in shared memory.
    int lay_per, lane_shift, per_lane, on_lanes, sub_shift;
    uint32_t inv_per;      // ceil(2^20 / per)
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

// a lane's logits of one row, experts e0 .. E - 1 (at most V); the places beyond them read as -inf
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

template <int LANES> __device__ __forceinline__ float seg_sum(float v) {
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
    return v;
}
// maximum over the token's lanes; a NaN loses against any number
template <int LANES> __device__ __forceinline__ float seg_max(float v) {
    if constexpr (LANES == 32) {
        float r;
        asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
        return r;
    } else {
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(kAll, v, o));
        return v;
    }
}

constexpr float kLog2e = 1.4426950408889634f;

// Scores on the special-function unit: 2^x and 1/x within 2^-22 relative.  sigma(x) = 1 / (1 + e^-x) keeps its digits at
// both ends (a small score is the reciprocal of a large number) down to 2^-126, below which it is 0; 1 - sigma(x) =
// sigma(-x).  The softmax's 2^x keeps subnormal results, so that far smaller experts still have an order.
__device__ __forceinline__ float ex2_subnormal(float x) {
    float y;
    asm("ex2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Softmax of the token's row, in place; a row without a finite maximum comes out as NaN.  The difference is taken before
// the factor log2 e: a finite mask (the type's lowest value) would overflow the other way round.
template <int LANES, int V>
__device__ __forceinline__ void softmax_row(float (&x)[V]) {
    float m = x[0];
#pragma unroll
    for (int j = 1; j < V; ++j) m = fmaxf(m, x[j]);
    m = seg_max<LANES>(m);
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < V; ++j) { x[j] = ex2_subnormal(__fmul_rn(x[j] - m, kLog2e)); sum += x[j]; }
    sum = seg_sum<LANES>(sum);
    const float inv = rcp_approx(sum);
#pragma unroll
    for (int j = 0; j < V; ++j) x[j] *= inv;
}

// the larger two of (a1 >= a2) and (b1 >= b2)
__device__ __forceinline__ void merge_top2(float& a1, float& a2, float b1, float b2) {
    a2 = fmaxf(fminf(a1, b1), fmaxf(a2, b2));
    a1 = fmaxf(a1, b1);
}
// a group's value; -inf: nothing to choose in it, and a missing second expert adds nothing.  Two finite values whose sum
// falls below fp32 (a bias of the lowest value) are held at its lowest: their group has something to choose.
__device__ __forceinline__ float group_value(float c1, float c2, int group_top) {
    return group_top == 2 && c2 > -CUDART_INF_F ? fmaxf(c1 + c2, -CUDART_MAX_NORMAL_F) : c1;
}

// 8 values into falling order (19 exchanges)
__device__ __forceinline__ void exchange(float& a, float& b) {
    const float hi = fmaxf(a, b);
    b = fminf(a, b);
    a = hi;
}
__device__ __forceinline__ void sort8(float (&c)[8]) {
    exchange(c[0], c[2]); exchange(c[1], c[3]); exchange(c[4], c[6]); exchange(c[5], c[7]);
    exchange(c[0], c[4]); exchange(c[1], c[5]); exchange(c[2], c[6]); exchange(c[3], c[7]);
    exchange(c[0], c[1]); exchange(c[2], c[3]); exchange(c[4], c[5]); exchange(c[6], c[7]);
    exchange(c[2], c[4]); exchange(c[3], c[5]);
    exchange(c[1], c[4]); exchange(c[3], c[6]);
    exchange(c[1], c[2]); exchange(c[3], c[4]); exchange(c[5], c[6]);
}
template <int V> __device__ __forceinline__ void put_row(float* row, const float (&v)[V]) {
#pragma unroll
    for (int j = 0; j < V; j += 4) *reinterpret_cast<float4*>(row + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
}

// Groups that do not fall on lanes: their values through shared memory (the row, then values and verdicts of the groups),
// 2^sub_shift lanes to a group.  Takes the experts of the groups that are not kept out of the lane's values.
template <int LANES, int V>
__device__ __forceinline__ void drop_groups_in_shared(const RouteArgs& a, int lane, int e0, float* row_c, float* group_c, float (&s)[V]) {
    put_row<V>(row_c + e0, s);
    __syncwarp();
    const int sub = lane & ((1 << a.sub_shift) - 1), sub_lanes = 1 << a.sub_shift, at_once = LANES >> a.sub_shift;
    for (int g0 = 0; g0 < a.G; g0 += at_once) {
        const int g = g0 + (lane >> a.sub_shift);
        float c1 = -CUDART_INF_F, c2 = -CUDART_INF_F;
        if (g < a.G) {
            for (int i = sub; i < a.per; i += sub_lanes) {
                const float v = row_c[g * a.per + i];
                c2 = fmaxf(c2, fminf(c1, v));
                c1 = fmaxf(c1, v);
            }
        }
        for (int o = 1; o < sub_lanes; o <<= 1) {
            const float b1 = __shfl_xor_sync(kAll, c1, o), b2 = __shfl_xor_sync(kAll, c2, o);
            merge_top2(c1, c2, b1, b2);
        }
        if (g < a.G && sub == 0) group_c[g] = group_value(c1, c2, a.group_top);
    }
    __syncwarp();
    float* group_keep = group_c + a.G;
    for (int g0 = 0; g0 < a.G; g0 += at_once) {
        const int g = g0 + (lane >> a.sub_shift);
        int rank = 0;
        if (g < a.G) {
            const float mine = group_c[g];
            for (int i = sub; i < a.G; i += sub_lanes) rank += (i < g ? group_c[i] >= mine : group_c[i] > mine) ? 1 : 0;
        }
        for (int o = 1; o < sub_lanes; o <<= 1) rank += __shfl_xor_sync(kAll, rank, o);
        if (g < a.G && sub == 0) group_keep[g] = rank < a.top_groups ? CUDART_INF_F : -CUDART_INF_F;
    }
    __syncwarp();
#pragma unroll
    for (int j = 0; j < V; ++j)          // e / per by a product that is exact for e, per <= 1024
        if (e0 + j < a.E) s[j] = fminf(s[j], group_keep[(static_cast<uint32_t>(e0 + j) * a.inv_per) >> 20]);
}

// Scores and values of the choice of one token, s: in logits, out values c; the scores go to row_s where a bias parts them.
template <int LANES, int V>
__device__ __forceinline__ void score_row(const RouteArgs& a, int e0, bool biased, const float (&bias)[V], float* row_s, float (&s)[V]) {
    // Sums that come out as a number above -inf show that no logit is masked and no value NaN or -inf: additions run beside
    // the comparisons (another pipe, the one that limits this kernel), and masks are rare.
    float sum_x = s[0];
    uint32_t masked = 0;
#pragma unroll
    for (int j = 1; j < V; ++j) sum_x += s[j];
    if (!(sum_x > -CUDART_INF_F)) {
#pragma unroll
        for (int j = 0; j < V; ++j) masked |= (s[j] == -CUDART_INF_F ? 1u : 0u) << j;
    }
    if (a.score == FP8MLP_SCORE_SOFTMAX) {
        softmax_row<LANES, V>(s);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) s[j] = sigmoid_f32(s[j]);
    }
    if (biased) {
        put_row<V>(row_s + e0, s);
#pragma unroll
        for (int j = 0; j < V; ++j) s[j] += bias[j];
    }
    float sum_c = s[0];
#pragma unroll
    for (int j = 1; j < V; ++j) sum_c += s[j];
    if (masked != 0u || !(sum_c > -CUDART_INF_F)) {
#pragma unroll
        for (int j = 0; j < V; ++j) s[j] = (masked >> j & 1u) != 0u ? -CUDART_INF_F : fmaxf(s[j], -CUDART_INF_F);   // NaN: -inf
    }
}

// The choice: every lane sorts its values c, eight at a time, and the token's lanes take the largest head k times.  Instructions
// cost more than the bytes (8 of 256 experts in 4 of 8 groups: 523 warp instructions a token with Q = 2; their issue takes 30
// of 35.6 us for 65536 tokens, and 7.5 of 11.2 us for 16384, where the rest goes to every block's first loads and a second
// wave that is not full), so a round moves values only; which expert a value belongs to is looked up once at the end, by k
// lanes side by side, in the unsorted row in shared memory.  -inf stands for "cannot be chosen".
// The lanes hold Q tokens, whose steps are interleaved: the group loops and rounds run once for both, and one's reductions
// wait behind the other's.  With Q = 2 those 16384 tokens take 11.2 us instead of 13.3 (65536: 35.6 and 43.1; the bytes need
// 2.7 at 16384; other sizes: two_at_a_time); without groups 9.7 and 9.4, one token 2.6 and 2.2.
// Blocks per SM with Q = 1: 12 of 40 registers with a whole warp per token (16 of 32: 14.0 us), 16 where tokens share a
// warp (64 experts: 5.9 us, 7.3 with 12).  More experts per lane and fewer lanes per token were slower or equal.
template <int LANES, int V, int Q, typename SRC>
__global__ void __launch_bounds__(kRouteThreads, Q > 1 ? 8 : V > 8 ? 4 : LANES == 32 ? 12 : 16) route_kernel(const RouteArgs a) {
    extern __shared__ __align__(16) float smem[];
    constexpr int kTokens = kRouteThreads / LANES * Q;
    constexpr int kRow = LANES * V + 4;                   // + 4: rows of neighbouring tokens start in other banks
    constexpr int kLists = V / 8;
    const int lane = threadIdx.x % LANES, seg_base = (threadIdx.x & 31) - lane;
    const int e0 = lane * V;                              // this lane's places in the rows in shared memory, and its experts
    const int first = (lane >> a.lane_shift) * a.lay_per + (lane & ((1 << a.lane_shift) - 1)) * a.per_lane;
    const int end = min(min(first + a.per_lane, ((lane >> a.lane_shift) + 1) * a.lay_per), a.E);
    const bool biased = a.bias != nullptr;
    float *row_c[Q], *row_s[Q], *group_c[Q];              // a token's values and scores; its groups, where they are off the lanes
    float2* sel[Q];                                       // a round's value and its lane
    int64_t t[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        const int tok = threadIdx.x / LANES * Q + q;
        row_c[q] = smem + tok * kRow;
        row_s[q] = smem + (kTokens + tok) * kRow;
        sel[q] = reinterpret_cast<float2*>(smem + 2 * kTokens * kRow) + tok * a.k;
        group_c[q] = smem + 2 * kTokens * (kRow + a.k) + tok * 2 * a.G;
        t[q] = static_cast<int64_t>(blockIdx.x) * kTokens + tok;
    }
    grid_dependency_wait();
    grid_launch_dependents();

    float s[Q][V], bias[V], c[Q][kLists][8];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        if (t[q] < a.T) {
            load_row<V, SRC>(static_cast<const SRC*>(a.logits) + t[q] * a.ld, first, end, a.wide != 0, s[q]);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) s[q][j] = -CUDART_INF_F;
        }
    }
    if (biased) load_row<V, float>(a.bias, first, end, a.wide_b != 0, bias);
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        score_row<LANES, V>(a, e0, biased, bias, row_s[q], s[q]);
        if constexpr (Q == 1) {
            if (a.G > 1 && !a.on_lanes) drop_groups_in_shared<LANES, V>(a, lane, e0, row_c[q], group_c[q], s[q]);
        }
        put_row<V>(row_c[q] + e0, s[q]);
#pragma unroll
        for (int l = 0; l < kLists; ++l) {
#pragma unroll
            for (int j = 0; j < 8; ++j) c[q][l][j] = s[q][l * 8 + j];
            sort8(c[q][l]);
        }
    }

    if (a.on_lanes) {
        const int width = 1 << a.lane_shift;             // lanes of a group
        float c1[Q], c2[Q], value[Q];
        int rank[Q];
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            c1[q] = c[q][0][0];
            c2[q] = c[q][0][1];
#pragma unroll
            for (int l = 1; l < kLists; ++l) merge_top2(c1[q], c2[q], c[q][l][0], c[q][l][1]);
        }
        for (int o = 1; o < width; o <<= 1) {
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                const float b1 = __shfl_xor_sync(kAll, c1[q], o), b2 = __shfl_xor_sync(kAll, c2[q], o);
                merge_top2(c1[q], c2[q], b1, b2);
            }
        }
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            value[q] = group_value(c1[q], c2[q], a.group_top);
            rank[q] = 0;
        }
        // the group's lanes share the comparisons with the other groups
        const int mine = lane >> a.lane_shift, sub = lane & (width - 1), steps = (a.G + width - 1) >> a.lane_shift;
        constexpr int kSteps = Q == 1 ? 4 : 1;
#pragma unroll kSteps
        for (int i = 0; i < steps; ++i) {
            const int g = (i << a.lane_shift) + sub;
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                const float other = __shfl_sync(kAll, value[q], (seg_base + (g << a.lane_shift)) & 31);
                if (g < a.G && (other > value[q] || (other == value[q] && g < mine))) ++rank[q];
            }
        }
        for (int o = 1; o < width; o <<= 1) {
#pragma unroll
            for (int q = 0; q < Q; ++q) rank[q] += __shfl_xor_sync(kAll, rank[q], o);
        }
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            if (rank[q] < a.top_groups) continue;
#pragma unroll
            for (int l = 0; l < kLists; ++l)
#pragma unroll
                for (int j = 0; j < 8; ++j) c[q][l][j] = -CUDART_INF_F;
        }
    }

    float best[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        best[q] = c[q][0][0];
#pragma unroll
        for (int l = 1; l < kLists; ++l) best[q] = fmaxf(best[q], c[q][l][0]);
    }
    const uint32_t lower = ((1u << lane) - 1u) << seg_base;      // the token's lanes below this one
    for (int r = 0; r < a.k; ++r) {
        float top[Q];
        bool gives[Q];
#pragma unroll
        for (int q = 0; q < Q; ++q) top[q] = seg_max<LANES>(best[q]);
#pragma unroll
        for (int q = 0; q < Q; ++q) {       // the lowest lane among equals holds the lowest expert
            const bool holds = best[q] == top[q];
            gives[q] = (__ballot_sync(kAll, holds) & lower) == 0u && holds;
        }
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            if (!gives[q]) continue;
            sel[q][r] = make_float2(top[q], __int_as_float(lane));
            bool taken = false;
            best[q] = -CUDART_INF_F;
#pragma unroll
            for (int l = 0; l < kLists; ++l) {
                if (kLists == 1 || (!taken && c[q][l][0] == top[q])) {
                    taken = true;
#pragma unroll
                    for (int j = 0; j < 7; ++j) c[q][l][j] = c[q][l][j + 1];
                    c[q][l][7] = -CUDART_INF_F;
                }
                best[q] = fmaxf(best[q], c[q][l][0]);
            }
        }
    }
    __syncwarp();
    constexpr int kMine = LANES >= 4 ? (FP8MLP_MAX_TOP_K + LANES - 1) / LANES : 8;      // k <= LANES * 8 where LANES < 4
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        float D = 0.0f, score[kMine];
        int32_t expert[kMine];
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int r = lane + i * LANES;
            score[i] = 0.0f;
            expert[i] = -1;
            if (r < a.k && sel[q][r].x > -CUDART_INF_F) {
                const float want = sel[q][r].x;
                const int owner = __float_as_int(sel[q][r].y), from = owner * V;
                // equal values of one lane are taken in turn, lowest expert first: the first place of the value, and for
                // the next of its equals one place further each
                int skip = 0;
                while (skip < r && sel[q][r - 1 - skip].x == want && __float_as_int(sel[q][r - 1 - skip].y) == owner) ++skip;
                int place = from;
#pragma unroll
                for (int j = V - 4; j >= 0; j -= 4) {
                    const float4 w = *reinterpret_cast<const float4*>(row_c[q] + from + j);
                    if (w.w == want) place = from + j + 3;
                    if (w.z == want) place = from + j + 2;
                    if (w.y == want) place = from + j + 1;
                    if (w.x == want) place = from + j;
                }
                for (; skip > 0; --skip)
                    do { ++place; } while (place < from + V - 1 && row_c[q][place] != want);
                expert[i] = (owner >> a.lane_shift) * a.lay_per + (owner & ((1 << a.lane_shift) - 1)) * a.per_lane + place - from;
                score[i] = biased ? row_s[q][place] : want;
            }
            D += score[i];
        }
        D = seg_sum<LANES>(D);
        if (a.can_lose) {
            // Where a bias or the groups hold back the experts of the large logits, the chosen scores can be so small that fp32
            // keeps few of their digits or none (D = 0).  Their ratios are the softmax over the chosen logits all the same, which
            // are read again for such tokens (D >= 2^-64 leaves every weight above 2^-62 all its digits).
            const bool lost = t[q] < a.T && D < 0x1p-64f;
            if (__any_sync(kAll, lost)) {
                const SRC* row = static_cast<const SRC*>(a.logits) + t[q] * a.ld;
                float top = -CUDART_INF_F, sum = 0.0f;
#pragma unroll
                for (int i = 0; i < kMine; ++i)
                    if (lost && expert[i] >= 0) top = fmaxf(top, load1<SRC>(row + expert[i]));
                top = seg_max<LANES>(top);
#pragma unroll
                for (int i = 0; i < kMine; ++i) {
                    if (lost && expert[i] >= 0) score[i] = ex2_subnormal(__fmul_rn(load1<SRC>(row + expert[i]) - top, kLog2e));
                    sum += score[i];
                }
                sum = seg_sum<LANES>(sum);
                if (lost) D = sum;
            }
        }
        if (t[q] >= a.T) continue;
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int r = lane + i * LANES;
            if (r < a.k) {
                const float w = a.renorm ? (D == 0.0f ? 0.0f : __fdiv_rn(score[i], D)) : score[i];
                a.experts[t[q] * a.k + r] = expert[i];
                a.weights[t[q] * a.k + r] = w * a.scale;
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
// their way and the k values follow.  One lane per slot, 32 / LANES tokens per warp.  16384 x 256 fp32: 6.0 us, of which
// the 17 MB written need 2.6 and launch and the chain of loads (expert, then its logit) most of the rest; reading and
// staging whole rows took 11.8.
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
        const float m = seg_max<LANES>(x);
        s = e < 0 ? 0.0f : ex2_approx(__fmul_rn(x - m, kLog2e));
    } else {
        s = e < 0 ? 0.0f : sigmoid_f32(x);
    }
    float g = s * dw;
    if (a.renorm) {
        const float D = seg_sum<LANES>(s);
        const float r = D == 0.0f ? 0.0f : __fdiv_rn(s, D);      // exactly 1, and no gradient, for a single expert
        g = r * (dw - seg_sum<LANES>(r * dw));
    }
    if (a.score == FP8MLP_SCORE_SIGMOID) g *= sigmoid_f32(-x);      // 1 - s
    __syncwarp();                                                      // the row is clear before its k values are written
    if (e >= 0) store1(dst + e, a.scale * g);
}

// Gradient of softmax weights that are not renormalised: every expert of the row has one.  The k gradients of the chosen
// scores are scattered in shared memory and read back by the lanes that hold those experts.  32768 x 64 bf16: 5.0 us.
template <int LANES, int V, typename SRC>
__global__ void __launch_bounds__(kRouteThreads) route_backward_dense_kernel(const RouteArgs a) {
    extern __shared__ __align__(16) float smem[];
    constexpr int kTokens = kRouteThreads / LANES;
    constexpr int kRow = LANES * V + 4;
    const int lane = threadIdx.x % LANES, tok = threadIdx.x / LANES;
    float* row = smem + tok * kRow;         // gradient of the row's scores, then of its logits
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
    any = seg_max<LANES>(any ? 1.0f : 0.0f) != 0.0f;
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

template <int LANES, int Q = 1>
int launch_tokens(void (*kernel)(const RouteArgs), const RouteArgs& a, size_t smem, cudaStream_t st) {
    constexpr int kTokens = kRouteThreads / LANES * Q;
    const int64_t blocks = (a.T + kTokens - 1) / kTokens;
    if (blocks > 0x7fffffff) return FP8MLP_ERR_SHAPE;
    if (smem > 48 * 1024) FP8MLP_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 72 * 1024));
    FP8MLP_CUDA_CHECK(launch_chained(kernel, dim3(static_cast<unsigned>(blocks)), kRouteThreads, smem, st, a));
    FP8MLP_LAUNCH_CHECK();
    return FP8MLP_OK;
}

// Lanes of a token whose groups lie on lanes of their own, V experts to a lane: a power of two for each group, and one of
// such groups.  More than 32: they do not fit.
int group_lanes(int G, int per, int V) {
    int groups = 1, width = 1;
    while (groups < G) groups *= 2;
    while (width * V < per) width *= 2;
    return groups * width;
}

template <int LANES, int V, int Q = 1>
int launch_route(RouteArgs a, int dtype, cudaStream_t st) {
    constexpr int kTokens = kRouteThreads / LANES * Q;
    a.on_lanes = a.G > 1 && group_lanes(a.G, a.per, V) <= LANES;
    a.lay_per = a.on_lanes ? a.per : a.E;
    a.lane_shift = 0;
    if (a.on_lanes) {
        int groups = 1;
        while (groups < a.G) groups *= 2;
        while ((groups << (a.lane_shift + 1)) <= LANES) ++a.lane_shift;
    } else {
        while ((1 << (a.lane_shift + 1)) <= LANES) ++a.lane_shift;
    }
    // Whole vectors where the groups divide into them; else the same share for every lane, and single loads (a group's first
    // expert is then off the vector boundaries).
    a.per_lane = V;
    if (a.on_lanes && a.per % 8 != 0) {
        a.per_lane = (a.per + (1 << a.lane_shift) - 1) >> a.lane_shift;
        a.wide = a.wide_b = 0;
    }
    a.sub_shift = 0;
    while ((a.G << (a.sub_shift + 1)) <= LANES && (2 << a.sub_shift) <= a.per) ++a.sub_shift;
    a.inv_per = ((1u << 20) + a.per - 1) / a.per;
    size_t words = static_cast<size_t>(kTokens) * (2 * a.k + 2 * (LANES * V + 4));
    if (a.G > 1 && !a.on_lanes) words += static_cast<size_t>(kTokens) * 2 * a.G;
    // below 36 KiB up to 512 experts, 65 KiB for 1024 in 1024 groups
    return launch_tokens<LANES, Q>(dtype == FP8MLP_F32 ? route_kernel<LANES, V, Q, float> : route_kernel<LANES, V, Q, uint16_t>, a,
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

// A whole warp per token, groups on lanes: whether each warp takes two tokens.  Two share the steps' waits and instructions, one
// ends sooner and lets more blocks in: 24 tokens an SM at a time beside a second launch (half of 12 blocks of 4), 40 in twos
// (half of 10 blocks of 8), so the better of the two changes with the number of tokens, and sooner where the row fills the warp.
// us one at a time / in twos, 8 of 256 in 8 groups and 6 of 160 in 8:
//   tokens      1024        3000        3500        5000        6144        8192        9600        10500       16384
//   256      3.1 / 3.3   4.7 / 4.5   4.9 / 4.6   6.7 / 5.9   7.0 / 8.4   8.0 / 8.7   8.9 / 8.8   9.4 / 8.9   13.3 / 11.2
//   160      2.7 / 3.1   3.6 / 3.9   3.8 / 3.9   5.9 / 5.1   5.9 / 8.3   6.8 / 8.4   7.8 / 8.4   8.3 / 8.4   11.8 / 11.3
bool two_at_a_time(const RouteArgs& a) {
    const bool full = a.E > 192;
    if (a.T <= 24 * 148) return full && a.T > 2048;
    if (a.T <= 40 * 148) return true;
    return a.T > (full ? 60 : 72) * 148;
}

// LANES x V covers the row with the fewest lanes that keep V at 8; beyond 256 experts V grows.  Groups get lanes of their own
// where 32 are enough for that.
int run_route(const RouteArgs& a, int dtype, cudaStream_t st) {
    int lanes = 1;
    while (lanes * 8 < a.E) lanes *= 2;
    if (a.G > 1 && a.E <= 256) {
        const int grouped = group_lanes(a.G, a.per, 8);
        if (grouped <= 32) lanes = grouped;
    }
    if (lanes == 1) return launch_route<1, 8>(a, dtype, st);
    if (lanes == 2) return launch_route<2, 8>(a, dtype, st);
    if (lanes == 4) return launch_route<4, 8>(a, dtype, st);
    if (lanes == 8) return launch_route<8, 8>(a, dtype, st);
    if (lanes == 16) return launch_route<16, 8>(a, dtype, st);
    if (lanes == 32)
        return a.G > 1 && group_lanes(a.G, a.per, 8) <= 32 && two_at_a_time(a) ? launch_route<32, 8, 2>(a, dtype, st)
                                                                                : launch_route<32, 8>(a, dtype, st);
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
    a.can_lose = a.renorm && a.score == FP8MLP_SCORE_SOFTMAX && (bias != nullptr || a.G > 1);
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
    if (logits == nullptr || experts == nullptr || d_weights == nullptr || d_logits == nullptr || d_logits == logits)
        return FP8MLP_ERR_ARG;
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
