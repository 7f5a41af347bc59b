// Tokens into expert order and back: the plan (a stable counting sort of the chosen experts), the copy of the rows, the
// weighted sum of the experts' outputs and its gradient.
#include <atomic>

#include "common.cuh"

namespace fp8mlp {

namespace {

constexpr uint32_t kAll = 0xffffffffu;

// ---------------------------------------------------------------- plan
// Counting sort by one cluster.  Every warp owns a contiguous piece of the slots: it counts them through, 32 at a time,
// which gives each slot its place among those of its expert in the piece; the counts of all pieces then become start
// positions (over experts, then CTAs, then warps), and a second walk adds them.  No atomics: the order is that of the
// slots.  Which lanes of 32 share an expert follows from one ballot per bit of the expert's number (a match instruction
// took about 70 cycles of its SM each and made the plan of 131072 slots take 39 us).
constexpr int kPlanWarps = 32;
constexpr int kPlanFill = 8;          // warps of a CTA that own slots before the cluster grows
constexpr int kPlanMaxCluster = 16;
constexpr int kPlanUnroll = 4;
constexpr int kPlanPiece = 32 * kPlanUnroll;

struct PlanArgs {
    const int32_t* experts; int32_t *counts, *offsets, *rows;
    int64_t n;             // slots
    int64_t per_warp;      // slots of a warp, a multiple of 32
    int E, bits;           // experts, bits of the largest expert's number
    int key_warps;         // warps of a CTA that own slots (a CTA has more where the experts outnumber them)
};

__global__ void __launch_bounds__(kPlanWarps * 32) plan_kernel(const PlanArgs a) {
    extern __shared__ int32_t hist[];                    // [key_warps][E]: counts, then start positions
    __shared__ int32_t scan_part[kPlanWarps];
    __shared__ int32_t total[FP8MLP_MAX_EXPERTS];        // this CTA's slots per expert; the cluster reads it
    __shared__ int32_t start[FP8MLP_MAX_EXPERTS];        // where this CTA's first slot of an expert goes
    const int warps = blockDim.x / 32, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    uint32_t n_cta;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(n_cta));
    const uint32_t rank = cluster_ctarank();
    const int E = a.E;
    for (int i = threadIdx.x; i < a.key_warps * E; i += blockDim.x) hist[i] = 0;
    grid_dependency_wait();
    grid_launch_dependents();
    int64_t begin = (static_cast<int64_t>(rank) * a.key_warps + warp) * a.per_warp;
    int64_t end = begin + a.per_warp < a.n ? begin + a.per_warp : a.n;
    if (warp >= a.key_warps) begin = end = 0;
    int32_t* mine = hist + warp * E;
    const uint32_t below = (1u << lane) - 1u;
    __syncthreads();
    const bool once = a.per_warp <= kPlanPiece;          // the piece stays in registers between the two walks
    int e[kPlanUnroll], place[kPlanUnroll];
    for (int64_t i0 = begin + lane; i0 - lane < end; i0 += kPlanPiece) {
#pragma unroll
        for (int u = 0; u < kPlanUnroll; ++u) e[u] = i0 + 32 * u < end ? __ldg(a.experts + i0 + 32 * u) : -1;
        uint32_t same[kPlanUnroll];
#pragma unroll
        for (int u = 0; u < kPlanUnroll; ++u) same[u] = __ballot_sync(kAll, static_cast<uint32_t>(e[u]) < static_cast<uint32_t>(E));
        for (int b = 0; b < a.bits; ++b) {
#pragma unroll
            for (int u = 0; u < kPlanUnroll; ++u) {
                const bool bit = (e[u] >> b & 1) != 0;
                const uint32_t ones = __ballot_sync(kAll, bit);
                same[u] &= bit ? ones : ~ones;
            }
        }
#pragma unroll
        for (int u = 0; u < kPlanUnroll; ++u) {
            const bool used = static_cast<uint32_t>(e[u]) < static_cast<uint32_t>(E);
            const int32_t lower = __popc(same[u] & below);
            place[u] = used ? mine[e[u]] + lower : -1;
            __syncwarp();
            if (used && lower == 0) mine[e[u]] = place[u] + __popc(same[u]);
            __syncwarp();
            if (!once && i0 + 32 * u < end) a.rows[i0 + 32 * u] = place[u];
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += blockDim.x) {
        int32_t run = 0;
        for (int w0 = 0; w0 < a.key_warps; w0 += 8) {        // eight counts are read before any is replaced
            int32_t c[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) c[i] = w0 + i < a.key_warps ? hist[(w0 + i) * E + e] : 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (w0 + i < a.key_warps) hist[(w0 + i) * E + e] = run;
                run += c[i];
            }
        }
        total[e] = run;
    }
    __syncwarp();                                        // the loop ends earlier for some lanes, the cluster's barriers take whole warps
    if (n_cta > 1) cluster_sync_all();                   // every CTA's totals are there
    else __syncthreads();
    // offsets: a scan over the experts, one per thread at a time
    int32_t carry = 0;
    for (int e_base = 0; e_base < E; e_base += blockDim.x) {
        const int e = e_base + threadIdx.x;
        int32_t before = 0, all = 0;
        if (e < E) {
#pragma unroll 8
            for (uint32_t r = 0; r < n_cta; ++r) {
                int32_t c;
                asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(c) : "r"(mapa_shared(smem_u32(&total[e]), r)) : "memory");
                if (r < rank) before += c;
                all += c;
            }
        }
        int32_t incl = all;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int32_t v = __shfl_up_sync(kAll, incl, o);
            if (lane >= o) incl += v;
        }
        if (lane == 31) scan_part[warp] = incl;
        __syncthreads();
        int32_t lower = carry, chunk = 0;
        for (int w = 0; w < warps; ++w) {
            if (w < warp) lower += scan_part[w];
            chunk += scan_part[w];
        }
        const int32_t offset = lower + incl - all;
        if (e < E) {
            if (rank == 0) {
                a.counts[e] = all;
                a.offsets[e] = offset;
                if (e == E - 1) a.offsets[E] = offset + all;
            }
            start[e] = offset + before;
        }
        carry += chunk;
        __syncthreads();
    }
    if (n_cta > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");      // this CTA has read all totals
    for (int64_t i0 = begin + lane; i0 < end; i0 += kPlanPiece) {
        if (!once) {
#pragma unroll
            for (int u = 0; u < kPlanUnroll; ++u) {
                const bool in = i0 + 32 * u < end;
                e[u] = in ? __ldg(a.experts + i0 + 32 * u) : -1;
                place[u] = in ? a.rows[i0 + 32 * u] : -1;
            }
        }
#pragma unroll
        for (int u = 0; u < kPlanUnroll; ++u)
            if (i0 + 32 * u < end) a.rows[i0 + 32 * u] = place[u] < 0 ? -1 : place[u] + mine[e[u]] + start[e[u]];
    }
    __syncwarp();                                        // a ragged piece ends earlier for some lanes
    if (n_cta > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");        // and none leaves before the others have
}

// ---------------------------------------------------------------- rows
// Rows are moved in units of W 32-bit words: 8 (32 bytes) where every row starts on a 32-byte boundary, else 4.  A token's
// threads walk its row together; what a kernel reads for several slots it reads before it uses or writes any of it, so
// that the loads overlap.
template <int W> __device__ __forceinline__ void load_unit(const uint8_t* p, uint32_t (&w)[W]) {
    if constexpr (W == 8) {
        ld_global_nc_v8(p, w);
    } else {
        const uint4 v = ld_global_nc_v4(p);
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    }
}
template <int W> __device__ __forceinline__ void store_unit(uint8_t* p, const uint32_t (&w)[W]) {
    if constexpr (W == 8) st_global_v8(p, w);
    else st_global_v4(p, w[0], w[1], w[2], w[3]);
}
// elements of a word: two bf16 or one fp32
template <typename T> struct Word;
template <> struct Word<uint16_t> {
    static constexpr int kElems = 2;
    static __device__ __forceinline__ void get(uint32_t w, float* v) { v[0] = bf16_lo(w); v[1] = bf16_hi(w); }
    static __device__ __forceinline__ uint32_t put(const float* v) { return cvt_bf16x2(v[0], v[1]); }
};
template <> struct Word<float> {
    static constexpr int kElems = 1;
    static __device__ __forceinline__ void get(uint32_t w, float* v) { v[0] = __uint_as_float(w); }
    static __device__ __forceinline__ uint32_t put(const float* v) { return __float_as_uint(v[0]); }
};

constexpr int kRowThreads = 256;

struct RowArgs {
    const uint8_t* src;        // dispatch: x; combine: ye; combine_backward: ye
    uint8_t* dst;              // dispatch: xe; combine: y; combine_backward: dye
    const uint8_t* dy;         // combine_backward
    const int32_t* rows; const float* weights; float* d_weights;
    int64_t T;
    int64_t token_bytes;       // row stride of the token side (x, y, dy)
    uint32_t n_rows;
    uint32_t row_bytes;        // a row; those of the expert side are contiguous
    int k;
    int threads_per_token;     // of a block, whose threads hold blockDim.x / threads_per_token tokens
};

// the byte offset of a slot's row, or -1
__device__ __forceinline__ int64_t row_offset(const RowArgs& a, int64_t slot) {
    const uint32_t row = static_cast<uint32_t>(__ldg(a.rows + slot));        // negative: beyond every n_rows
    return row < a.n_rows ? static_cast<int64_t>(row) * a.row_bytes : -1;
}

// A row of x is read once and written once per slot: bound by DRAM writes.  16384 x 4096 bf16 to two rows each: 61 us for
// 403 MB, 6.6 TB/s.
template <int W>
__global__ void __launch_bounds__(kRowThreads) dispatch_kernel(const RowArgs a) {
    grid_dependency_wait();
    grid_launch_dependents();
    const int in_block = threadIdx.x / a.threads_per_token, lane = threadIdx.x - in_block * a.threads_per_token;
    const int64_t t = static_cast<int64_t>(blockIdx.x) * (blockDim.x / a.threads_per_token) + in_block;
    if (t >= a.T) return;
    const uint32_t step = a.threads_per_token * W * 4;
    for (uint32_t at = lane * W * 4; at < a.row_bytes; at += step) {
        uint32_t w[W];
        load_unit<W>(a.src + t * a.token_bytes + at, w);
#pragma unroll 4
        for (int j = 0; j < a.k; ++j) {
            const int64_t off = row_offset(a, t * a.k + j);
            if (off >= 0) store_unit<W>(a.dst + off + at, w);
        }
    }
}

// Bound by DRAM reads: 8192 x 4096 bf16 from six rows each take 70.4 us for 470 MB, 6.7 TB/s.  S slots of U units are in
// flight together.  More would cost occupancy (6 or 8 slots of 32 bytes ran 14 and 22 % slower than 3), fewer leave the
// memory idle, and a last batch that is not full does too.
template <typename T, int W, bool WEIGHTED, int S, int U>
__global__ void __launch_bounds__(kRowThreads, S == 4 ? 4 : 0) combine_kernel(const RowArgs a) {
    constexpr int E = Word<T>::kElems;
    grid_dependency_wait();
    grid_launch_dependents();
    const int in_block = threadIdx.x / a.threads_per_token, lane = threadIdx.x - in_block * a.threads_per_token;
    const int64_t t = static_cast<int64_t>(blockIdx.x) * (blockDim.x / a.threads_per_token) + in_block;
    if (t >= a.T) return;
    const uint32_t step = a.threads_per_token * W * 4;
    for (uint32_t at = lane * W * 4; at < a.row_bytes; at += U * step) {
        float acc[U][W * E];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < W * E; ++i) acc[u][i] = 0.0f;
        for (int j0 = 0; j0 < a.k; j0 += S) {
            uint32_t w[S][U][W];
            int64_t off[S];
            float scale[S];
#pragma unroll
            for (int j = 0; j < S; ++j) {
                off[j] = j0 + j < a.k ? row_offset(a, t * a.k + j0 + j) : -1;
                scale[j] = WEIGHTED && off[j] >= 0 ? __ldg(a.weights + t * a.k + j0 + j) : 1.0f;
            }
#pragma unroll
            for (int j = 0; j < S; ++j)
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (off[j] >= 0 && (u == 0 || at + u * step < a.row_bytes)) load_unit<W>(a.src + off[j] + at + u * step, w[j][u]);
#pragma unroll
            for (int j = 0; j < S; ++j) {
                if (off[j] < 0) continue;
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int i = 0; i < W; ++i) {
                        float v[E];
                        Word<T>::get(w[j][u][i], v);
#pragma unroll
                        for (int e = 0; e < E; ++e) {
                            float& sum = acc[u][i * E + e];
                            sum = WEIGHTED ? fmaf(scale[j], v[e], sum) : sum + v[e];
                        }
                    }
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u > 0 && at + u * step >= a.row_bytes) break;
            uint32_t out[W];
#pragma unroll
            for (int i = 0; i < W; ++i) out[i] = Word<T>::put(acc[u] + i * E);
            store_unit<W>(a.dst + t * a.token_bytes + at + u * step, out);
        }
    }
}

// One block per token; dy is read once for kSlots slots, every slot's row of ye once, and the dot products stay in
// registers until the row's end.  8192 x 4096 bf16 with six rows each: 131.5 us for 873 MB, 6.6 TB/s (the measured copy
// rate is 6.5); with four 32-byte units in flight 157 us, with eight 16-byte units 143.
constexpr int kSlots = 8;

template <typename T, int W>
__global__ void __launch_bounds__(kRowThreads) combine_backward_kernel(const RowArgs a) {
    constexpr int E = Word<T>::kElems, kBatch = W == 8 ? 2 : 4;       // slots whose loads are in flight together
    __shared__ float part[kRowThreads / 32][kSlots];
    grid_dependency_wait();
    grid_launch_dependents();
    const int64_t t = blockIdx.x;
    const uint8_t* dy = a.dy + t * a.token_bytes;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int j0 = 0; j0 < a.k; j0 += kSlots) {
        const int slots = min(kSlots, a.k - j0);
        int64_t off[kSlots];
        float scale[kSlots], dot[kSlots];
#pragma unroll
        for (int j = 0; j < kSlots; ++j) {
            off[j] = j < slots ? row_offset(a, t * a.k + j0 + j) : -1;
            scale[j] = off[j] >= 0 ? __ldg(a.weights + t * a.k + j0 + j) : 0.0f;
            dot[j] = 0.0f;
        }
        for (uint32_t at = threadIdx.x * W * 4; at < a.row_bytes; at += blockDim.x * W * 4) {
            uint32_t g[W];
            load_unit<W>(dy + at, g);
#pragma unroll
            for (int b = 0; b < kSlots; b += kBatch) {
                uint32_t w[kBatch][W];
#pragma unroll
                for (int j = 0; j < kBatch; ++j)
                    if (off[b + j] >= 0) load_unit<W>(a.src + off[b + j] + at, w[j]);
#pragma unroll
                for (int j = 0; j < kBatch; ++j) {
                    if (off[b + j] < 0) continue;
                    uint32_t out[W];
#pragma unroll
                    for (int i = 0; i < W; ++i) {
                        float v[E], d[E], o[E];
                        Word<T>::get(g[i], d);
                        Word<T>::get(w[j][i], v);
#pragma unroll
                        for (int e = 0; e < E; ++e) { dot[b + j] = fmaf(d[e], v[e], dot[b + j]); o[e] = scale[b + j] * d[e]; }
                        out[i] = Word<T>::put(o);
                    }
                    store_unit<W>(a.dst + off[b + j] + at, out);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < kSlots; ++j) {
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) dot[j] += __shfl_xor_sync(kAll, dot[j], o);
            if (lane == 0) part[warp][j] = dot[j];
        }
        __syncthreads();
        if (threadIdx.x < slots) {
            float sum = 0.0f;
            for (int i = 0; i < static_cast<int>(blockDim.x) / 32; ++i) sum += part[i][threadIdx.x];
            a.d_weights[t * a.k + j0 + threadIdx.x] = sum;
        }
        __syncthreads();
    }
}

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// Clusters of 16 CTAs are beyond the portable size: whether the device has room for one (a part of a GPU may not) is asked
// once per device, for the largest CTA that a plan launches, whose shared memory is allowed here as well.  Plans that do not
// ask have at most kPlanFill warps with slots to a CTA: 32 KiB and the 8 KiB of static arrays, within the default 48.
int plan_max_cluster(int* limit) {
    static std::atomic<int> known[64];
    int dev = 0;
    FP8MLP_CUDA_CHECK(cudaGetDevice(&dev));
    *limit = dev < 64 ? known[dev].load(std::memory_order_relaxed) : 0;
    if (*limit != 0) return FP8MLP_OK;
    const int smem = kPlanWarps * FP8MLP_MAX_EXPERTS * static_cast<int>(sizeof(int32_t));
    FP8MLP_CUDA_CHECK(cudaFuncSetAttribute(plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    FP8MLP_CUDA_CHECK(cudaFuncSetAttribute(plan_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(kPlanMaxCluster);
    cfg.blockDim = dim3(kPlanWarps * 32);
    cfg.dynamicSmemBytes = smem;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = kPlanMaxCluster;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int fit = 0;
    FP8MLP_CUDA_CHECK(cudaOccupancyMaxActiveClusters(&fit, plan_kernel, &cfg));
    *limit = fit > 0 ? kPlanMaxCluster : 8;
    if (dev < 64) known[dev].store(*limit, std::memory_order_relaxed);
    return FP8MLP_OK;
}

// What dispatch, combine and its gradient refuse alike; token / expert are the two row tensors.
int check_rows(int64_t T, int top_k, int64_t d, int dtype, const void* token, int64_t ld, const void* expert, int64_t n_rows,
               const int32_t* rows) {
    if (dtype != FP8MLP_BF16 && dtype != FP8MLP_F32) return FP8MLP_ERR_ARG;
    if (T < 0 || n_rows < 0 || d <= 0 || d % 16 != 0 || d > (1 << 24) || top_k < 1 || top_k > FP8MLP_MAX_TOP_K)
        return FP8MLP_ERR_SHAPE;
    if (T > 0x7fffffff / top_k || n_rows > 0x7fffffff) return FP8MLP_ERR_SHAPE;
    if (T == 0) return FP8MLP_OK;
    if (ld < d) return FP8MLP_ERR_SHAPE;
    if (token == nullptr || rows == nullptr || (expert == nullptr && n_rows > 0) || token == expert) return FP8MLP_ERR_ARG;
    const int64_t esize = dtype == FP8MLP_F32 ? 4 : 2;
    if (!aligned(token, 16) || !aligned(expert, 16) || ld * esize % 16 != 0 || !aligned(rows, 4)) return FP8MLP_ERR_ALIGN;
    return FP8MLP_OK;
}

RowArgs row_args(int64_t T, int top_k, int64_t d, int dtype, int64_t ld, int64_t n_rows, const int32_t* rows) {
    const int64_t esize = dtype == FP8MLP_F32 ? 4 : 2;
    RowArgs a{};
    a.rows = rows;
    a.T = T; a.k = top_k; a.n_rows = static_cast<uint32_t>(n_rows);
    a.token_bytes = ld * esize;
    a.row_bytes = static_cast<uint32_t>(d * esize);
    return a;
}

// Blocks of about kRowThreads threads.  A row's units are dealt evenly to as few rounds of threads as fit a block (whole
// warps, so that a warp's accesses are neighbours); short rows share a block.
struct RowGrid { dim3 grid; int threads; };
int row_grid(RowArgs* a, int unit_bytes, RowGrid* g) {      // unit_bytes: what a thread takes at a time
    const int units = (static_cast<int>(a->row_bytes) + unit_bytes - 1) / unit_bytes;
    const int rounds = (units + kRowThreads - 1) / kRowThreads;
    a->threads_per_token = units <= 32 ? units : ((units + rounds - 1) / rounds + 31) / 32 * 32;
    int tokens = kRowThreads / a->threads_per_token;
    if (tokens > a->T) tokens = static_cast<int>(a->T);
    const int64_t blocks = (a->T + tokens - 1) / tokens;
    if (blocks > 0x7fffffff) return FP8MLP_ERR_SHAPE;
    g->grid = dim3(static_cast<unsigned>(blocks));
    g->threads = tokens * a->threads_per_token;
    return FP8MLP_OK;
}

template <typename T, int W, bool WEIGHTED, int S, int U>
int launch_combine(RowArgs a, cudaStream_t st) {
    RowGrid g;
    const int rg = row_grid(&a, W * 4 * U, &g);
    if (rg != FP8MLP_OK) return rg;
    FP8MLP_CUDA_CHECK(launch_chained(combine_kernel<T, W, WEIGHTED, S, U>, g.grid, g.threads, 0, st, a));
    FP8MLP_LAUNCH_CHECK();
    return FP8MLP_OK;
}

template <typename T, bool WEIGHTED>
int run_combine(const RowArgs& a, bool wide, cudaStream_t st) {
    if (!wide) return launch_combine<T, 4, WEIGHTED, 4, 1>(a, st);
    if (a.k == 1) return launch_combine<T, 8, WEIGHTED, 1, 2>(a, st);
    // As many slots at a time as leave the fewest places of the last batch empty, and of these the most.  8192 rows of
    // 4096 bf16 in us, 2 / 3 / 4 at a time (k = 1: one slot of two units 25.7, else 29.5 / 30.4 / 34.1):
    //   k = 2: 35.8 / 36.6 / 39.4   3: 48.1 / 42.8 / 45.3   4: 54.0 / 55.8 / 52.2   5: 66.6 / 62.7 / 67.8
    //   k = 6: 73.2 / 70.4 / 73.7   7: 85.8 / 82.7 / 80.9   8: 92.7 / 90.6 / 89.1
    int best = 4;
    for (int s = 3; s >= 2; --s)
        if ((a.k + s - 1) / s * s < (a.k + best - 1) / best * best) best = s;
    if (best == 4) return launch_combine<T, 8, WEIGHTED, 4, 1>(a, st);
    return best == 3 ? launch_combine<T, 8, WEIGHTED, 3, 1>(a, st) : launch_combine<T, 8, WEIGHTED, 2, 1>(a, st);
}

}  // namespace

}  // namespace fp8mlp

using namespace fp8mlp;

extern "C" int fp8mlp_dispatch_plan(int64_t T, int top_k, int n_experts, const int32_t* experts, int32_t* counts,
                                    int32_t* offsets, int32_t* rows, void* stream) {
    if (T < 0 || top_k < 1 || top_k > FP8MLP_MAX_TOP_K || n_experts < 1 || n_experts > FP8MLP_MAX_EXPERTS ||
        T > 0x7fffffff / top_k)
        return FP8MLP_ERR_SHAPE;
    if (counts == nullptr || offsets == nullptr || (T > 0 && (experts == nullptr || rows == nullptr || rows == experts)))
        return FP8MLP_ERR_ARG;
    if (!aligned(experts, 4) || !aligned(counts, 4) || !aligned(offsets, 4) || !aligned(rows, 4)) return FP8MLP_ERR_ALIGN;
    PlanArgs a{};
    a.experts = experts; a.counts = counts; a.offsets = offsets; a.rows = rows;
    a.n = T * top_k; a.E = n_experts;
    while ((1 << a.bits) < n_experts) ++a.bits;
    // Pieces of kPlanPiece slots fill kPlanFill warps of one CTA, then of a cluster, then more warps of it, and then grow.
    // A CTA's warps share the ballots' issue slots, so CTAs first: 32768 slots 6.1 / 4.3 / 4.3 us with 32 / 16 / 8 warps, 8192
    // slots of 256 experts 7.5 / 5.1 / 3.9 us.  Pieces of 64 slots take 5.0 and 3.6 us there, but 7.3 instead of 5.8 for 49152.
    int64_t workers = (a.n + kPlanPiece - 1) / kPlanPiece;
    int cluster = 1;
    int max_cluster = 8;
    if (workers > 8 * kPlanFill) {
        const int rc = plan_max_cluster(&max_cluster);
        if (rc != FP8MLP_OK) return rc;
    }
    while (cluster < max_cluster && workers > static_cast<int64_t>(cluster) * kPlanFill) cluster *= 2;
    int64_t key_warps = (workers + cluster - 1) / cluster;
    a.key_warps = static_cast<int>(key_warps < 1 ? 1 : key_warps > kPlanWarps ? kPlanWarps : key_warps);
    workers = static_cast<int64_t>(cluster) * a.key_warps;
    a.per_warp = ((a.n + workers - 1) / workers + 31) / 32 * 32;
    int warps = (n_experts + 31) / 32;                   // the scan takes a thread per expert
    if (warps < a.key_warps) warps = a.key_warps;
    const size_t smem = static_cast<size_t>(a.key_warps) * n_experts * sizeof(int32_t);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(cluster));
    cfg.blockDim = dim3(static_cast<unsigned>(warps * 32));
    cfg.dynamicSmemBytes = smem;
    cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = static_cast<unsigned>(cluster);
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    FP8MLP_CUDA_CHECK(cudaLaunchKernelEx(&cfg, plan_kernel, static_cast<const PlanArgs>(a)));
    FP8MLP_LAUNCH_CHECK();
    return FP8MLP_OK;
}

extern "C" int fp8mlp_dispatch(int64_t T, int top_k, int64_t d, int dtype, const void* x, int64_t ld_x, const int32_t* rows,
                               void* xe, int64_t n_rows, void* stream) {
    const int rc = check_rows(T, top_k, d, dtype, x, ld_x, xe, n_rows, rows);
    if (rc != FP8MLP_OK) return rc;
    if (T == 0 || n_rows == 0) return FP8MLP_OK;
    RowArgs a = row_args(T, top_k, d, dtype, ld_x, n_rows, rows);
    a.src = static_cast<const uint8_t*>(x);
    a.dst = static_cast<uint8_t*>(xe);
    const bool wide = aligned(x, 32) && aligned(xe, 32) && a.token_bytes % 32 == 0;
    RowGrid g;
    const int rg = row_grid(&a, wide ? 32 : 16, &g);
    if (rg != FP8MLP_OK) return rg;
    FP8MLP_CUDA_CHECK(launch_chained(wide ? dispatch_kernel<8> : dispatch_kernel<4>, g.grid, g.threads, 0,
                                     static_cast<cudaStream_t>(stream), a));
    FP8MLP_LAUNCH_CHECK();
    return FP8MLP_OK;
}

extern "C" int fp8mlp_combine(int64_t T, int top_k, int64_t d, int dtype, const void* ye, int64_t n_rows, const int32_t* rows,
                              const float* weights, void* y, int64_t ld_y, void* stream) {
    const int rc = check_rows(T, top_k, d, dtype, y, ld_y, ye, n_rows, rows);
    if (rc != FP8MLP_OK) return rc;
    if (!aligned(weights, 4)) return FP8MLP_ERR_ALIGN;
    if (T == 0) return FP8MLP_OK;
    RowArgs a = row_args(T, top_k, d, dtype, ld_y, n_rows, rows);
    a.src = static_cast<const uint8_t*>(ye);
    a.dst = static_cast<uint8_t*>(y);
    a.weights = weights;
    const bool wide = aligned(y, 32) && aligned(ye, 32) && a.token_bytes % 32 == 0;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dtype == FP8MLP_F32) return weights != nullptr ? run_combine<float, true>(a, wide, st) : run_combine<float, false>(a, wide, st);
    return weights != nullptr ? run_combine<uint16_t, true>(a, wide, st) : run_combine<uint16_t, false>(a, wide, st);
}

extern "C" int fp8mlp_combine_backward(int64_t T, int top_k, int64_t d, int dtype, const void* dy, int64_t ld_dy,
                                       const void* ye, int64_t n_rows, const int32_t* rows, const float* weights, void* dye,
                                       float* d_weights, void* stream) {
    const int rc = check_rows(T, top_k, d, dtype, dy, ld_dy, ye, n_rows, rows);
    if (rc != FP8MLP_OK) return rc;
    if (T == 0) return FP8MLP_OK;
    if (weights == nullptr || d_weights == nullptr || (n_rows > 0 && (dye == nullptr || dye == ye || dye == dy)))
        return FP8MLP_ERR_ARG;
    if (!aligned(dye, 16) || !aligned(weights, 4) || !aligned(d_weights, 4)) return FP8MLP_ERR_ALIGN;
    RowArgs a = row_args(T, top_k, d, dtype, ld_dy, n_rows, rows);
    a.src = static_cast<const uint8_t*>(ye);
    a.dst = static_cast<uint8_t*>(dye);
    a.dy = static_cast<const uint8_t*>(dy);
    a.weights = weights;
    a.d_weights = d_weights;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const dim3 grid(static_cast<unsigned>(T));
    const bool wide = aligned(dy, 32) && aligned(ye, 32) && aligned(dye, 32) && a.token_bytes % 32 == 0;
    const int units = static_cast<int>(a.row_bytes / (wide ? 32 : 16)), rounds = (units + kRowThreads - 1) / kRowThreads;
    const int threads = ((units + rounds - 1) / rounds + 31) / 32 * 32;
    auto kernel = dtype == FP8MLP_F32 ? (wide ? combine_backward_kernel<float, 8> : combine_backward_kernel<float, 4>)
                                      : (wide ? combine_backward_kernel<uint16_t, 8> : combine_backward_kernel<uint16_t, 4>);
    FP8MLP_CUDA_CHECK(launch_chained(kernel, grid, threads, 0, st, a));
    FP8MLP_LAUNCH_CHECK();
    return FP8MLP_OK;
}
