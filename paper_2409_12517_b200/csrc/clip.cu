// Global gradient norm over many tensors, and clipping to it.
//
// The list travels in the kernel's parameters, cut into chunks that are numbered through and dealt to the blocks whatever
// tensor they belong to, so a thousand small tensors cost one launch and no block waits for a large one.
//
// The norm reads every byte once (541 MB fp32: 79 us, 6.9 TB/s; 271 MB bf16: 41 us).  Clipping has to know the norm before it
// writes, so it reads them again: three passes over the bytes, less what L2 keeps (541 MB: 243 us, at the measured copy rate
// the three passes less 64 MB would take 238).  The Adam pass can apply the coefficient instead and saves two of the three.
#include <cmath>

#include "common.cuh"

namespace fp8mlp {

namespace {

constexpr uint32_t kAll = 0xffffffffu;
constexpr int kClipThreads = 256;
constexpr int kClipBlocksPerSm = 4;
constexpr int kClipMaxBlocks = FP8MLP_NORM_WORKSPACE_BYTES / 8;    // one fp64 partial each
constexpr int kUnroll = 4;                                         // 32-byte accesses in flight per thread (2: 1 % slower)
constexpr int64_t kChunkUnits = kClipThreads * kUnroll;            // 32-byte units of a chunk
constexpr float kNormEps = 1e-6f;
// The clipping pass walks the chunks from the last to the first: it finds what the norm pass read last still in L2.  So that
// this is not pushed out, only the last 64 MB (of 126) are read to stay, all else is marked as the first to go.
constexpr uint32_t kKeepChunks = (64u << 20) / (32 * kChunkUnits);

struct ClipSeg {
    const uint8_t* g;
    uint8_t* out;
    int64_t n;
    uint32_t first_chunk;
    int32_t f32;
};
// kCap tensors per launch
template <int kCap> struct ClipArgs {
    double* partial;
    float* norm_coef;
    float max_norm;
    int n_partial, count, inf, accumulate;
    uint32_t chunks;
    ClipSeg seg[kCap];
};

template <typename SRC> struct GradUnit;                           // a unit is 32 bytes
template <> struct GradUnit<float> { static constexpr int kElems = 8; };
template <> struct GradUnit<uint16_t> { static constexpr int kElems = 16; };
__device__ __forceinline__ float as_float(float v) { return v; }
__device__ __forceinline__ float as_float(uint16_t v) { return __uint_as_float(static_cast<uint32_t>(v) << 16); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(uint16_t* p, float v) { *p = static_cast<uint16_t>(cvt_bf16x2(v, 0.0f) & 0xffffu); }

template <typename SRC> __device__ __forceinline__ void unpack_unit(const uint32_t (&w)[8], float (&v)[GradUnit<SRC>::kElems]);
template <> __device__ __forceinline__ void unpack_unit<float>(const uint32_t (&w)[8], float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
}
template <> __device__ __forceinline__ void unpack_unit<uint16_t>(const uint32_t (&w)[8], float (&v)[16]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) { v[2 * i] = bf16_lo(w[i]); v[2 * i + 1] = bf16_hi(w[i]); }
}

// Squares are summed in fp64.  Converting every element costs more than the addition (16 conversions a clock and SM), so a
// whole unit is first summed in fp32, as a tree (at most 4 roundings of 2^-24 one after the other), and taken as that if it
// lies well inside fp32's range; else - large or tiny values, zeros, infinities, NaN - its elements go in one by one, exact.
// The maximum norm keeps the bit pattern of |g|, which orders like an unsigned integer with NaN above infinity, so a NaN
// survives it.
template <bool INF> struct NormAcc;
template <> struct NormAcc<false> {
    double sum = 0.0;
    __device__ __forceinline__ void add(float v) { sum = fma(static_cast<double>(v), static_cast<double>(v), sum); }
    template <int N> __device__ __forceinline__ void add_unit(const float (&v)[N]) {
        float t[N / 2];
#pragma unroll
        for (int i = 0; i < N / 2; ++i) t[i] = fmaf(v[2 * i], v[2 * i], __fmul_rn(v[2 * i + 1], v[2 * i + 1]));
#pragma unroll
        for (int m = N / 4; m > 0; m >>= 1)
#pragma unroll
            for (int i = 0; i < m; ++i) t[i] = t[i] + t[i + m];
        if (t[0] > 0x1p-100f && t[0] < 0x1p+126f) {
            sum += static_cast<double>(t[0]);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) add(v[i]);
        }
    }
    __device__ __forceinline__ double word() const { return sum; }
};
template <> struct NormAcc<true> {
    uint32_t top = 0;
    __device__ __forceinline__ void add(float v) { top = max(top, __float_as_uint(v) & 0x7fffffffu); }
    template <int N> __device__ __forceinline__ void add_unit(const float (&v)[N]) {
#pragma unroll
        for (int i = 0; i < N; ++i) add(v[i]);
    }
    __device__ __forceinline__ double word() const { return __longlong_as_double(static_cast<long long>(top)); }
};

// Loads of 32 bytes whose line is the first to be replaced in L2
__device__ __forceinline__ void ld_stream_v8(const void* p, uint32_t (&w)[8]) {
    asm volatile("ld.global.L2::evict_first.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                 : "l"(p) : "memory");
}

// The tensor's elements lie in units of 32 bytes counted from the 32-byte boundary at or before its first element, so
// every whole unit is one aligned access whatever the tensor's own alignment.  The part units at its two ends go element
// by element, a thread each.  Chunks inside the tensor need no comparison per unit.
template <typename SRC> struct ChunkView {
    static constexpr int N = GradUnit<SRC>::kElems;
    const SRC* base;
    int64_t lead, last, first;     // first and one past the last element, the chunk's first, all counted from base
    bool whole;
    __device__ __forceinline__ ChunkView(const ClipSeg& s, uint32_t chunk) {
        lead = static_cast<int64_t>(reinterpret_cast<uintptr_t>(s.g) & 31u) / static_cast<int64_t>(sizeof(SRC));
        base = reinterpret_cast<const SRC*>(s.g) - lead;
        last = lead + s.n;
        first = static_cast<int64_t>(chunk) * kChunkUnits * N;
        whole = first >= lead && first + kChunkUnits * N <= last;
    }
    // this thread's k-th unit, and whether all of it belongs to the tensor
    __device__ __forceinline__ int64_t unit(int k) const { return first + (static_cast<int64_t>(k) * kClipThreads + threadIdx.x) * N; }
    __device__ __forceinline__ bool full(int64_t e) const { return e >= lead && e + N <= last; }
    // calls f(e) for this thread's elements of the part units in this chunk
    template <typename F> __device__ __forceinline__ void part_units(F f) const {
        if (threadIdx.x >= 2 * N) return;
        const bool tail = threadIdx.x >= N;
        const int64_t u = tail ? last / N * N : 0;                             // the unit that the tensor ends in, starts in
        const int64_t e = u + (threadIdx.x & (N - 1));
        const bool part = !full(u) && u >= first && u < first + kChunkUnits * N && !(tail && u == 0);   // one unit: once
        if (part && e >= lead && e < last) f(e);
    }
};

template <typename SRC, bool INF>
__device__ __forceinline__ void norm_chunk(const ClipSeg& s, uint32_t chunk, bool keep, NormAcc<INF>& acc) {
    constexpr int N = GradUnit<SRC>::kElems;
    const ChunkView<SRC> c(s, chunk);
    uint32_t w[kUnroll][8];
    if (c.whole) {
        const SRC* p = c.base + c.unit(0);
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) {
            if (keep) ld_global_nc_v8(p + k * kClipThreads * N, w[k]);
            else ld_stream_v8(p + k * kClipThreads * N, w[k]);
        }
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) {
            float v[N];
            unpack_unit<SRC>(w[k], v);
            acc.add_unit(v);
        }
    } else {
        c.part_units([&](int64_t e) { acc.add(as_float(c.base[e])); });
#pragma unroll 2
        for (int k = 0; k < kUnroll; ++k) {
            if (!c.full(c.unit(k))) continue;
            float v[N];
            ld_global_nc_v8(c.base + c.unit(k), w[0]);
            unpack_unit<SRC>(w[0], v);
            acc.add_unit(v);
        }
    }
}

template <typename SRC> __device__ __forceinline__ void scale_unit(uint32_t (&w)[8], float coef) {
    constexpr int N = GradUnit<SRC>::kElems;
    float v[N];
    unpack_unit<SRC>(w, v);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = __fmul_rn(v[i], coef);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (N == 8) w[i] = __float_as_uint(v[i]);
        else w[i] = cvt_bf16x2(v[2 * i], v[2 * i + 1]);
    }
}

// COEF() gives the coefficient; it is asked for after the loads of a whole chunk have been issued.
// EARLY: it is at hand, and asked for before the loads of a tensor that is clipped in place, which needs none where it is 1
// (541 MB in place: 91 us instead of 141, and 233 as before where it is below 1).
template <typename SRC, bool EARLY, typename COEF>
__device__ __forceinline__ void clip_chunk(const ClipSeg& s, uint32_t chunk, COEF coef_of) {
    if (EARLY && s.out == s.g && coef_of() == 1.0f) return;
    constexpr int N = GradUnit<SRC>::kElems;
    const ChunkView<SRC> c(s, chunk);
    SRC* const out = reinterpret_cast<SRC*>(s.out) - c.lead;
    if (((reinterpret_cast<uintptr_t>(s.out) ^ reinterpret_cast<uintptr_t>(s.g)) & 31u) == 0) {
        uint32_t w[kUnroll][8];
        if (c.whole) {
            const SRC* p = c.base + c.unit(0);
#pragma unroll
            for (int k = 0; k < kUnroll; ++k) ld_stream_v8(p + k * kClipThreads * N, w[k]);
        } else {
#pragma unroll
            for (int k = 0; k < kUnroll; ++k)
                if (c.full(c.unit(k))) ld_global_v8(c.base + c.unit(k), w[k]);
        }
        const float coef = coef_of();
        if (coef == 1.0f && s.out == s.g) return;
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) scale_unit<SRC>(w[k], coef);
        if (c.whole) {
            SRC* q = out + c.unit(0);
#pragma unroll
            for (int k = 0; k < kUnroll; ++k) st_global_v8(q + k * kClipThreads * N, w[k]);
        } else {
#pragma unroll
            for (int k = 0; k < kUnroll; ++k)
                if (c.full(c.unit(k))) st_global_v8(out + c.unit(k), w[k]);
            c.part_units([&](int64_t e) { put(out + e, __fmul_rn(as_float(c.base[e]), coef)); });
        }
    } else {
        // Buffers whose alignments differ: one element per thread at a time, neighbours in neighbouring threads.
        const float coef = coef_of();
        const int64_t stop = c.first + kChunkUnits * N < c.last ? c.first + kChunkUnits * N : c.last;
#pragma unroll 8
        for (int64_t e = (c.first > c.lead ? c.first : c.lead) + threadIdx.x; e < stop; e += kClipThreads)
            put(out + e, __fmul_rn(as_float(c.base[e]), coef));
    }
}

// the tensor that chunk c belongs to
template <int kCap>
__device__ __forceinline__ int find_seg(const ClipArgs<kCap>& a, uint32_t c) {
    int lo = 0, hi = a.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.seg[mid].first_chunk <= c) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ double block_reduce(double v, bool inf, double* part) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const double w = __shfl_xor_sync(kAll, v, o);
        v = inf ? __longlong_as_double(max(__double_as_longlong(v), __double_as_longlong(w))) : v + w;
    }
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int i = 1; i < kClipThreads / 32; ++i)
        v = inf ? __longlong_as_double(max(__double_as_longlong(v), __double_as_longlong(part[i]))) : v + part[i];
    return v;
}

// A block's partial: the sum of its squares, or the bit pattern of its maximum (kept as an integer in the fp64 word).
template <int kCap, bool INF>
__global__ void __launch_bounds__(kClipThreads, kClipBlocksPerSm) norm_kernel(const __grid_constant__ ClipArgs<kCap> a) {
    __shared__ double part[kClipThreads / 32];
    grid_dependency_wait();
    grid_launch_dependents();
    NormAcc<INF> acc;
    for (uint32_t c = blockIdx.x; c < a.chunks; c += gridDim.x) {
        const ClipSeg& s = a.seg[find_seg(a, c)];
        const bool keep = a.chunks - c <= kKeepChunks;
        if (s.f32) norm_chunk<float, INF>(s, c - s.first_chunk, keep, acc);
        else norm_chunk<uint16_t, INF>(s, c - s.first_chunk, keep, acc);
    }
    double v = block_reduce(acc.word(), INF, part);
    if (threadIdx.x == 0) {
        if (a.accumulate) {      // a further launch of the same call (a list longer than one launch holds)
            const double w = a.partial[blockIdx.x];
            v = INF ? __longlong_as_double(max(__double_as_longlong(v), __double_as_longlong(w))) : v + w;
        }
        a.partial[blockIdx.x] = v;
    }
}

// Every thread of the block returns (norm, coef), from all partials in their fixed order.
__device__ __forceinline__ float2 finish_norm(const double* partial, int n_partial, bool inf, float max_norm, double* part) {
    double v = 0.0;
    for (int i = threadIdx.x; i < n_partial; i += kClipThreads) {
        const double w = __ldcg(partial + i);
        v = inf ? __longlong_as_double(max(__double_as_longlong(v), __double_as_longlong(w))) : v + w;
    }
    v = block_reduce(v, inf, part);
    const float norm = inf ? __uint_as_float(static_cast<uint32_t>(__double_as_longlong(v))) : static_cast<float>(sqrt(v));
    const float q = __fdiv_rn(max_norm, norm + kNormEps);
    return make_float2(norm, q >= 1.0f ? 1.0f : q);       // a NaN is not >= 1 and stays
}

__global__ void __launch_bounds__(kClipThreads) norm_finish_kernel(const double* partial, int n_partial, int inf, float max_norm,
                                                                  float* norm_coef) {
    __shared__ double part[kClipThreads / 32];
    grid_dependency_wait();
    grid_launch_dependents();
    const float2 r = finish_norm(partial, n_partial, inf != 0, max_norm, part);
    if (threadIdx.x == 0) { norm_coef[0] = r.x; norm_coef[1] = r.y; }
}

// One block per chunk, the last chunk first.  FINISH: every block sums the partials itself, behind its loads (short lists,
// where a launch in between costs more); otherwise the norm and coefficient are there already.
template <int kCap, bool FINISH>
__global__ void __launch_bounds__(kClipThreads, kClipBlocksPerSm) clip_kernel(const __grid_constant__ ClipArgs<kCap> a) {
    __shared__ double part[kClipThreads / 32];
    grid_dependency_wait();
    grid_launch_dependents();
    auto coef_of = [&]() {
        if constexpr (FINISH) {
            const float2 r = finish_norm(a.partial, a.n_partial, a.inf != 0, a.max_norm, part);
            if (blockIdx.x == 0 && threadIdx.x == 0) { a.norm_coef[0] = r.x; a.norm_coef[1] = r.y; }
            return r.y;
        } else {
            return a.norm_coef[1];              // an SM reads it once: later blocks find it in L1
        }
    };
    if (a.chunks == 0u) {                       // nothing to scale, but a norm to report
        if (FINISH) coef_of();
        return;
    }
    const uint32_t c = a.chunks - 1u - blockIdx.x;
    const ClipSeg& s = a.seg[find_seg(a, c)];
    if (s.f32) clip_chunk<float, !FINISH>(s, c - s.first_chunk, coef_of);
    else clip_chunk<uint16_t, !FINISH>(s, c - s.first_chunk, coef_of);
}

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

int64_t seg_chunks(const fp8mlp_grad_tensor& g) {
    const int64_t esize = g.dtype == FP8MLP_F32 ? 4 : 2;
    const int64_t bytes = static_cast<int64_t>(reinterpret_cast<uintptr_t>(g.g) & 31u) + g.n * esize;
    return g.n == 0 ? 0 : (bytes + 32 * kChunkUnits - 1) / (32 * kChunkUnits);
}

struct ClipCall {
    const fp8mlp_grad_tensor* grads;
    int count, inf;
    float max_norm;
    float* norm_coef;
    double* partial;
    int blocks;
    bool finish_in_clip;
    cudaStream_t st;
};

// One launch over grads[from, to); CLIP: the scaling pass, otherwise the norm pass.
template <bool CLIP, int kCap>
int clip_launch(const ClipCall& c, int from, int to) {
    ClipArgs<kCap> a;
    a.partial = c.partial; a.norm_coef = c.norm_coef; a.max_norm = c.max_norm;
    a.n_partial = c.blocks; a.inf = c.inf; a.accumulate = from > 0;
    int64_t chunks = 0;
    int m = 0;
    for (int i = from; i < to; ++i) {
        const fp8mlp_grad_tensor& g = c.grads[i];
        if (g.n == 0) continue;
        ClipSeg& s = a.seg[m++];
        s.g = static_cast<const uint8_t*>(g.g);
        s.out = static_cast<uint8_t*>(g.out);
        s.n = g.n;
        s.first_chunk = static_cast<uint32_t>(chunks);
        s.f32 = g.dtype == FP8MLP_F32;
        chunks += seg_chunks(g);
    }
    a.count = m;
    a.chunks = static_cast<uint32_t>(chunks);
    if constexpr (CLIP) {
        auto kernel = c.finish_in_clip ? clip_kernel<kCap, true> : clip_kernel<kCap, false>;
        FP8MLP_CUDA_CHECK(launch_chained(kernel, chunks > 0 ? static_cast<unsigned>(chunks) : 1u, kClipThreads, 0, c.st, a));
    } else {
        auto kernel = c.inf ? norm_kernel<kCap, true> : norm_kernel<kCap, false>;
        FP8MLP_CUDA_CHECK(launch_chained(kernel, c.blocks, kClipThreads, 0, c.st, a));
    }
    FP8MLP_LAUNCH_CHECK();
    return FP8MLP_OK;
}

// Tensors a launch holds: 4 or 31 KB of parameters, whose copy makes a launch take the host 1.8 or 3.8 us (0.7 KB: also 1.8).
constexpr int kCapSmall = 120, kCapLarge = 960;

template <bool CLIP>
int clip_range(const ClipCall& c, int from) {
    const int to = c.count - from < kCapLarge ? c.count : from + kCapLarge;
    return to - from <= kCapSmall ? clip_launch<CLIP, kCapSmall>(c, from, to) : clip_launch<CLIP, kCapLarge>(c, from, to);
}

int clip_run(const fp8mlp_grad_tensor* grads, int count, int kind, float max_norm, float* norm_coef, void* workspace, bool clip,
             void* stream) {
    if (kind != FP8MLP_NORM_L2 && kind != FP8MLP_NORM_INF) return FP8MLP_ERR_ARG;
    if (count < 0 || (count > 0 && grads == nullptr) || norm_coef == nullptr || workspace == nullptr || !(max_norm >= 0.0f))
        return FP8MLP_ERR_ARG;
    int64_t chunks = 0;
    for (int i = 0; i < count; ++i) {
        const fp8mlp_grad_tensor& g = grads[i];
        if (g.dtype != FP8MLP_BF16 && g.dtype != FP8MLP_F32) return FP8MLP_ERR_ARG;
        if (g.n < 0 || g.n > (int64_t(1) << 40)) return FP8MLP_ERR_SHAPE;
        if (g.n == 0) continue;
        if (g.g == nullptr || (clip && g.out == nullptr)) return FP8MLP_ERR_ARG;
        const uintptr_t esize = g.dtype == FP8MLP_F32 ? 4 : 2;
        if (!aligned(g.g, esize) || (clip && !aligned(g.out, esize))) return FP8MLP_ERR_ALIGN;
        chunks += seg_chunks(g);
        if (chunks > 0x7fffffff) return FP8MLP_ERR_SHAPE;
    }
    if (!aligned(norm_coef, 4) || !aligned(workspace, 16)) return FP8MLP_ERR_ALIGN;
    int dev = 0, sms = 0;
    FP8MLP_CUDA_CHECK(cudaGetDevice(&dev));
    FP8MLP_CUDA_CHECK(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    ClipCall c{grads, count, kind == FP8MLP_NORM_INF, max_norm, norm_coef, static_cast<double*>(workspace), 0,
               false, static_cast<cudaStream_t>(stream)};
    int64_t blocks = static_cast<int64_t>(sms) * kClipBlocksPerSm;
    if (blocks > kClipMaxBlocks) blocks = kClipMaxBlocks;
    if (blocks > chunks) blocks = chunks > 0 ? chunks : 1;
    c.blocks = static_cast<int>(blocks);
    for (int from = 0; from == 0 || from < count; from += kCapLarge) {
        const int rc = clip_range<false>(c, from);
        if (rc != FP8MLP_OK) return rc;
    }
    // A norm launch of its own between the passes costs 0.8 us; summing the partials in every block costs more than that
    // once there are more chunks than resident blocks (2 MB: 4.9 us in the blocks, 5.7 apart; 57 MB: 29.5 and 27.9).
    c.finish_in_clip = clip && chunks <= blocks && count <= kCapLarge;
    if (!c.finish_in_clip) {
        FP8MLP_CUDA_CHECK(launch_chained(norm_finish_kernel, 1, kClipThreads, 0, c.st, static_cast<const double*>(c.partial), c.blocks,
                                         c.inf, max_norm, norm_coef));
        FP8MLP_LAUNCH_CHECK();
    }
    if (clip) {
        for (int from = count > 0 ? (count - 1) / kCapLarge * kCapLarge : 0; from >= 0; from -= kCapLarge) {
            const int rc = clip_range<true>(c, from);
            if (rc != FP8MLP_OK) return rc;
        }
    }
    return FP8MLP_OK;
}

}  // namespace

}  // namespace fp8mlp

using namespace fp8mlp;

extern "C" int fp8mlp_grad_norm(const fp8mlp_grad_tensor* grads, int count, int norm_kind, float max_norm, float* norm_coef,
                                void* workspace, void* stream) {
    return clip_run(grads, count, norm_kind, max_norm, norm_coef, workspace, false, stream);
}

extern "C" int fp8mlp_clip_grads(const fp8mlp_grad_tensor* grads, int count, int norm_kind, float max_norm, float* norm_coef,
                                 void* workspace, void* stream) {
    return clip_run(grads, count, norm_kind, max_norm, norm_coef, workspace, true, stream);
}
