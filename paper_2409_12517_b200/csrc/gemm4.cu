// Product of two 4-bit operands with block scales: tcgen05.mma kind::mxf4 / kind::mxf4nvf4 on operands streamed by TMA, block
// scales brought from shared into tensor memory next to the accumulators, fp32 accumulation.
//
//   D[p, q] = sum_k P(p, k) Q(q, k)          P: the operand whose rows are the accumulator's rows (128 per CTA)
//
// P is A and Q is B, or the other way round where A has few rows: a product of one token with a large weight matrix is bound by
// reading the weights, so their rows fill the 128 accumulator rows and the tokens are its 16 to 128 columns.
//
// A CTA is two TMA warps, which take turns, one warp that issues the MMAs and 4 or 8 epilogue warps.  A stage is 512 cycles of MMAs
// at most, and the loops of the first three must be shorter: a wait takes 100 cycles though nothing is to be waited for, a stage's
// loads 290 (one TMA warp of a pair could not keep up).  So the MMA warp has one barrier to look at, asks for the next stage's before
// it issues the present stage, and all of it walks the loop while one elected lane issues, for addresses and descriptors then are
// the warp's, as the tensor instructions need them (moving them over from a lane's registers: 115 cycles for each of 10 to 16
// instructions a stage).  A stage holds 256 columns of the contraction: 128 bytes of codes a row, and the scales' tiles of 512 bytes
// as they lie in memory (32 rows of 16 bytes), which tcgen05.cp copies to the four lane quadrants of 4 tensor-memory columns.
// Tensor memory holds the scales of every stage of the ring beside the accumulator.
//
// Large products: CTA pairs on 256 x 256 tiles (cta_group::2; each CTA loads its 128 rows of P, half of the rows of Q, and the
// scales of all of Q).  What bounds them is the way from L2 to the SMs, some 60 bytes a clock: 35 KB (MXFP4) a stage of 512 cycles
// of MMAs.  (256 x 192 tiles with two accumulators want 31 KB for 384: 8192 x 8192 x 16384 NVFP4 445 us, this way 360.)  The one
// accumulator goes to registers as a whole, so that the next tile's MMAs have it back at once; the loads, which set the pace, run on
// meanwhile.  The output leaves through shared memory in bulk stores (8192 x 8192 x 256: 49 us with stores of 32 bytes a lane, 26).
// Others: single CTAs, two to an SM, on one 128 x 16 .. 128 tile each; with few tiles the contraction is cut among the 2, 4 or 8
// CTAs of a cluster, which add their shares over distributed shared memory in the order of their ranks.
// Every wait is bounded; one that gives up raises the status word of products without a context.
#include "gemm.cuh"

#include <mutex>

namespace fp8mlp {

namespace {

constexpr int kRows = 128;                   // accumulator rows of a CTA
constexpr int kStageK = 256;                 // columns of the contraction per stage
constexpr int kStepK = 64;                   // and per MMA
constexpr int kScaleTile = 512;              // 128 rows x 4 blocks
constexpr uint32_t kAll = 0xffffffffu;
constexpr int kOtherWarps = 3;               // two TMA producers, the MMA issuer
__device__ int wait_status;                  // status word of these products, which have no context: a wait gave up

struct Gemm4Args {
    int P, Q, K;
    int p_tiles, q_tiles, stages_k;          // stages_k: stages of the whole contraction
    int split;                               // CTAs of a cluster that share a tile's contraction (at most stages_k)
    int group;                               // rasterisation: bands of this many p tiles
    int swap;                                // out is [Q, P]
    int f32, vec;                            // fp32 output; 16: its rows start on 16-byte boundaries
    const float *s0, *s1;
    uint8_t* out;
    int64_t ld_out;                          // elements
};

template <int FMT, int TN, bool PAIR> struct Shape {
    static constexpr int kBlock = FMT == FP8MLP_MXFP4 ? 32 : 16;
    static constexpr int kTiles = kStageK / (4 * kBlock);                 // scale tiles of a stage, per 128 rows
    static constexpr int kQGroups = (TN + 127) / 128;                     // 128-row groups of scales that a tile of Q touches
    static constexpr int kPBytes = kRows * 128, kQBytes = (PAIR ? TN / 2 : TN) * 128;
    static constexpr int kSfBytes = kTiles * kScaleTile;                  // per 128 rows
    static constexpr int kStageBytes = kPBytes + kQBytes + (1 + kQGroups) * kSfBytes;
    // A single CTA shares its SM with another that works while it starts or ends.
    static constexpr int kCtasPerSm = PAIR ? 1 : 2;
    static constexpr int kStoreBytes = PAIR ? 8 * 4096 : 0;               // staging of the output, 4 KB for each epilogue warp
    static constexpr int kFit = (232448 - 1024 - 256 - kStoreBytes) / kStageBytes;
    static constexpr int kStages = PAIR ? (kFit < 6 ? kFit : 6) : TN >= 64 ? 3 : 4;
    static constexpr int kEpiWarps = TN >= 64 ? 8 : 4;
    static constexpr int kThreads = 32 * (kOtherWarps + kEpiWarps);
    static constexpr int kWarpCols = TN / (kEpiWarps / 4);                // columns of a tile that an epilogue warp drains
    static constexpr int kSfCols = 4 * kTiles * (1 + kQGroups);           // tensor-memory columns of a stage's scales
    static constexpr int kCols = TN + kStages * kSfCols;                  // the accumulator and the scales of all stages
    static constexpr int kTmem = kCols <= 128 ? 128 : kCols <= 256 ? 256 : 512;
    static_assert(kCols <= 512 && kTmem * kCtasPerSm <= 512, "tensor memory");
};

struct __align__(8) Tail4 {
    uint64_t full[6], empty[6], tmem_full, tmem_empty;
    uint32_t tmem_base;
    int abort;
};

template <int FMT, int TN, bool PAIR>
constexpr size_t smem4_bytes() {
    return 1024 + size_t(Shape<FMT, TN, PAIR>::kStages) * Shape<FMT, TN, PAIR>::kStageBytes + Shape<FMT, TN, PAIR>::kStoreBytes + sizeof(Tail4);
}
static_assert(smem4_bytes<FP8MLP_NVFP4, 256, true>() <= 232448 && smem4_bytes<FP8MLP_MXFP4, 256, true>() <= 232448, "shared memory");
static_assert(2 * (smem4_bytes<FP8MLP_NVFP4, 128, false>() + 1024) <= 233472 && 2 * (smem4_bytes<FP8MLP_NVFP4, 32, false>() + 1024) <= 233472,
              "two single CTAs share an SM");

// Matrix descriptors: address / 16 in the low 14 bits, then (bit 16) a leading offset that neither layout uses, and in the
// upper half the distance of 8-row groups / 16, the version and the swizzle.
// Operand rows of 128 bytes with the 128-byte swizzle: 8-row groups 1024 bytes apart.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr16) {
    return (uint64_t((1024u >> 4) | (1u << 14) | (2u << 29)) << 32) | (addr16 | (1u << 16));
}
// A tile of scales, 32 rows of 16 bytes one after the other, no swizzle: 8-row groups 128 bytes apart.
__device__ __forceinline__ uint64_t scales_desc(uint32_t addr16) {
    return (uint64_t((128u >> 4) | (1u << 14)) << 32) | (addr16 | (1u << 16));
}
// The place in the ring of stages and the parity of its round.
template <int N> struct Ring {
    uint32_t stage = 0, phase = 0;
    __device__ __forceinline__ void next() {
        if (++stage == N) { stage = 0; phase ^= 1u; }
    }
};
// Whether a barrier's phase is complete, without waiting for it.
__device__ __forceinline__ bool mbar_peek(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}\n"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ uint32_t elect_one() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}\n" : "=r"(r));
    return r;
}
// 512 bytes of scales -> 4 columns of tensor memory, the same in each quadrant of 32 lanes
template <bool PAIR>
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint64_t desc) {
    if constexpr (PAIR) asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
    else asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
template <int FMT, bool PAIR>
__device__ __forceinline__ void umma_f4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sf_a, uint32_t sf_b, uint32_t accumulate) {
#define FP8MLP_UMMA4(GROUP, KIND, VEC)                                                                             \
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"                                                  \
                 "tcgen05.mma.cta_group::" GROUP ".kind::" KIND ".block_scale.scale_vec::" VEC " [%0], %1, %2, %3, [%4], [%5], p;\n\t}\n" \
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sf_a), "r"(sf_b), "r"(accumulate) : "memory")
    if constexpr (FMT == FP8MLP_MXFP4) {
        if constexpr (PAIR) FP8MLP_UMMA4("2", "mxf4", "2X"); else FP8MLP_UMMA4("1", "mxf4", "2X");
    } else {
        if constexpr (PAIR) FP8MLP_UMMA4("2", "mxf4nvf4", "4X"); else FP8MLP_UMMA4("1", "mxf4nvf4", "4X");
    }
#undef FP8MLP_UMMA4
}
// Instruction descriptor: [7,10) and [10,12) element types (E2M1 = 1); [17,23) N >> 3; bit 23 scale type (E4M3 = 0, E8M0 = 1);
// [24,29) M >> 4; [29,31) and [4,6): byte of the 32-bit tensor-memory cell where A's and B's scales begin.
template <int FMT, int TN, bool PAIR>
__device__ __forceinline__ uint32_t idesc4(uint32_t sf_byte) {
    return (sf_byte << 4) | (1u << 7) | (1u << 10) | (uint32_t(TN >> 3) << 17) | (uint32_t(FMT == FP8MLP_MXFP4 ? 1 : 0) << 23) |
           (uint32_t((PAIR ? 256 : 128) >> 4) << 24) | (sf_byte << 29);
}

// Scales are a tensor of 128-byte rows, four to a tile, by the tiles of a row group, by the row groups.
__device__ __forceinline__ void tma_load_3d(uint32_t smem_dst, const CUtensorMap* m, uint32_t bar, int32_t x, int32_t y, int32_t z) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
        ::"r"(smem_dst), "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void tma_load_3d_pair(uint32_t smem_dst, const CUtensorMap* m, uint32_t bar_cluster, int32_t x, int32_t y, int32_t z) {
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
        ::"r"(smem_dst), "l"(reinterpret_cast<uint64_t>(m)), "r"(bar_cluster), "r"(x), "r"(y), "r"(z) : "memory");
}

// The scale copies and MMAs of one stage (FULL: all 256 columns of it; else the `left` that there are).
template <int FMT, int TN, bool PAIR, bool FULL>
__device__ __forceinline__ void issue_stage(uint32_t d_tmem, uint32_t base, uint32_t sf_base, uint32_t sf_p, uint32_t sf_q,
                                            uint32_t q_offset, bool accumulate, int left) {
    using S = Shape<FMT, TN, PAIR>;
#pragma unroll
    for (int t = 0; t < S::kTiles; ++t) {
        if (!FULL && t * 4 * S::kBlock >= left) break;
        copy_scales<PAIR>(sf_p + 4 * t, scales_desc(sf_base + t * (kScaleTile >> 4)));
#pragma unroll
        for (int j = 0; j < S::kQGroups; ++j)
            copy_scales<PAIR>(sf_q + 4 * (t * S::kQGroups + j), scales_desc(sf_base + ((1 + j) * S::kSfBytes + t * kScaleTile) / 16));
    }
#pragma unroll
    for (int k = 0; k < kStageK / kStepK; ++k) {
        if (!FULL && k * kStepK >= left) break;
        // a cell of four scales is 64 columns of NVFP4, and 128 of MXFP4, which take it in two halves
        const int t = FMT == FP8MLP_MXFP4 ? k / 2 : k;
        const uint32_t byte = FMT == FP8MLP_MXFP4 ? 2u * (k & 1) : 0u;
        umma_f4<FMT, PAIR>(d_tmem, operand_desc(base + 2 * k), operand_desc(base + (S::kPBytes >> 4) + 2 * k), idesc4<FMT, TN, PAIR>(byte),
                           sf_p + 4 * t, sf_q + 4 * t * S::kQGroups + q_offset, (accumulate || k != 0) ? 1u : 0u);
    }
}

template <bool PAIR>
__device__ __forceinline__ void tile4_coords(const Gemm4Args& p, int tile, int& p_tile, int& q_tile) {
    if constexpr (!PAIR) {                       // all on the SMs at once, or nearly: any order does
        q_tile = p.q_tiles == 1 ? 0 : tile / p.p_tiles;
        p_tile = tile - q_tile * p.p_tiles;
        return;
    }
    const int per_band = p.group * p.q_tiles, band = tile / per_band, first = band * p.group;
    const int rows = min(p.p_tiles - first, p.group), in_band = tile - band * per_band;
    p_tile = first + in_band % rows;
    q_tile = in_band / rows;
}

template <int N>
__device__ __forceinline__ void tmem_ld_cols(uint32_t taddr, uint32_t (&r)[N]) {
    if constexpr (N == 32) {
        tmem_ld32(taddr, r);
    } else {
        static_assert(N == 16, "16 or 32 columns");
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                       "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                     : "r"(taddr) : "memory");
    }
}

__device__ __forceinline__ void store_one(const Gemm4Args& p, int64_t at, float v) {
    if (p.f32) reinterpret_cast<float*>(p.out)[at] = v;
    else reinterpret_cast<uint16_t*>(p.out)[at] = static_cast<uint16_t>(cvt_bf16x2(v, 0.0f) & 0xffffu);
}

// N neighbouring outputs of a row, `have` of them inside the matrix
template <int N>
__device__ __forceinline__ void store_cols(const Gemm4Args& p, int64_t at, const float (&v)[N], int have) {
    if (have < N || p.vec != 16) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < have) store_one(p, at + i, v[i]);
    } else if (p.f32) {
        float* dst = reinterpret_cast<float*>(p.out) + at;
#pragma unroll
        for (int i = 0; i < N; i += 4)
            st_global_v4(dst + i, __float_as_uint(v[i]), __float_as_uint(v[i + 1]), __float_as_uint(v[i + 2]), __float_as_uint(v[i + 3]));
    } else {
        uint16_t* dst = reinterpret_cast<uint16_t*>(p.out) + at;
#pragma unroll
        for (int i = 0; i < N; i += 8)
            st_global_v4(dst + i, cvt_bf16x2(v[i], v[i + 1]), cvt_bf16x2(v[i + 2], v[i + 3]), cvt_bf16x2(v[i + 4], v[i + 5]), cvt_bf16x2(v[i + 6], v[i + 7]));
    }
}

// 32 columns of a warp's 32 rows (a lane has a row) into its 4 KB of staging: rows of 128 bytes (fp32) or 64 (bf16), their 16-byte
// pieces swizzled as a tensor map with rows of that length does it.
__device__ __forceinline__ void stage_rows(bool f32, uint32_t block, int lane, const float (&v)[32]) {
    if (f32) {
#pragma unroll
        for (int c = 0; c < 8; ++c)
            st_shared_v4(block + lane * 128u + ((c ^ (lane & 7)) << 4), __float_as_uint(v[4 * c]), __float_as_uint(v[4 * c + 1]),
                         __float_as_uint(v[4 * c + 2]), __float_as_uint(v[4 * c + 3]));
    } else {
#pragma unroll
        for (int c = 0; c < 4; ++c)
            st_shared_v4(block + lane * 64u + ((c ^ ((lane >> 1) & 3)) << 4), cvt_bf16x2(v[8 * c], v[8 * c + 1]), cvt_bf16x2(v[8 * c + 2], v[8 * c + 3]),
                         cvt_bf16x2(v[8 * c + 4], v[8 * c + 5]), cvt_bf16x2(v[8 * c + 6], v[8 * c + 7]));
    }
}

// Rows on 16-byte boundaries: one lane sends the block off as a bulk tensor store, which cuts off what lies outside the matrix, but
// along a row in pieces of 16 bytes: a row's end inside such a piece is for write_rows.
__device__ __forceinline__ void send_rows(const CUtensorMap* out, bool f32, uint32_t stage, uint32_t& sent, int lane, int row, int col,
                                          const float (&v)[32]) {
    if (!f32) stage += (sent++ & 1u) * 2048u;                 // the staging holds two blocks of bf16, one of fp32
    if (lane == 0) {                                          // the store that used this block last has read it
        if (f32) tma_store_wait_read<0>(); else tma_store_wait_read<1>();
    }
    __syncwarp();
    stage_rows(f32, stage, lane, v);
    fence_smem_to_async_proxy();
    __syncwarp();
    if (lane == 0) {
        tma_store_2d(out, stage, col, row);
        tma_store_commit();
    }
}

__device__ __forceinline__ uint32_t shared_word(uint32_t at) {
    uint32_t w;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w) : "r"(at) : "memory");
    return w;
}

// Rows on any boundary, `rows` x `cols` of the block inside the matrix: each row is written by neighbouring lanes, in words of four
// bytes (16384 x 1411 bf16 with a row per lane, element by element: 234 us; this way 74, with write_wide 39; behind large products,
// when power holds the clock down, 48 to 52).
__device__ __forceinline__ void write_rows(const Gemm4Args& p, uint32_t stage, int lane, int row, int col, int rows, int cols,
                                           const float (&v)[32]) {
    if (lane == 0) tma_store_wait_read<0>();
    __syncwarp();                                             // the last block has been read
    stage_rows(p.f32 != 0, stage, lane, v);
    __syncwarp();
    constexpr int kBatch = 8;                                 // loads under way together
    if (p.f32) {
        float* dst = reinterpret_cast<float*>(p.out) + static_cast<int64_t>(row) * p.ld_out + col + lane;
#pragma unroll 1
        for (int r0 = 0; r0 < rows; r0 += kBatch) {
            uint32_t w[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) w[k] = shared_word(stage + (r0 + k) * 128u + (((lane >> 2) ^ k) << 4) + (lane & 3) * 4u);
#pragma unroll
            for (int k = 0; k < kBatch; ++k)
                if (lane < cols && r0 + k < rows) dst[(r0 + k) * p.ld_out] = __uint_as_float(w[k]);
        }
    } else {
        // two rows at a time, 16 lanes each; a row on an odd element begins with one element, and every lane's word is the upper
        // half of its own and the lower half of the next one's
        const int l = lane & 15;
        uint16_t* base = reinterpret_cast<uint16_t*>(p.out) + static_cast<int64_t>(row + (lane >> 4)) * p.ld_out + col;
#pragma unroll 1
        for (int r0 = 0; r0 < rows; r0 += 2 * kBatch) {
            uint32_t w[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const int r = r0 + 2 * k + (lane >> 4);
                w[k] = shared_word(stage + r * 64u + (((l >> 2) ^ (k & 3)) << 4) + (l & 3) * 4u);
            }
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                uint16_t* dst = base + (r0 + 2 * k) * p.ld_out;
                const bool odd = (reinterpret_cast<uintptr_t>(dst) & 2) != 0, here = r0 + 2 * k + (lane >> 4) < rows;
                const uint32_t next = __shfl_down_sync(kAll, w[k], 1, 16), pair = odd ? __funnelshift_r(w[k], next, 16) : w[k];
                const int c = 2 * l + (odd ? 1 : 0);            // the columns of `pair`: c, c + 1
                if (here && c + 1 < cols && c + 1 < 32) *reinterpret_cast<uint32_t*>(dst + c) = pair;
                else if (here && c < cols) dst[c] = static_cast<uint16_t>(pair & 0xffffu);
                if (here && odd && l == 0) dst[0] = static_cast<uint16_t>(w[k] & 0xffffu);
            }
        }
    }
}

// The same for 128 bf16 columns, all inside the matrix, with stores of 16 bytes: 16 lanes take a row, each a piece of 8 elements that
// begins on a 16-byte boundary of the output, i.e. the row's elements from head + 8 l on, put together from the staged pieces l and
// l + 1; what is left at the ends of the row, 8 elements in all, goes one by one.  16 rows at a time in the 4 KB of staging.
__device__ __forceinline__ void write_wide(const Gemm4Args& p, uint32_t stage, int lane, int row, int col, int rows, const uint32_t (&w)[64]) {
    constexpr int kBatch = 2;
    const int l = lane & 15;
#pragma unroll
    for (int pass = 0; pass < 2; ++pass) {
        __syncwarp();                                         // the last block has been read
        if ((lane >> 4) == pass)
#pragma unroll
            for (int c = 0; c < 16; ++c) st_shared_v4(stage + l * 256u + ((c ^ l) << 4), w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]);
        __syncwarp();
#pragma unroll
        for (int r0 = 0; r0 < 16; r0 += 2 * kBatch) {         // the loads of a batch of rows are under way together
            uint4 own[kBatch];
            uint32_t edge[kBatch];
            int head[kBatch];
            uint16_t* dst[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const int r = r0 + 2 * k + (lane >> 4);
                dst[k] = reinterpret_cast<uint16_t*>(p.out) + static_cast<int64_t>(row + 16 * pass + r) * p.ld_out + col;
                head[k] = static_cast<int>((0u - static_cast<uint32_t>(reinterpret_cast<uintptr_t>(dst[k]) >> 1)) & 7u);
                own[k] = ld_shared_v4(stage + r * 256u + ((l ^ r) << 4));
                const int e = l < head[k] ? l : 120 + (l & 7);
                edge[k] = shared_word(stage + r * 256u + (((e >> 3) ^ r) << 4) + ((e & 7) >> 1) * 4u) >> (16 * (e & 1));
            }
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const bool here = 16 * pass + r0 + 2 * k + (lane >> 4) < rows;
                const uint32_t x[8] = {own[k].x, own[k].y, own[k].z, own[k].w, __shfl_down_sync(kAll, own[k].x, 1, 16), __shfl_down_sync(kAll, own[k].y, 1, 16),
                                       __shfl_down_sync(kAll, own[k].z, 1, 16), __shfl_down_sync(kAll, own[k].w, 1, 16)};
                uint32_t y[6], z[5], o[4];
#pragma unroll
                for (int i = 0; i < 6; ++i) y[i] = (head[k] & 4) ? x[i + 2] : x[i];
#pragma unroll
                for (int i = 0; i < 5; ++i) z[i] = (head[k] & 2) ? y[i + 1] : y[i];
                const uint32_t pick = (head[k] & 1) ? 0x5432u : 0x3210u;
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] = __byte_perm(z[i], z[i + 1], pick);
                if (here && (head[k] == 0 || l < 15)) st_global_v4(dst[k] + head[k] + 8 * l, o[0], o[1], o[2], o[3]);
                if (here && head[k] != 0 && l < 8) dst[k][l < head[k] ? l : 120 + l] = static_cast<uint16_t>(edge[k] & 0xffffu);
            }
        }
    }
}

// BULK (pairs): the output's rows are on 16-byte boundaries and leave in bulk stores.
template <int FMT, int TN, bool PAIR, bool BULK>
__global__ void __launch_bounds__(Shape<FMT, TN, PAIR>::kThreads, Shape<FMT, TN, PAIR>::kCtasPerSm)
gemm4_kernel(const __grid_constant__ CUtensorMap tmP, const __grid_constant__ CUtensorMap tmQ,
             const __grid_constant__ CUtensorMap tmSfP, const __grid_constant__ CUtensorMap tmSfQ,
             const __grid_constant__ CUtensorMap tmOut, const Gemm4Args p) {
    using S = Shape<FMT, TN, PAIR>;
    constexpr int kStages = S::kStages, kStageBytes = S::kStageBytes;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw_addr = smem_u32(smem_raw);
    const uint32_t tiles_addr = (raw_addr + 1023u) & ~1023u;
    Tail4* tail = reinterpret_cast<Tail4*>(smem_raw + (tiles_addr - raw_addr) + size_t(kStages) * kStageBytes + S::kStoreBytes);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = (PAIR || p.split > 1) ? cluster_ctarank() : 0u;
    const int ctas_log2 = PAIR ? 1 : 31 - __clz(p.split);            // CTAs per tile
    const int first_tile = static_cast<int>(blockIdx.x) >> ctas_log2, tile_step = static_cast<int>(gridDim.x) >> ctas_log2;
    const int num_tiles = p.p_tiles * p.q_tiles;
    // a cluster that splits the contraction has one tile, and this CTA these stages of it
    const int kb_begin = p.split > 1 ? static_cast<int>(rank) * p.stages_k / p.split : 0;
    const int kb_end = p.split > 1 ? (static_cast<int>(rank) + 1) * p.stages_k / p.split : p.stages_k;
    volatile int* abort_flag = &tail->abort;
    bool freed = false;                                              // warp 2: tensor memory

    if (threadIdx.x == 0) {
        tma_prefetch_desc(&tmP);
        tma_prefetch_desc(&tmQ);
        tma_prefetch_desc(&tmSfP);
        tma_prefetch_desc(&tmSfQ);
        if (BULK) tma_prefetch_desc(&tmOut);
        for (int s = 0; s < kStages; ++s) {
            mbar_init(smem_u32(&tail->full[s]), 1);
            mbar_init(smem_u32(&tail->empty[s]), 1);
        }
        mbar_init(smem_u32(&tail->tmem_full), 1);
        mbar_init(smem_u32(&tail->tmem_empty), (PAIR ? 2 : 1) * S::kEpiWarps);
        tail->abort = 0;
        mbar_init_fence();
    }
    if (warp == 2) {
        if constexpr (PAIR) { tmem_alloc_pair(smem_u32(&tail->tmem_base), S::kTmem); tmem_relinquish_pair(); }
        else { tmem_alloc(smem_u32(&tail->tmem_base), S::kTmem); tmem_relinquish(); }
    }
    tc_fence_before();
    if constexpr (PAIR) cluster_sync_all(); else __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = tail->tmem_base;
    grid_dependency_wait();
    grid_launch_dependents();

    if (warp < 2) {
        // ------------------------------------------------------------ TMA producers: every other stage each
        if (lane == 0) {
            const int per_tile = kb_end - kb_begin, my_tiles = !PAIR ? 1 : first_tile < num_tiles ? (num_tiles - 1 - first_tile) / tile_step + 1 : 0;
            const uint32_t total = static_cast<uint32_t>(per_tile) * my_tiles;
            int tile = first_tile, kb = kb_begin + warp, p_tile, q_tile;
            tile4_coords<PAIR>(p, tile, p_tile, q_tile);
            for (uint32_t n = warp; n < total; n += 2, kb += 2) {
                const uint32_t stage = n % kStages, parity = (n / kStages) & 1u;
                if (!mbar_wait(smem_u32(&tail->empty[stage]), parity ^ 1u, abort_flag, &wait_status)) break;
                if (!PAIR || rank == 0) mbar_expect_tx(smem_u32(&tail->full[stage]), (PAIR ? 2 : 1) * kStageBytes);      // a pair's bytes are counted by rank 0
                while (kb >= kb_end) { kb -= per_tile; tile += tile_step; tile4_coords<PAIR>(p, tile, p_tile, q_tile); }
                const int p_group = PAIR ? 2 * p_tile + static_cast<int>(rank) : p_tile, p0 = p_group * kRows;
                const int q0 = q_tile * TN, q_first = q0 + (PAIR ? static_cast<int>(rank) * (TN / 2) : 0), q_group = q0 / kRows;
                const uint32_t dst = tiles_addr + stage * kStageBytes, sf = dst + S::kPBytes + S::kQBytes;
                const uint32_t bar = PAIR ? mapa_shared(smem_u32(&tail->full[stage]), 0) : smem_u32(&tail->full[stage]);
                if constexpr (PAIR) {
                    tma_load_2d_pair(dst, &tmP, bar, kb * (kStageK / 2), p0);
                    tma_load_2d_pair(dst + S::kPBytes, &tmQ, bar, kb * (kStageK / 2), q_first);
                    tma_load_3d_pair(sf, &tmSfP, bar, 0, kb * S::kTiles * 4, p_group);
                    tma_load_3d_pair(sf + S::kSfBytes, &tmSfQ, bar, 0, kb * S::kTiles * 4, q_group);
                } else {
                    tma_load_2d(dst, &tmP, bar, kb * (kStageK / 2), p0);
                    tma_load_2d(dst + S::kPBytes, &tmQ, bar, kb * (kStageK / 2), q_first);
                    tma_load_3d(sf, &tmSfP, bar, 0, kb * S::kTiles * 4, p_group);
                    tma_load_3d(sf + S::kSfBytes, &tmSfQ, bar, 0, kb * S::kTiles * 4, q_group);
                }
            }
        }
    } else if (warp == 2) {
        // ------------------------------------------------------------ MMA issuer (CTA pair: rank 0 only)
        if (!PAIR || rank == 0u) {
            const uint32_t leader = elect_one();
            Ring<kStages> ring;
            bool ok = true, ready = false;
            int it = 0;
            for (int tile = first_tile; ok && tile < num_tiles; tile += tile_step, ++it) {
                int p_tile, q_tile;
                tile4_coords<PAIR>(p, tile, p_tile, q_tile);
                if (!__all_sync(kAll, mbar_wait(smem_u32(&tail->tmem_empty), (it & 1) ^ 1u, abort_flag, &wait_status))) break;
                tc_fence_after();
                // first column of the tile's scales; the MMA takes them from even columns only, so that tiles narrower than 64 are
                // for products with one such tile
                const uint32_t q_offset = TN >= 64 ? static_cast<uint32_t>((q_tile * TN) % kRows) / 32u : 0u;
                for (int kb = kb_begin; kb < kb_end; ++kb) {
                    if (!ready) {
                        ok = __all_sync(kAll, mbar_wait(smem_u32(&tail->full[ring.stage]), ring.phase, abort_flag, &wait_status));
                        if (!ok) break;
                    }
                    tc_fence_after();
                    const uint32_t sf_p = tmem_base + TN + ring.stage * S::kSfCols, sf_q = sf_p + 4 * S::kTiles;
                    const uint32_t base = (tiles_addr + ring.stage * kStageBytes) >> 4;        // descriptors count in 16 bytes
                    const uint32_t sf_base = base + ((S::kPBytes + S::kQBytes) >> 4), done = smem_u32(&tail->empty[ring.stage]);
                    ring.next();
                    const bool filled = mbar_peek(smem_u32(&tail->full[ring.stage]), ring.phase);
                    if (leader) {
                        const int left = p.K - kb * kStageK;
                        if (left >= kStageK) issue_stage<FMT, TN, PAIR, true>(tmem_base, base, sf_base, sf_p, sf_q, q_offset, kb != kb_begin, left);
                        else issue_stage<FMT, TN, PAIR, false>(tmem_base, base, sf_base, sf_p, sf_q, q_offset, kb != kb_begin, left);
                        if constexpr (PAIR) umma_commit_pair(done); else umma_commit(done);
                    }
                    ready = __all_sync(kAll, filled);
                }
                if (ok && leader) {
                    if constexpr (PAIR) umma_commit_pair(smem_u32(&tail->tmem_full)); else umma_commit(smem_u32(&tail->tmem_full));
                }
                __syncwarp();
            }
            if constexpr (!PAIR) {
                // the accumulator has been read: tensor memory is given back while the output is on its way (1 x 4096 x 1024: 4.0 -> 3.2 us)
                if (ok && __all_sync(kAll, mbar_wait(smem_u32(&tail->tmem_empty), 0u, abort_flag, &wait_status))) {
                    tc_fence_after();
                    tmem_dealloc(tmem_base, S::kTmem);
                    freed = true;
                }
            }
        }
    } else {
        // ------------------------------------------------------------ epilogue
        const int quad = warp & 3, part = (warp - kOtherWarps) >> 2;
        const float dq = __fmul_rn(p.s0 != nullptr ? __fdiv_rn(1.0f, *p.s0) : 1.0f, p.s1 != nullptr ? __fdiv_rn(1.0f, *p.s1) : 1.0f);
        constexpr int kChunk = S::kWarpCols < 32 ? 16 : 32, kShareRows = kRows + 4, kShareCols = TN + 4;
        // staging of the output: a pair's own, or (a single CTA has one tile) operand stages, which have all been read by then
        const uint32_t stage = tiles_addr + (PAIR ? kStages * kStageBytes : 0) + (warp - kOtherWarps) * 4096;
        uint32_t sent = 0;
        int it = 0;
        for (int tile = first_tile; tile < num_tiles; tile += tile_step, ++it) {
            int p_tile, q_tile;
            tile4_coords<PAIR>(p, tile, p_tile, q_tile);
            const bool got = mbar_wait(smem_u32(&tail->tmem_full), it & 1, abort_flag, &wait_status);
            if (!__all_sync(kAll, got)) break;
            tc_fence_after();
            const uint32_t taddr = tmem_base + part * S::kWarpCols + (static_cast<uint32_t>(quad * 32) << 16);
            const int row = (PAIR ? 2 * p_tile + static_cast<int>(rank) : p_tile) * kRows + quad * 32 + lane;
            const int col0 = q_tile * TN + part * S::kWarpCols;
            if constexpr (PAIR) {
                // the whole accumulator into registers first, so that the next tile's MMAs may have it while this one is stored
                uint32_t r[S::kWarpCols / 32][32];
#pragma unroll
                for (int c = 0; c < S::kWarpCols / 32; ++c) tmem_ld32(taddr + 32 * c, r[c]);
                tmem_ld_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(mapa_shared(smem_u32(&tail->tmem_empty), 0));
                static_assert(S::kWarpCols == 128, "write_wide");
                if (!BULK && !p.f32 && col0 + 128 <= p.Q) {
                    uint32_t w[64];
#pragma unroll
                    for (int i = 0; i < 64; ++i) w[i] = cvt_bf16x2(__fmul_rn(__uint_as_float(r[i >> 4][2 * i & 31]), dq), __fmul_rn(__uint_as_float(r[i >> 4][(2 * i + 1) & 31]), dq));
                    if (row - lane < p.P) write_wide(p, stage, lane, row - lane, col0, min(32, p.P - (row - lane)), w);
                    continue;
                }
#pragma unroll
                for (int c = 0; c < S::kWarpCols / 32; ++c) {
                    const int col = col0 + 32 * c;
                    if (col >= p.Q || row - lane >= p.P) break;
                    float v[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = __fmul_rn(__uint_as_float(r[c][i]), dq);
                    const bool cut = col + 32 > p.Q && (p.Q & (p.f32 ? 3 : 7)) != 0;
                    if (BULK && !cut) send_rows(&tmOut, p.f32 != 0, stage, sent, lane, row - lane, col, v);
                    else write_rows(p, stage, lane, row - lane, col, min(32, p.P - (row - lane)), min(32, p.Q - col), v);
                }
            } else {
                // here too the accumulator goes to registers first
                uint32_t r[S::kWarpCols / kChunk][kChunk];
#pragma unroll
                for (int c = 0; c < S::kWarpCols / kChunk; ++c) tmem_ld_cols<kChunk>(taddr + kChunk * c, r[c]);
                tmem_ld_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&tail->tmem_empty));
#pragma unroll
                for (int c = 0; c < S::kWarpCols / kChunk; ++c) {
                    const int col = col0 + kChunk * c, have = min(kChunk, p.Q - col);      // columns of these that there are
                    if (have <= 0) break;
                    if (p.split > 1) {
                        // this share of the tile into shared memory (every operand stage has been read), in the order of the output's
                        // rows: [column][accumulator row] if the output is [Q, P], else [accumulator row][column]
                        float* share = reinterpret_cast<float*>(smem_raw + (tiles_addr - raw_addr));
                        const int first = part * S::kWarpCols + kChunk * c, mine = quad * 32 + lane;
                        if (p.swap) {
#pragma unroll
                            for (int i = 0; i < kChunk; ++i) {
                                if (i >= have) break;
                                share[(first + i) * kShareRows + mine] = __uint_as_float(r[c][i]);
                            }
                        } else {
#pragma unroll
                            for (int i = 0; i < kChunk; i += 4)
                                *reinterpret_cast<float4*>(share + mine * kShareCols + first + i) =
                                    make_float4(__uint_as_float(r[c][i]), __uint_as_float(r[c][i + 1]), __uint_as_float(r[c][i + 2]), __uint_as_float(r[c][i + 3]));
                        }
                        continue;
                    }
                    if (row - lane >= p.P) break;
                    if (p.swap) {
                        if (row >= p.P) break;
                        const int64_t at = static_cast<int64_t>(col) * p.ld_out + row;
#pragma unroll
                        for (int i = 0; i < kChunk; ++i) {
                            if (i >= have) break;
                            store_one(p, at + i * p.ld_out, __fmul_rn(__uint_as_float(r[c][i]), dq));
                        }
                        continue;
                    }
                    float v[kChunk];
#pragma unroll
                    for (int i = 0; i < kChunk; ++i) v[i] = __fmul_rn(__uint_as_float(r[c][i]), dq);
                    if constexpr (kChunk == 32) {
                        if (p.vec != 16) {
                            write_rows(p, stage, lane, row - lane, col, min(32, p.P - (row - lane)), have, v);
                            continue;
                        }
                    }
                    if (row < p.P) store_cols<kChunk>(p, static_cast<int64_t>(row) * p.ld_out + col, v, have);
                }
            }
        }
        if (BULK && lane == 0) tma_store_wait_all();          // the staged output has reached global memory
    }

    // ---------------------------------------------------------------- teardown
    tc_fence_before();
    __syncthreads();
    if (*abort_flag) {
        for (int i = 0; i < 200; ++i) __nanosleep(1000);      // copies in flight land before shared memory is released
        __syncthreads();
        if (!PAIR && p.split > 1)                             // a share that is not there is NaN, and so is the tile
            for (int i = threadIdx.x; i < max(TN * (kRows + 4), kRows * (TN + 4)); i += S::kThreads)
                reinterpret_cast<float*>(smem_raw + (tiles_addr - raw_addr))[i] = __uint_as_float(0x7fffffffu);
    }
    if (!PAIR && p.split > 1) {
        cluster_sync_all();                                   // all shares of the tile lie in their CTAs' shared memory
        const float dq = __fmul_rn(p.s0 != nullptr ? __fdiv_rn(1.0f, *p.s0) : 1.0f, p.s1 != nullptr ? __fdiv_rn(1.0f, *p.s1) : 1.0f);
        int p_tile, q_tile;
        tile4_coords<PAIR>(p, first_tile, p_tile, q_tile);
        const int cols = min(TN, p.Q - q_tile * TN), rows = min(kRows, p.P - p_tile * kRows);
        // rows of the output, four words of one at a time; this CTA's part of them, each the sum of the shares in rank order
        const int lines = p.swap ? cols : rows, len = p.swap ? rows : cols, pitch = p.swap ? kRows + 4 : TN + 4;
        const int quads = (len + 3) / 4;
        const int64_t line0 = p.swap ? int64_t(q_tile) * TN : int64_t(p_tile) * kRows, word0 = p.swap ? int64_t(p_tile) * kRows : int64_t(q_tile) * TN;
        for (int i = static_cast<int>(rank) * S::kThreads + threadIdx.x; i < lines * quads; i += p.split * S::kThreads) {
            const int line = i / quads, word = 4 * (i - line * quads);
            const uint32_t at = tiles_addr + 4u * static_cast<uint32_t>(line * pitch + word);
            float4 v[8];
#pragma unroll
            for (int s = 0; s < 8; ++s)
                if (s < p.split)
                    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                                 : "=f"(v[s].x), "=f"(v[s].y), "=f"(v[s].z), "=f"(v[s].w) : "r"(mapa_shared(at, s)) : "memory");
            float4 sum = v[0];
#pragma unroll
            for (int s = 1; s < 8; ++s)
                if (s < p.split) {
                    sum.x = __fadd_rn(sum.x, v[s].x); sum.y = __fadd_rn(sum.y, v[s].y);
                    sum.z = __fadd_rn(sum.z, v[s].z); sum.w = __fadd_rn(sum.w, v[s].w);
                }
            const float out[4] = {__fmul_rn(sum.x, dq), __fmul_rn(sum.y, dq), __fmul_rn(sum.z, dq), __fmul_rn(sum.w, dq)};
            const int64_t to = (line0 + line) * p.ld_out + word0 + word;
            if (p.vec == 16 && word + 4 <= len) {
                if (p.f32) st_global_v4(reinterpret_cast<float*>(p.out) + to, __float_as_uint(out[0]), __float_as_uint(out[1]), __float_as_uint(out[2]), __float_as_uint(out[3]));
                else st_global_v2(reinterpret_cast<uint16_t*>(p.out) + to, cvt_bf16x2(out[0], out[1]), cvt_bf16x2(out[2], out[3]));
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (word + k < len) store_one(p, to + k, out[k]);
            }
        }
    }
    if (PAIR || p.split > 1) cluster_sync_all();              // nobody leaves while its memory can be reached
    if (warp == 2 && !freed) {
        __syncwarp();
        tc_fence_after();
        if constexpr (PAIR) tmem_dealloc_pair(tmem_base, S::kTmem); else tmem_dealloc(tmem_base, S::kTmem);
    }
}

// ---------------------------------------------------------------- host side
bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

template <int FMT, int TN, bool PAIR, bool BULK>
int launch4(const CUtensorMap (&tm)[5], const Gemm4Args& a, int sm_count, cudaStream_t st) {
    using S = Shape<FMT, TN, PAIR>;
    constexpr size_t kSmem = smem4_bytes<FMT, TN, PAIR>();
    constexpr int kMaxDevices = 64;
    static std::once_flag once_dev[kMaxDevices];
    static cudaError_t err_dev[kMaxDevices] = {};
    static int clusters_dev[kMaxDevices] = {};
    int dev = 0;
    FP8MLP_CUDA_CHECK(cudaGetDevice(&dev));
    if (dev < 0 || dev >= kMaxDevices) { set_cuda_error_str("4-bit product", "device ordinal out of range"); return FP8MLP_ERR_CUDA; }
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    cfg.blockDim = dim3(S::kThreads);
    cfg.dynamicSmemBytes = kSmem;
    cfg.stream = st;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const int cluster = PAIR ? 2 : a.split;
    if (cluster > 1) {
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = cluster;
        attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
        cfg.numAttrs = 2;
    }
    std::call_once(once_dev[dev], [&] {
        err_dev[dev] = cudaFuncSetAttribute(gemm4_kernel<FMT, TN, PAIR, BULK>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kSmem));
        if (PAIR && err_dev[dev] == cudaSuccess) {
            cfg.gridDim = dim3(static_cast<unsigned>(sm_count) & ~1u);
            err_dev[dev] = cudaOccupancyMaxActiveClusters(&clusters_dev[dev], gemm4_kernel<FMT, TN, PAIR, BULK>, &cfg);
        }
    });
    FP8MLP_CUDA_CHECK(err_dev[dev]);
    const int64_t tiles = static_cast<int64_t>(a.p_tiles) * a.q_tiles;
    int64_t grid;
    if (PAIR) {
        if (clusters_dev[dev] < 1) { set_cuda_error_str("4-bit product", "no CTA pair fits on the device"); return FP8MLP_ERR_CUDA; }
        grid = 2 * (tiles < clusters_dev[dev] ? tiles : clusters_dev[dev]);
    } else {
        grid = tiles * a.split;                               // a tile per CTA or cluster
    }
    cfg.gridDim = dim3(static_cast<unsigned>(grid));
    FP8MLP_CUDA_CHECK(cudaLaunchKernelEx(&cfg, gemm4_kernel<FMT, TN, PAIR, BULK>, tm[0], tm[1], tm[2], tm[3], tm[4], a));
    count_launch();
    return FP8MLP_OK;
}

struct Plan4 { bool pair, swap; int tn, split; };

// How a product runs, by what was measured on 148 SMs (NVFP4, bf16 out; us in a chain of launches).
// CTA pairs on 256 x 256 tiles, where at least half of the SMs get one (1536 x 2048 x 4096, 48 pairs: 11.2, single CTAs 14.2;
// 1500 x 1500 x 4096, 36 pairs: 14.8 and 11.3).  Otherwise single CTAs: their 128 rows are of the longer side where the other one has
// at most 128, by as many columns as that one needs; with more than 64 of them, tiles 64 wide as long as all are on the SMs at once
// (1024 x 1024 x 1024: 4.3, 128 wide 6.1; 512 x 8192 x 1024, 512 tiles: 10.1 and 8.9).  The contraction is split where it has 8 stages
// or more (1 x 4096 x 4096, 16 stages: 5.7 -> 5.1 with 4 shares; 1 x 4096 x 1024, 4 stages: 3.3 -> 4.2 with 2), into shares of at least
// 2 stages, for as many CTAs as there are SMs (256 x 4096 x 4096, 128 tiles: 8.2 whole, 9.9 with 2 shares), or twice as many
// where a share still has 16 stages (1 x 11008 x 11008, 86 tiles: 17.5 -> 15.6).
Plan4 plan4(int64_t M, int64_t N, int64_t K, int sms) {
    Plan4 pl{};
    const int64_t shorter = M < N ? M : N;
    const int64_t pairs = (M + 255) / 256 * ((N + 255) / 256);
    pl.pair = shorter > 128 && 2 * pairs >= sms / 2;
    if (pl.pair) { pl.tn = 256; pl.split = 1; return pl; }
    pl.swap = shorter <= 128 && M < N;
    const int64_t P = pl.swap ? N : M, Q = pl.swap ? M : N;
    auto tiles = [&](int tn) { return (P + 127) / 128 * ((Q + tn - 1) / tn); };
    pl.tn = shorter <= 16 ? 16 : shorter <= 32 ? 32 : shorter <= 64 || tiles(64) <= 2 * sms ? 64 : 128;
    const int64_t stages = (K + kStageK - 1) / kStageK;
    auto fits = [&](int split) {
        const int64_t ctas = tiles(pl.tn) * split;
        return stages >= 8 && stages >= 2 * split && (ctas <= sms || (ctas <= 2 * sms && stages >= 16 * split));
    };
    pl.split = 8;
    while (pl.split > 1 && !fits(pl.split)) pl.split /= 2;
    return pl;
}

template <int FMT>
int dispatch4(const Plan4& pl, const CUtensorMap (&tm)[5], const Gemm4Args& a, int sms, cudaStream_t st) {
    if (pl.pair) return a.vec == 16 ? launch4<FMT, 256, true, true>(tm, a, sms, st) : launch4<FMT, 256, true, false>(tm, a, sms, st);
    switch (pl.tn) {
        case 16: return launch4<FMT, 16, false, false>(tm, a, sms, st);
        case 32: return launch4<FMT, 32, false, false>(tm, a, sms, st);
        case 64: return launch4<FMT, 64, false, false>(tm, a, sms, st);
        default: return launch4<FMT, 128, false, false>(tm, a, sms, st);
    }
}

}  // namespace

int gemm4_status_word(int** word) {
    FP8MLP_CUDA_CHECK(cudaGetSymbolAddress(reinterpret_cast<void**>(word), wait_status));
    return FP8MLP_OK;
}

}  // namespace fp8mlp

using namespace fp8mlp;

extern "C" int fp8mlp_gemm_fp4(int64_t M, int64_t N, int64_t K, int fmt, const uint8_t* A, int64_t ld_a, const uint8_t* a_scales,
                               const float* scale_a, const uint8_t* B, int64_t ld_b, const uint8_t* b_scales, const float* scale_b,
                               void* out, int out_dtype, int64_t ld_out, void* stream) {
    if (fmt != FP8MLP_MXFP4 && fmt != FP8MLP_NVFP4) return FP8MLP_ERR_ARG;
    if (out_dtype != FP8MLP_BF16 && out_dtype != FP8MLP_F32) return FP8MLP_ERR_ARG;
    if (fmt == FP8MLP_MXFP4 && (scale_a != nullptr || scale_b != nullptr)) return FP8MLP_ERR_ARG;
    constexpr int64_t kMost = int64_t(1) << 24;
    if (M < 0 || N < 0 || K < 1 || M > kMost || N > kMost || K > kMost) return FP8MLP_ERR_SHAPE;
    const int64_t row = (K + 31) / 32 * 16;
    if (ld_a % 16 != 0 || ld_b % 16 != 0 || ld_a < row || ld_b < row || (M > 1 && ld_out < N)) return FP8MLP_ERR_SHAPE;
    const int block = fmt == FP8MLP_MXFP4 ? 32 : 16;
    const int64_t scale_tiles = (K + 4 * block - 1) / (4 * block);
    if ((M + 127) / 128 * ((N + 15) / 16) > INT32_MAX / 8) return FP8MLP_ERR_SHAPE;
    if (M == 0 || N == 0) return FP8MLP_OK;
    if (A == nullptr || a_scales == nullptr || B == nullptr || b_scales == nullptr || out == nullptr) return FP8MLP_ERR_ARG;
    const int bytes = out_dtype == FP8MLP_F32 ? 4 : 2;
    if (!aligned(A, 16) || !aligned(B, 16) || !aligned(a_scales, 16) || !aligned(b_scales, 16) || !aligned(out, bytes)) return FP8MLP_ERR_ALIGN;
    if (!aligned(scale_a, 4) || !aligned(scale_b, 4)) return FP8MLP_ERR_ALIGN;
    int dev = 0, sms = 0;
    FP8MLP_CUDA_CHECK(cudaGetDevice(&dev));
    FP8MLP_CUDA_CHECK(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    const Plan4 pl = plan4(M, N, K, sms);
    struct Side { const uint8_t *codes, *scales; int64_t ld, rows; };
    const Side a_side{A, a_scales, ld_a, M}, b_side{B, b_scales, ld_b, N};
    const Side &P = pl.swap ? b_side : a_side, &Q = pl.swap ? a_side : b_side;
    CUtensorMap tm[5] = {};
    const uint64_t row_bytes = static_cast<uint64_t>((K + 1) / 2);
    const uint32_t sf_rows = 4u * kStageK / (4u * block);                     // 128-byte rows of a stage's scales
    auto codes_map = [&](CUtensorMap* m, const Side& s, uint32_t box) { return make_tmap_fp4(m, s.codes, row_bytes, s.rows, s.ld, box); };
    auto scales_map = [&](CUtensorMap* m, const Side& s, uint32_t groups) {
        return make_tmap_fp4_scales(m, s.scales, static_cast<uint64_t>(scale_tiles), static_cast<uint64_t>((s.rows + 127) / 128), sf_rows, groups);
    };
    int rc = codes_map(&tm[0], P, kRows);
    if (rc == FP8MLP_OK) rc = codes_map(&tm[1], Q, pl.pair ? pl.tn / 2 : pl.tn);
    if (rc == FP8MLP_OK) rc = scales_map(&tm[2], P, 1);
    if (rc == FP8MLP_OK) rc = scales_map(&tm[3], Q, (pl.tn + 127) / 128);
    const int vec = aligned(out, 16) && (M <= 1 || ld_out * bytes % 16 == 0) ? 16 : 1;
    if (rc == FP8MLP_OK && pl.pair && vec == 16)
        rc = out_dtype == FP8MLP_F32 ? make_tmap_out_f32(&tm[4], out, N, M, ld_out * bytes) : make_tmap_out_bf16(&tm[4], out, N, M, ld_out * bytes);
    if (rc != FP8MLP_OK) return rc;
    Gemm4Args a{};
    a.P = static_cast<int>(P.rows); a.Q = static_cast<int>(Q.rows); a.K = static_cast<int>(K);
    a.p_tiles = (a.P + (pl.pair ? 255 : 127)) / (pl.pair ? 256 : 128);
    a.q_tiles = (a.Q + pl.tn - 1) / pl.tn;
    if (pl.tn < 64 && a.q_tiles != 1) return FP8MLP_ERR_SHAPE;               // (the plan makes none: see q_offset)
    a.stages_k = static_cast<int>((K + kStageK - 1) / kStageK);
    a.split = pl.split;
    a.group = 16;
    a.swap = pl.swap ? 1 : 0;
    a.f32 = out_dtype == FP8MLP_F32 ? 1 : 0;
    a.vec = vec;
    a.s0 = scale_a; a.s1 = scale_b;
    a.out = static_cast<uint8_t*>(out);
    a.ld_out = ld_out;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return fmt == FP8MLP_MXFP4 ? dispatch4<FP8MLP_MXFP4>(pl, tm, a, sms, st) : dispatch4<FP8MLP_NVFP4>(pl, tm, a, sms, st);
}
