// 4-bit operands: quantisation of a matrix or its transpose into E2M1 codes with block scales, and back.
//
// Both directions stream their matrix once.  A block of threads owns 128 rows of the operand, so that it owns whole tiles of
// block scales (512 bytes each, gathered in shared memory and written in one piece), and a stretch of columns.  The quotient
// v / scale is rounded once: a product with the reciprocal, corrected with its remainder (Markstein's correction), so that the
// one rounding to E2M1 is right in ties and next to them; MXFP4 scales are powers of two and need none of that.
#include "common.cuh"

namespace fp8mlp {

namespace {

constexpr int kThreads = 256;
constexpr int kTileRows = 128;            // operand rows of a block of threads, and of a tile of scales
constexpr int kScaleTile = 512;           // bytes: 128 rows x 4 blocks
constexpr int kCols = 128;                // operand columns of a block of threads, matrix as it is
constexpr int kColsBack = 256;            // and back
template <int FMT> struct Fmt;
template <> struct Fmt<FP8MLP_MXFP4> { static constexpr int kBlock = 32; };
template <> struct Fmt<FP8MLP_NVFP4> { static constexpr int kBlock = 16; };


struct QuantArgs {
    const uint8_t* src;
    int64_t ld;                           // bytes
    int64_t rows, cols;                   // of the operand
    uint8_t *codes, *scales;
    int64_t ld_codes;
    const unsigned int* amax_in;          // null: the scale is given
    unsigned int* amax_out;               // raised to max |src|; null: not wanted
    float* scale;                         // NVFP4; written where amax_in is given
    int col_tiles, scale_tiles;           // blocks of threads / tiles of scales along the columns
};
// the same matrix as the search for its maximum takes it: units of 16 bytes, a matrix without gaps as one row
struct AmaxArgs {
    const uint8_t* src;
    int64_t ld, rows, cols, units;
    unsigned int* amax;
};

// place of a block's scale in its tile
__device__ __forceinline__ int scale_at(int row, int block) { return (row & 31) * 16 + (row >> 5) * 4 + block; }

// eight floats -> eight E2M1 codes, first in the low half of the low byte; nearest, ties to even, saturating
__device__ __forceinline__ uint32_t cvt_e2m1x8(const float (&v)[8]) {
    uint32_t r;
    asm("{\n\t"
        ".reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t"
        "}\n"
        : "=r"(r) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}
// two codes (a byte) -> two floats
__device__ __forceinline__ void e2m1x2_to_f32(uint32_t byte, float& lo, float& hi) {
    uint32_t h2;
    // (taken apart as 16 bits: with four bytes of a 32-bit register a byte loaded from memory came out as 0)
    asm("{\n\t"
        ".reg .b8 a, b;\n\t"
        "mov.b16 {a, b}, %1;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
        "}\n"
        : "=r"(h2) : "h"(static_cast<unsigned short>(byte)));
    asm("cvt.f32.f16 %0, %1;" : "=f"(lo) : "h"(static_cast<unsigned short>(h2 & 0xFFFFu)));
    asm("cvt.f32.f16 %0, %1;" : "=f"(hi) : "h"(static_cast<unsigned short>(h2 >> 16)));
}

// Largest power of two g with g * amax <= 448 * 6 = 0.65625 * 2^12; 1 for a zero or non-finite amax; within 2^-100 .. 2^100.
__device__ __forceinline__ float tensor_scale(float amax) {
    if (!(amax > 0.0f) || isinf(amax)) return 1.0f;
    int e;
    const float m = frexpf(amax, &e);
    const int k = m <= 0.65625f ? 12 - e : 11 - e;
    return ldexpf(1.0f, max(-100, min(100, k)));
}

// A block of values, or N of them (those past the matrix are 0) -> their codes, eight to a word, and the block's scale's byte.
// `top`: max |src| of the block's bit patterns (a NaN is above infinity there).  g: the tensor's scale (NVFP4).
template <int FMT, int N>
__device__ __forceinline__ uint32_t quantise_block(const float (&v)[N], uint32_t top, float g, uint32_t (&code)[N / 8]) {
    if constexpr (FMT == FP8MLP_MXFP4) {
        // exponent field of 2^(floor(log2 a) - 2), biased as E8M0; subnormal and zero maxima get the smallest scale
        uint32_t byte = top >> 23;
        byte = byte > 2u ? byte - 2u : 0u;
        const bool finite = top < 0x7f800000u;
        const float inv = __uint_as_float((254u - byte) << 23);          // 2^(127 - byte): exact products
#pragma unroll
        for (int i = 0; i < N / 8; ++i) {
            float q[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) q[k] = __fmul_rn(v[8 * i + k], inv);
            code[i] = cvt_e2m1x8(q);
        }
        return finite ? byte : 0xffu;
    } else {
        const float a = __fmul_rn(__uint_as_float(top), fabsf(g));         // (a negative g is the elements' sign)
        const bool finite = __float_as_uint(a) < 0x7f800000u;
        // a / 6: a product with the reciprocal, corrected with its remainder (Markstein's correction).  E4M3's borders times 6 are fp32 numbers, and for any
        // other a the quotient is more than half a last place from them, so that what is left of its error turns no scale.
        constexpr float kSixth = 1.0f / 6.0f;
        const float near = __fmul_rn(a, kSixth), sixth = __fmaf_rn(__fmaf_rn(-6.0f, near, a), kSixth, near);
        const uint32_t byte = cvt_fp8x2<FP8MLP_E4M3>(finite ? sixth : 0.0f, 0.0f) & 0xffu;
        float s, unused;
        e4m3x2_to_f32(byte, s, unused);
        const float r = s > 0.0f ? rcp_approx(s) : 0.0f;       // within a last place, which the correction below squares
        const f32x2 g2 = pack2(g, g), s2 = pack2(-s, -s), r2 = pack2(r, r);
#pragma unroll
        for (int i = 0; i < N / 8; ++i) {
            float q[8];
#pragma unroll
            for (int k = 0; k < 8; k += 2) {
                const f32x2 x = mul2(pack2(v[8 * i + k], v[8 * i + k + 1]), g2);
                // x / s rounded once to fp32 (s has four bits, so the remainder is exact).  That is a border between two
                // codes only if x / s is one: s * border has at most seven bits, so an x next to it is at least one of
                // its last places off, and x / s more than half a place of the quotient's (1 / 1.875)
                const f32x2 t = mul2(x, r2);
                unpack2(fma2(fma2(s2, t, x), r2, t), q[k], q[k + 1]);
            }
            code[i] = cvt_e2m1x8(q);
        }
        return finite ? byte : 0x7fu;
    }
}

template <typename SRC> __device__ __forceinline__ float to_f32(SRC v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<uint16_t>(uint16_t v) { return __uint_as_float(static_cast<uint32_t>(v) << 16); }

// The bit pattern of max |v|, a NaN (above infinity) if there is one; two values an instruction.
template <int N>
__device__ __forceinline__ uint32_t top_bits(const float (&v)[N]) {
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < N; i += 2) asm("max.NaN.abs.f32 %0, %0, %1, %2;" : "+f"(top) : "f"(v[i]), "f"(v[i + 1]));
    return __float_as_uint(top) & 0x7fffffffu;
}

// max |src| of a block of threads, NaN left out, raised to *out
__device__ __forceinline__ void raise_amax(float v, unsigned int* out) {
    __shared__ float part[kThreads / 32];
    v = warp_max_nonneg(v);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    if (threadIdx.x < 32) {
        v = warp_max_nonneg(threadIdx.x < kThreads / 32 ? part[threadIdx.x] : 0.0f);
        if (threadIdx.x == 0 && v > 0.0f) atomicMax(out, __float_as_uint(v));
    }
}

__device__ __forceinline__ float scale_of(const QuantArgs& p) {
    if (p.amax_in == nullptr) return *p.scale;
    const float g = tensor_scale(__uint_as_float(__ldcg(p.amax_in)));
    if (blockIdx.x == 0 && threadIdx.x == 0) *p.scale = g;
    return g;
}

// Tiles are walked from the last to the first where the maximum has just been looked for: the end of the matrix is what L2
// still holds of that pass.
// A transpose goes along the source's rows first (4096 x 4096 bf16 MXFP4 10.0 -> 9.5 us).
template <bool TRANSPOSED>
__device__ __forceinline__ void tile_of(const QuantArgs& p, int64_t& row_tile, int64_t& col_tile) {
    const int64_t tile = p.amax_in != nullptr ? gridDim.x - 1 - blockIdx.x : blockIdx.x;
    if constexpr (TRANSPOSED) {
        const int64_t row_tiles = (p.rows + kTileRows - 1) / kTileRows;
        col_tile = tile / row_tiles;
        row_tile = tile - col_tile * row_tiles;
    } else {
        row_tile = tile / p.col_tiles;
        col_tile = tile - row_tile * p.col_tiles;
    }
}

// The block's tiles of scales, gathered in shared memory, to their place.
__device__ __forceinline__ void write_scales(const QuantArgs& p, const uint8_t* scales, int64_t row_tile, int64_t first, int tiles) {
    uint8_t* out = p.scales + (row_tile * p.scale_tiles + first) * kScaleTile;
    const int bytes = static_cast<int>(min(static_cast<int64_t>(tiles), p.scale_tiles - first)) * kScaleTile;
    for (int i = 16 * threadIdx.x; i < bytes; i += 16 * kThreads) *reinterpret_cast<uint4*>(out + i) = *reinterpret_cast<const uint4*>(scales + i);
}

// ---------------------------------------------------------------- the matrix as it is
// A block of threads has 128 columns of 128 rows, a thread 16 columns of every 32nd row (NVFP4 a block; MXFP4 half of one, whose
// maximum it shares with its neighbour).  VEC: rows start on 16-byte boundaries; the loads of 128 bytes a thread are on their way
// together, which takes addresses without branches: 16 columns that are not wholly inside the matrix read the first ones instead,
// and their own elements one by one.  Other rows are fetched element by element, neighbouring lanes neighbouring elements, 32 rows
// at a time while those before are worked on, and go through shared memory.
// INSIDE: the block's rows and columns are all in the matrix.
constexpr int kPart = 16, kParts = kCols / kPart, kRowStep = kThreads / kParts, kChunks = kTileRows / kRowStep;
template <typename SRC> constexpr int kPitch = kCols + 16 / sizeof(SRC);

template <typename SRC>
__device__ __forceinline__ void unpack_part(const uint4 (&w)[kPart * sizeof(SRC) / 16], float (&v)[kPart]) {
#pragma unroll
    for (int i = 0; i < int(kPart * sizeof(SRC) / 16); ++i) {
        const uint32_t words[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (sizeof(SRC) == 4) v[4 * i + j] = __uint_as_float(words[j]);
            else { v[(8 * i + 2 * j) % kPart] = bf16_lo(words[j]); v[(8 * i + 2 * j + 1) % kPart] = bf16_hi(words[j]); }
        }
    }
}

// The scales of rows of a tile that do not exist.
__device__ __forceinline__ void no_rows(uint8_t* scales, int tiles, int first_row) {
    for (int t = 0; t < tiles; ++t)
        for (int r = first_row + threadIdx.x; r < kTileRows; r += kThreads) *reinterpret_cast<uint32_t*>(scales + t * kScaleTile + scale_at(r, 0)) = 0u;
}

// The 16 columns from `col` on of row r of the tile: codes (to `out`), scale, and what they add to the maximum.
template <int FMT, bool INSIDE>
__device__ __forceinline__ void finish_part(const QuantArgs& p, uint8_t* scales, int64_t row0, int64_t col, int part, int r, float g,
                                            uint8_t* out, const float (&v)[kPart], float& seen) {
    uint32_t top = top_bits(v);
    if (p.amax_out != nullptr) {
        if (top <= 0x7f800000u) {
            seen = fmaxf(seen, __uint_as_float(top));
        } else {
#pragma unroll
            for (int i = 0; i < kPart; ++i) seen = fmaxf(seen, fabsf(v[i]));
        }
    }
    if (FMT == FP8MLP_MXFP4) top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    uint32_t code[kPart / 8];
    uint32_t byte = quantise_block<FMT, kPart>(v, top, g, code);
    const bool here = INSIDE || row0 + r < p.rows;
    const int64_t block_col = FMT == FP8MLP_MXFP4 ? col & ~int64_t(31) : col;
    if (!INSIDE && (!here || block_col >= p.cols)) byte = 0;             // blocks that do not exist
    if (INSIDE || (here && col < ((p.cols + 31) & ~int64_t(31)))) st_global_v2(out, code[0], code[1]);
    const int b = FMT == FP8MLP_MXFP4 ? part >> 1 : part;
    if (FMT == FP8MLP_NVFP4 || (part & 1) == 0) scales[(b >> 2) * kScaleTile + scale_at(r, b & 3)] = static_cast<uint8_t>(byte);
}

template <typename SRC, int FMT, bool INSIDE>
__device__ __forceinline__ float quantise_aligned(const QuantArgs& p, uint8_t* scales, int64_t row0, int64_t col, int part, int r0, float g) {
    constexpr int kWords = kPart * sizeof(SRC) / 16, kBatch = 8 / kWords;
    float seen = 0.0f;
    const bool whole = INSIDE || col + kPart <= p.cols;
    const uint8_t* src = p.src + (row0 + r0) * p.ld + col * static_cast<int64_t>(sizeof(SRC));
    uint8_t* out = p.codes + (row0 + r0) * p.ld_codes + col / 2;
#pragma unroll 1
    for (int first = 0; first < kChunks; first += kBatch) {
        if (!INSIDE && row0 + first * kRowStep >= p.rows) {
            no_rows(scales, kCols / (4 * Fmt<FMT>::kBlock), first * kRowStep);
            break;
        }
        uint4 w[kBatch][kWords];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const uint8_t* at = src + (first + k) * kRowStep * p.ld;
            if (!INSIDE && !(whole && row0 + r0 + (first + k) * kRowStep < p.rows)) at = p.src;
#pragma unroll
            for (int i = 0; i < kWords; ++i) w[k][i] = ld_global_nc_v4(at + 16 * i);
        }
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const int r = r0 + (first + k) * kRowStep;
            float v[kPart];
            unpack_part<SRC>(w[k], v);
            if (!INSIDE && row0 + r >= p.rows) {
#pragma unroll
                for (int i = 0; i < kPart; ++i) v[i] = 0.0f;
            } else if (!INSIDE && !whole) {
                const SRC* at = reinterpret_cast<const SRC*>(src + (first + k) * kRowStep * p.ld);
#pragma unroll
                for (int i = 0; i < kPart; ++i) v[i] = col + i < p.cols ? to_f32(at[i]) : 0.0f;
            }
            finish_part<FMT, INSIDE>(p, scales, row0, col, part, r, g, out + (first + k) * kRowStep * p.ld_codes, v, seen);
        }
    }
    return seen;
}

template <typename SRC, int FMT>
__device__ __forceinline__ float quantise_unaligned(const QuantArgs& p, uint8_t* scales, int64_t row0, int64_t col0, int part, int r0, float g) {
    constexpr int kRowsPerWarp = kRowStep / (kThreads / 32), kPerLane = kCols / 32;
    constexpr int kBuffers = sizeof(SRC) == 4 ? 1 : 2;            // 17 KB either way
    __shared__ __align__(16) SRC stage[kBuffers][kRowStep][kPitch<SRC>];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    float seen = 0.0f;
    SRC next[kRowsPerWarp][kPerLane];
    auto fetch = [&](int chunk) {
#pragma unroll
        for (int k = 0; k < kRowsPerWarp; ++k) {
            const int64_t row = row0 + chunk * kRowStep + warp * kRowsPerWarp + k;
            const SRC* at = reinterpret_cast<const SRC*>(p.src + row * p.ld) + col0;
#pragma unroll
            for (int i = 0; i < kPerLane; ++i) next[k][i] = row < p.rows && col0 + lane + 32 * i < p.cols ? at[lane + 32 * i] : SRC(0);
        }
    };
    fetch(0);
#pragma unroll 1
    for (int chunk = 0; chunk < kChunks; ++chunk) {
        if (row0 + chunk * kRowStep >= p.rows) {
            no_rows(scales, kCols / (4 * Fmt<FMT>::kBlock), chunk * kRowStep);
            break;
        }
#pragma unroll
        for (int k = 0; k < kRowsPerWarp; ++k)
#pragma unroll
            for (int i = 0; i < kPerLane; ++i) stage[chunk % kBuffers][warp * kRowsPerWarp + k][lane + 32 * i] = next[k][i];
        __syncthreads();
        if (chunk + 1 < kChunks) fetch(chunk + 1);
        uint4 w[kPart * sizeof(SRC) / 16];
#pragma unroll
        for (int i = 0; i < int(kPart * sizeof(SRC) / 16); ++i) w[i] = reinterpret_cast<const uint4*>(&stage[chunk % kBuffers][r0][part * kPart])[i];
        if (kBuffers == 1) __syncthreads();
        float v[kPart];
        unpack_part<SRC>(w, v);
        finish_part<FMT, false>(p, scales, row0, col0 + part * kPart, part, r0 + chunk * kRowStep, g,
                                p.codes + (row0 + r0 + chunk * kRowStep) * p.ld_codes + (col0 + part * kPart) / 2, v, seen);
    }
    return seen;
}

template <typename SRC, int FMT, bool VEC>
__device__ __forceinline__ float quantise_tile(const QuantArgs& p, int64_t row_tile, int64_t col_tile, float g) {
    constexpr int kTiles = kCols / (4 * Fmt<FMT>::kBlock);
    __shared__ __align__(16) uint8_t scales[kTiles * kScaleTile];
    const int64_t row0 = row_tile * kTileRows, col0 = col_tile * kCols;
    const int part = threadIdx.x % kParts, r0 = threadIdx.x / kParts;
    float seen;
    if constexpr (!VEC) seen = quantise_unaligned<SRC, FMT>(p, scales, row0, col0, part, r0, g);
    else if (row0 + kTileRows <= p.rows && col0 + kCols <= p.cols) seen = quantise_aligned<SRC, FMT, true>(p, scales, row0, col0 + part * kPart, part, r0, g);
    else seen = quantise_aligned<SRC, FMT, false>(p, scales, row0, col0 + part * kPart, part, r0, g);
    __syncthreads();
    write_scales(p, scales, row_tile, col0 / (4 * Fmt<FMT>::kBlock), kTiles);
    return seen;
}

// ---------------------------------------------------------------- the transposed matrix
// Operand rows are the source's columns.  A thread takes two neighbouring columns over one block of source rows (a warp reads 64
// neighbouring columns of a row at once), a block of threads 128 columns over four blocks: one tile of scales.  All loads of a
// thread are on their way together (addresses past the matrix are moved to its last row and column, their values cleared); the
// codes go through shared memory, so that they leave in pieces of 32 or 64 bytes.  VEC: the source's columns come in pairs
// that can be read at once.
template <typename SRC, int FMT, bool VEC>
__device__ __forceinline__ float quantise_transposed_tile(const QuantArgs& p, int64_t row_tile, int64_t col_tile, float g) {
    constexpr int N = Fmt<FMT>::kBlock, kColsT = 4 * N, kCodePitch = kColsT / 2 + 16;
    __shared__ __align__(16) uint8_t scales[kScaleTile];
    __shared__ __align__(16) uint8_t codes[kTileRows * kCodePitch];
    const int64_t row0 = row_tile * kTileRows, col0 = col_tile * kColsT;
    const int pair = 2 * (threadIdx.x & 63), b = threadIdx.x >> 6, k0 = N * b;        // operand rows of the tile, block
    const int rows = static_cast<int>(min(p.rows - row0, static_cast<int64_t>(kTileRows)));
    const int cols = static_cast<int>(min(p.cols - col0, static_cast<int64_t>(kColsT)));
    float v[2][N];
    {
        const int c0 = VEC ? min(pair, rows - 2) : min(pair, rows - 1), c1 = min(pair + 1, rows - 1);      // (VEC: rows is even)
        const uint8_t* base = p.src + (col0 + min(k0, cols - 1)) * p.ld + row0 * static_cast<int64_t>(sizeof(SRC));
        const int last = max(cols - 1 - k0, 0);                 // rows of the source that lie behind the first of the thread's
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const SRC* at = reinterpret_cast<const SRC*>(base);
            if (i < last) base += p.ld;
            if constexpr (VEC && sizeof(SRC) == 4) {
                const float2 w = __ldg(reinterpret_cast<const float2*>(at + c0));
                v[0][i] = w.x; v[1][i] = w.y;
            } else if constexpr (VEC) {
                v[0][i] = __uint_as_float(__ldg(reinterpret_cast<const uint32_t*>(at + c0)));
            } else {
                v[0][i] = to_f32(__ldg(at + c0)); v[1][i] = to_f32(__ldg(at + c1));
            }
        }
        if constexpr (VEC && sizeof(SRC) == 2) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const uint32_t w = __float_as_uint(v[0][i]);
                v[0][i] = bf16_lo(w); v[1][i] = bf16_hi(w);
            }
        }
        if (rows < kTileRows || cols < kColsT) {
            const bool one = pair < rows, two = pair + 1 < rows;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const bool in = k0 + i < cols;
                v[0][i] = in && one ? v[0][i] : 0.0f;
                v[1][i] = in && two ? v[1][i] : 0.0f;
            }
        }
    }
    float seen = 0.0f;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const int r = pair + c;
        const uint32_t top = top_bits(v[c]);
        if (p.amax_out != nullptr) {
            if (top <= 0x7f800000u) {
                seen = fmaxf(seen, __uint_as_float(top));
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) seen = fmaxf(seen, fabsf(v[c][i]));
            }
        }
        uint32_t code[N / 8];
        const uint32_t byte = quantise_block<FMT, N>(v[c], top, g, code);
        scales[scale_at(r, b)] = static_cast<uint8_t>(r < rows && k0 < cols ? byte : 0u);
        if constexpr (N == 32) *reinterpret_cast<uint4*>(codes + r * kCodePitch + k0 / 2) = make_uint4(code[0], code[1], code[2], code[3]);
        else *reinterpret_cast<uint2*>(codes + r * kCodePitch + k0 / 2) = make_uint2(code[0], code[1]);
    }
    __syncthreads();
    write_scales(p, scales, row_tile, col_tile, 1);
    const int padded = (cols + 31) & ~31;
    for (int i = threadIdx.x; i < kTileRows * (kColsT / 32); i += kThreads) {
        const int r = i / (kColsT / 32), c = i % (kColsT / 32);
        if (r < rows && 32 * c < padded)
            *reinterpret_cast<uint4*>(p.codes + (row0 + r) * p.ld_codes + (col0 + 32 * c) / 2) = *reinterpret_cast<const uint4*>(codes + r * kCodePitch + 16 * c);
    }
    return seen;
}

// ---------------------------------------------------------------- kernels
// TRANSPOSED: of the source's transpose.  A block of threads to a tile.
template <typename SRC, int FMT, bool TRANSPOSED, bool VEC>
__global__ void __launch_bounds__(kThreads, TRANSPOSED && FMT == FP8MLP_MXFP4 ? 3 : 4) quantise_kernel(const QuantArgs p) {
    int64_t row_tile, col_tile;
    tile_of<TRANSPOSED>(p, row_tile, col_tile);
    grid_dependency_wait();
    grid_launch_dependents();
    const float g = FMT == FP8MLP_NVFP4 ? scale_of(p) : 1.0f;
    float seen;
    if constexpr (TRANSPOSED) seen = quantise_transposed_tile<SRC, FMT, VEC>(p, row_tile, col_tile, g);
    else seen = quantise_tile<SRC, FMT, VEC>(p, row_tile, col_tile, g);
    if (p.amax_out != nullptr) raise_amax(seen, p.amax_out);
}

// max |src| over the units first, first + step, .. of a matrix with a row stride, NaN left out.  A row is cut into units of 16 bytes
// on 16-byte boundaries, the first and the last of which it may fill in part.  FLAT: one row.
template <typename SRC, bool FLAT>
__device__ __forceinline__ float amax_of(const AmaxArgs& p, int64_t first_unit, int64_t step) {
    constexpr int kPer = 16 / sizeof(SRC);
    const int64_t units = p.units, step_rows = FLAT ? 0 : step / units, step_units = step - step_rows * units;
    int64_t unit = first_unit, row = FLAT ? 0 : unit / units;
    unit -= row * units;
    float seen = 0.0f;
    while (FLAT ? unit < units : row < p.rows) {
        uint4 w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            w[k] = make_uint4(0u, 0u, 0u, 0u);
            if (FLAT ? unit < units : row < p.rows) {
                const SRC* at = reinterpret_cast<const SRC*>(p.src + row * p.ld);
                const int64_t first = unit * kPer - static_cast<int64_t>((reinterpret_cast<uintptr_t>(at) & 15) / sizeof(SRC));
                if (first >= 0 && first + kPer <= p.cols) {
                    w[k] = ld_global_nc_v4(at + first);
                } else {
#pragma unroll
                    for (int e = 0; e < kPer; ++e)
                        if (first + e >= 0 && first + e < p.cols) seen = fmaxf(seen, fabsf(to_f32(at[first + e])));
                }
            }
            row += step_rows;
            unit += step_units;
            if (!FLAT && unit >= units) { unit -= units; ++row; }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t words[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (sizeof(SRC) == 4) seen = fmaxf(seen, fabsf(__uint_as_float(words[j])));
                else seen = fmaxf(seen, fmaxf(fabsf(bf16_lo(words[j])), fabsf(bf16_hi(words[j]))));
            }
        }
    }
    return seen;
}
template <typename SRC, bool FLAT>
__global__ void __launch_bounds__(kThreads) amax_kernel(const AmaxArgs p) {
    grid_dependency_wait();
    grid_launch_dependents();
    raise_amax(amax_of<SRC, FLAT>(p, static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x, static_cast<int64_t>(gridDim.x) * kThreads), p.amax);
}

// A small matrix with a scale of its own data (NVFP4) in one launch: the blocks of one cluster look for the maximum together,
// exchange it over distributed shared memory and share the tiles.
constexpr int kCluster = kWideCluster;
template <typename SRC, bool TRANSPOSED, bool VEC>
__global__ void __launch_bounds__(kThreads) quantise_small_kernel(const QuantArgs p, const AmaxArgs m, int tiles) {
    __shared__ float warp_max[kThreads / 32], block_max[kCluster];
    const int rank = static_cast<int>(cluster_ctarank());
    cluster_begin();
    grid_dependency_wait();
    grid_launch_dependents();
    float top = warp_max_nonneg(amax_of<SRC, false>(m, rank * kThreads + threadIdx.x, kCluster * kThreads));
    if ((threadIdx.x & 31) == 0) warp_max[threadIdx.x >> 5] = top;
    cluster_begun();
    __syncthreads();
    if (threadIdx.x < kCluster) {                     // to every block's list
        top = warp_max[0];
#pragma unroll
        for (int i = 1; i < kThreads / 32; ++i) top = fmaxf(top, warp_max[i]);
        st_cluster_f32(mapa_shared(smem_u32(&block_max[rank]), threadIdx.x), top);
    }
    cluster_sync_all();
    top = block_max[0];
#pragma unroll
    for (int i = 1; i < kCluster; ++i) top = fmaxf(top, block_max[i]);
    const float g = tensor_scale(top);
    if (rank == 0 && threadIdx.x == 0) {
        *m.amax = __float_as_uint(top);
        *p.scale = g;
    }
    for (int tile = rank; tile < tiles; tile += kCluster) {
        const int row_tile = tile / p.col_tiles;
        if constexpr (TRANSPOSED) quantise_transposed_tile<SRC, FP8MLP_NVFP4, VEC>(p, row_tile, tile - row_tile * p.col_tiles, g);
        else quantise_tile<SRC, FP8MLP_NVFP4, VEC>(p, row_tile, tile - row_tile * p.col_tiles, g);
        __syncthreads();                              // the tile's shared memory is free
    }
}

__global__ void scale_only_kernel(const unsigned int* amax, float* scale) {        // a matrix without elements
    grid_dependency_wait();
    grid_launch_dependents();
    *scale = tensor_scale(__uint_as_float(__ldcg(amax)));
}

// ---------------------------------------------------------------- back to values
struct DequantArgs {
    const uint8_t *codes, *scales;
    const float* scale;
    uint8_t* out;
    int64_t ld_codes, ld_out;             // bytes
    int64_t rows, cols;
    int col_tiles, scale_tiles;
};

// What a scale's byte stands for.
template <int FMT>
__device__ __forceinline__ float block_scale(uint32_t byte) {
    if constexpr (FMT == FP8MLP_MXFP4) {          // 2^(byte - 127); the smallest is subnormal in fp32, the last NaN
        return __uint_as_float(byte == 0xffu ? 0x7fffffffu : byte == 0u ? 0x00400000u : byte << 23);
    } else {
        float s, unused;
        e4m3x2_to_f32(byte, s, unused);
        return s;
    }
}

// The 16 columns of 8 bytes of codes.
template <int FMT>
__device__ __forceinline__ void values_of(uint2 code, float scale, float inv_g, float (&v)[16]) {
    const uint32_t words[2] = {code.x, code.y};
#pragma unroll
    for (int i = 0; i < 8; ++i) e2m1x2_to_f32((words[i / 4] >> (8 * (i & 3))) & 0xffu, v[2 * i], v[2 * i + 1]);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        v[i] = __fmul_rn(v[i], scale);            // exact, but for MXFP4 scales at the ends of fp32's range
        if constexpr (FMT == FP8MLP_NVFP4) v[i] = __fmul_rn(v[i], inv_g);
    }
}

// A thread takes 64 bytes of output of a row at a time, 32 columns of bf16 or 16 of fp32; the loads of its rows are on their way
// together.  ALIGN: bytes that output rows are aligned to (32 or 16).
template <typename DST, int FMT, int ALIGN>
__global__ void __launch_bounds__(kThreads) dequantise_kernel(const DequantArgs p) {
    constexpr int N = Fmt<FMT>::kBlock, kPer = 64 / sizeof(DST), kHalves = kPer / 16;
    constexpr int kPerRow = kColsBack / kPer, kStep = kThreads / kPerRow, kBatch = 4, kItems = kTileRows / kStep;
    const int64_t row_tile = blockIdx.x / p.col_tiles;
    const int64_t row0 = row_tile * kTileRows, col = (blockIdx.x - row_tile * p.col_tiles) * kColsBack + kPer * (threadIdx.x % kPerRow);
    grid_dependency_wait();
    grid_launch_dependents();
    if (col >= p.cols) return;
    const float inv_g = p.scale != nullptr ? __fdiv_rn(1.0f, *p.scale) : 1.0f;
    const int r0 = threadIdx.x / kPerRow;
    const int64_t block = col / N;                    // the first of the columns' blocks (two: NVFP4 to bf16)
    const uint8_t* scales = p.scales + (row_tile * p.scale_tiles + block / 4) * kScaleTile + (block & 3);
#pragma unroll 1
    for (int first = 0; first < kItems; first += kBatch) {
        if (row0 + first * kStep >= p.rows) break;
        uint2 code[kBatch][kHalves];
        uint32_t bytes[kBatch];
#pragma unroll
        for (int it = 0; it < kBatch; ++it) {
            const int r = static_cast<int>(min(static_cast<int64_t>(r0 + (first + it) * kStep), p.rows - 1 - row0));
            const uint8_t* at = p.codes + (row0 + r) * p.ld_codes + col / 2;
            if constexpr (kHalves == 2) {
                const uint4 w = ld_global_nc_v4(at);
                code[it][0] = make_uint2(w.x, w.y);
                code[it][1] = make_uint2(w.z, w.w);
            } else {
                code[it][0] = __ldg(reinterpret_cast<const uint2*>(at));
            }
            if constexpr (N == 16 && kHalves == 2) bytes[it] = __ldg(reinterpret_cast<const unsigned short*>(scales + scale_at(r, 0)));
            else bytes[it] = __ldg(scales + scale_at(r, 0));
        }
#pragma unroll
        for (int it = 0; it < kBatch; ++it) {
            const int64_t row = row0 + r0 + (first + it) * kStep;
            if (row >= p.rows) break;
            DST* out = reinterpret_cast<DST*>(p.out + row * p.ld_out) + col;
#pragma unroll
            for (int h = 0; h < kHalves; ++h) {       // 16 columns at a time
                float v[16];
                values_of<FMT>(code[it][h], block_scale<FMT>((N == 16 ? bytes[it] >> (8 * h) : bytes[it]) & 0xffu), inv_g, v);
                if (col + 16 * h + 16 <= p.cols) {
#pragma unroll
                    for (int i = 0; i < 16; i += 32 / sizeof(DST)) {
                        uint32_t w[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            if constexpr (sizeof(DST) == 4) w[k] = __float_as_uint(v[(i + k) % 16]);
                            else w[k] = cvt_bf16x2(v[(i + 2 * k) % 16], v[(i + 2 * k + 1) % 16]);
                        }
                        if constexpr (ALIGN >= 32) {
                            st_global_v8(out + 16 * h + i, w);
                        } else {
                            st_global_v4(out + 16 * h + i, w[0], w[1], w[2], w[3]);
                            st_global_v4(out + 16 * h + i + 16 / sizeof(DST), w[4], w[5], w[6], w[7]);
                        }
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (col + 16 * h + i < p.cols) {
                            if constexpr (sizeof(DST) == 4) out[16 * h + i] = v[i];
                            else out[16 * h + i] = static_cast<uint16_t>(cvt_bf16x2(v[i], 0.0f) & 0xffffu);
                        }
                }
            }
        }
    }
}

// The same for output rows on any boundary: 128 columns, 32 rows at a time, go through shared memory and leave in words of four
// bytes, neighbouring lanes neighbouring words (8191 x 4099 NVFP4 to bf16: 118 us with two columns a lane and a scale for each, 24).
// CHUNKS: times 32 rows to a block of threads.
template <typename DST, int FMT, int CHUNKS>
__global__ void __launch_bounds__(kThreads, 4) dequantise_narrow_kernel(const DequantArgs p) {
    constexpr int N = Fmt<FMT>::kBlock, kBuffers = sizeof(DST) == 4 ? 1 : 2, kRowsPerWarp = kRowStep / (kThreads / 32);
    __shared__ __align__(16) DST stage[kBuffers][kRowStep][kPitch<DST>];
    const int64_t row_group = blockIdx.x / p.col_tiles;
    const int64_t row0 = row_group * CHUNKS * kRowStep, col0 = (blockIdx.x - row_group * p.col_tiles) * kCols;
    const int row_in_tile = static_cast<int>(row0 % kTileRows);
    const int part = threadIdx.x % kParts, r0 = threadIdx.x / kParts, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    grid_dependency_wait();
    grid_launch_dependents();
    const float inv_g = p.scale != nullptr ? __fdiv_rn(1.0f, *p.scale) : 1.0f;
    // parts past the row's end take its last one, and rows past the matrix its last
    const int64_t col = min(col0 + part * kPart, (p.cols - 1) & ~int64_t(kPart - 1)), block = col / N;
    const uint8_t* scales = p.scales + (row0 / kTileRows * p.scale_tiles + block / 4) * kScaleTile;
    uint2 code[CHUNKS];
    uint32_t byte[CHUNKS];
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) {
        const int r = static_cast<int>(min(static_cast<int64_t>(r0 + k * kRowStep), p.rows - 1 - row0));
        code[k] = __ldg(reinterpret_cast<const uint2*>(p.codes + (row0 + r) * p.ld_codes + col / 2));
        byte[k] = __ldg(scales + scale_at(row_in_tile + r, static_cast<int>(block & 3)));
    }
    const int cols = static_cast<int>(min(p.cols - col0, static_cast<int64_t>(kCols)));
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) {
        if (row0 + k * kRowStep >= p.rows) break;
        float v[kPart];
        values_of<FMT>(code[k], block_scale<FMT>(byte[k]), inv_g, v);
        uint4* to = reinterpret_cast<uint4*>(&stage[k % kBuffers][r0][part * kPart]);
#pragma unroll
        for (int i = 0; i < int(kPart * sizeof(DST) / 16); ++i) {
            if constexpr (sizeof(DST) == 4) to[i] = make_uint4(__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]), __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3]));
            else to[i] = make_uint4(cvt_bf16x2(v[(8 * i) % kPart], v[(8 * i + 1) % kPart]), cvt_bf16x2(v[(8 * i + 2) % kPart], v[(8 * i + 3) % kPart]),
                                    cvt_bf16x2(v[(8 * i + 4) % kPart], v[(8 * i + 5) % kPart]), cvt_bf16x2(v[(8 * i + 6) % kPart], v[(8 * i + 7) % kPart]));
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kRowsPerWarp; ++i) {
            const int r = warp * kRowsPerWarp + i;
            if (row0 + k * kRowStep + r >= p.rows) break;
            DST* out = reinterpret_cast<DST*>(p.out + (row0 + k * kRowStep + r) * p.ld_out) + col0;
            const DST* from = stage[k % kBuffers][r];
            if constexpr (sizeof(DST) == 4) {
#pragma unroll
                for (int q = 0; q < kCols; q += 32)
                    if (q + lane < cols) out[q + lane] = from[q + lane];
            } else {
                const int odd = static_cast<int>(reinterpret_cast<uintptr_t>(out) >> 1) & 1;      // a row's first word may begin with its second column
#pragma unroll
                for (int q = 0; q < kCols; q += 64) {
                    const int c = q + 2 * lane + odd;
                    const uint32_t lo = from[min(c, kCols - 1)], hi = from[min(c + 1, kCols - 1)];
                    if (c + 1 < cols) *reinterpret_cast<uint32_t*>(out + c) = lo | (hi << 16);
                    else if (c < cols) out[c] = static_cast<DST>(lo);
                }
                if (odd && lane == 0) out[0] = from[0];
            }
        }
        if (kBuffers == 1) __syncthreads();
    }
}

// ---------------------------------------------------------------- host side
bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
constexpr int64_t kMost = int64_t(1) << 24;      // rows and columns
// One launch instead of three (its call 5.5 us, theirs 9.4) up to where 16 SMs take longer for the data: 256 x 1024 bf16 4.8 us on the
// device either way, 512 x 1024 7.4 and 4.9.
constexpr int64_t kSmallBytes = int64_t(512) << 10, kSmallTiles = 2 * kCluster;

constexpr unsigned int kLittleShared = 8;        // percent

template <typename SRC>
bool vec_rows(const void* src, int64_t ld, int64_t cols) { return aligned(src, 16) && ld % 16 == 0 && cols >= kPart; }
// pairs of columns can be read at once
template <typename SRC>
bool vec_pairs(const QuantArgs& a) { return aligned(a.src, 2 * sizeof(SRC)) && a.ld % (2 * sizeof(SRC)) == 0 && a.rows % 2 == 0; }

template <typename SRC, int FMT>
cudaError_t launch_quantise(const QuantArgs& a, bool transpose, dim3 grid, cudaStream_t st) {
    if (transpose)
        return vec_pairs<SRC>(a) ? launch_chained(quantise_kernel<SRC, FMT, true, true>, grid, dim3(kThreads), 0, st, a)
                                 : launch_chained(quantise_kernel<SRC, FMT, true, false>, grid, dim3(kThreads), 0, st, a);
    if (!vec_rows<SRC>(a.src, a.ld, a.cols)) return launch_chained(quantise_kernel<SRC, FMT, false, false>, grid, dim3(kThreads), 0, st, a);
    // behind the search for the maximum the SMs are divided nearly as needed, and asking again costs 4 us of blocks not set up early:
    // worth it for large matrices only (1531 x 512 fp32 6.0 us, asking again 9.7; 4096 x 4096 29.5 and 27.2; 11008 x 4096 70 and 62.6)
    const bool divided = a.amax_in != nullptr && a.rows * a.cols * static_cast<int64_t>(sizeof(SRC)) < (int64_t(64) << 20);
    return divided ? launch_chained(quantise_kernel<SRC, FMT, false, true>, grid, dim3(kThreads), 0, st, a)
                   : launch_chained_shared(kLittleShared, quantise_kernel<SRC, FMT, false, true>, grid, dim3(kThreads), 0, st, a);
}

template <typename SRC>
AmaxArgs amax_args(const void* src, int64_t ld, int64_t rows, int64_t cols, unsigned int* amax) {
    constexpr int64_t kPer = 16 / sizeof(SRC);
    if (ld == cols * static_cast<int64_t>(sizeof(SRC)) || rows == 1) { cols *= rows; rows = 1; }
    // a row that begins inside a unit reaches into one more than its length says
    const int64_t units = (cols + kPer - 1) / kPer + (aligned(src, 16) && (rows == 1 || ld % 16 == 0) ? 0 : 1);
    return AmaxArgs{static_cast<const uint8_t*>(src), ld, rows, cols, units, amax};
}

template <typename SRC>
cudaError_t launch_amax(const AmaxArgs& a, int sms, cudaStream_t st) {
    const int64_t blocks = (a.rows * a.units + 4 * kThreads - 1) / (4 * kThreads);
    const dim3 grid(static_cast<unsigned>(blocks < 8 * sms ? blocks : 8 * sms));
    return a.rows == 1 ? launch_chained_shared(kLittleShared, amax_kernel<SRC, true>, grid, dim3(kThreads), 0, st, a)
                       : launch_chained_shared(kLittleShared, amax_kernel<SRC, false>, grid, dim3(kThreads), 0, st, a);
}

template <typename SRC, bool TRANSPOSED, bool VEC>
cudaError_t launch_small(const QuantArgs& a, const AmaxArgs& m, int tiles, cudaStream_t st) {
    cudaError_t e = cudaFuncSetAttribute(quantise_small_kernel<SRC, TRANSPOSED, VEC>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(kCluster);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = kCluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, quantise_small_kernel<SRC, TRANSPOSED, VEC>, a, m, tiles);
}
template <typename SRC>
cudaError_t dispatch_small(const QuantArgs& a, const AmaxArgs& m, bool transpose, int tiles, cudaStream_t st) {
    if (transpose) return vec_pairs<SRC>(a) ? launch_small<SRC, true, true>(a, m, tiles, st) : launch_small<SRC, true, false>(a, m, tiles, st);
    return vec_rows<SRC>(a.src, a.ld, a.cols) ? launch_small<SRC, false, true>(a, m, tiles, st) : launch_small<SRC, false, false>(a, m, tiles, st);
}

}  // namespace
}  // namespace fp8mlp

using namespace fp8mlp;

extern "C" int64_t fp8mlp_fp4_scale_bytes(int fmt, int64_t rows, int64_t cols) {
    if ((fmt != FP8MLP_MXFP4 && fmt != FP8MLP_NVFP4) || rows < 0 || cols < 0 || rows > kMost || cols > kMost) return 0;
    const int64_t per_tile = 4 * (fmt == FP8MLP_MXFP4 ? 32 : 16);
    return (rows + kTileRows - 1) / kTileRows * ((cols + per_tile - 1) / per_tile) * kScaleTile;
}

extern "C" int fp8mlp_quantize_fp4(const void* src, int src_dtype, int64_t rows, int64_t cols, int64_t ld_src, int transpose,
                                   int fmt, int scale_mode, float* scale, float* amax, uint8_t* codes, int64_t ld_codes,
                                   uint8_t* block_scales, void* stream) {
    if (src_dtype != FP8MLP_BF16 && src_dtype != FP8MLP_F32) return FP8MLP_ERR_ARG;
    if (fmt != FP8MLP_MXFP4 && fmt != FP8MLP_NVFP4) return FP8MLP_ERR_ARG;
    const bool current = scale_mode == FP8MLP_SCALE_FROM_CURRENT_AMAX;
    if (scale_mode != FP8MLP_SCALE_GIVEN && !current) return FP8MLP_ERR_ARG;
    if (fmt == FP8MLP_MXFP4 && (scale != nullptr || current)) return FP8MLP_ERR_ARG;
    if (fmt == FP8MLP_NVFP4 && scale == nullptr) return FP8MLP_ERR_ARG;
    if (current && amax == nullptr) return FP8MLP_ERR_ARG;
    if (rows < 0 || cols < 0 || rows > kMost || cols > kMost || (rows > 1 && ld_src < cols)) return FP8MLP_ERR_SHAPE;
    const bool t = transpose != 0;
    const int64_t R = t ? cols : rows, C = t ? rows : cols;                 // of the operand
    if (ld_codes % 16 != 0 || (R > 0 && ld_codes < (C + 31) / 32 * 16)) return FP8MLP_ERR_SHAPE;
    const int width = t ? 4 * (fmt == FP8MLP_MXFP4 ? 32 : 16) : kCols;
    const int64_t tiles = (R + kTileRows - 1) / kTileRows * ((C + width - 1) / width);          // blocks of threads
    if (tiles > INT32_MAX) return FP8MLP_ERR_SHAPE;
    if (rows > 0 && cols > 0 && (src == nullptr || codes == nullptr || block_scales == nullptr)) return FP8MLP_ERR_ARG;
    const int bytes = src_dtype == FP8MLP_F32 ? 4 : 2;
    if (!aligned(src, bytes) || !aligned(codes, 16) || !aligned(block_scales, 16) || !aligned(scale, 4) || !aligned(amax, 4)) return FP8MLP_ERR_ALIGN;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int dev = 0, sms = 0;
    FP8MLP_CUDA_CHECK(cudaGetDevice(&dev));
    FP8MLP_CUDA_CHECK(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    bool one_launch = current && rows > 0 && cols > 0 && rows * cols * bytes <= kSmallBytes && tiles <= kSmallTiles;
    if (one_launch)
        if (int rc = wide_cluster_fits(&one_launch)) return rc;
    if (amax != nullptr && !one_launch)
        if (int rc = clear_float(amax, st)) return rc;
    unsigned int* amax_bits = reinterpret_cast<unsigned int*>(amax);
    if (rows == 0 || cols == 0) {
        if (current) {
            FP8MLP_CUDA_CHECK(launch_chained(scale_only_kernel, dim3(1), dim3(1), 0, st, static_cast<const unsigned int*>(amax_bits), scale));
            count_launch();
        }
        return FP8MLP_OK;
    }
    const int64_t ld = ld_src * bytes;
    const bool f32 = src_dtype == FP8MLP_F32;
    const AmaxArgs m = f32 ? amax_args<float>(src, ld, rows, cols, amax_bits) : amax_args<uint16_t>(src, ld, rows, cols, amax_bits);
    if (current && !one_launch) {
        FP8MLP_CUDA_CHECK(f32 ? launch_amax<float>(m, sms, st) : launch_amax<uint16_t>(m, sms, st));
        count_launch();
    }
    QuantArgs a{};
    a.src = static_cast<const uint8_t*>(src); a.ld = ld; a.rows = R; a.cols = C;
    a.codes = codes; a.scales = block_scales; a.ld_codes = ld_codes; a.scale = scale;
    a.amax_in = current ? amax_bits : nullptr;
    a.amax_out = current ? nullptr : amax_bits;
    const int per_tile = 4 * (fmt == FP8MLP_MXFP4 ? 32 : 16);
    a.scale_tiles = static_cast<int>((C + per_tile - 1) / per_tile);
    a.col_tiles = static_cast<int>((C + width - 1) / width);
    const dim3 grid(static_cast<unsigned>(tiles));
    if (one_launch) {
        FP8MLP_CUDA_CHECK(f32 ? dispatch_small<float>(a, m, t, static_cast<int>(tiles), st) : dispatch_small<uint16_t>(a, m, t, static_cast<int>(tiles), st));
        count_launch();
        return FP8MLP_OK;
    }
    const cudaError_t e = fmt == FP8MLP_MXFP4 ? (f32 ? launch_quantise<float, FP8MLP_MXFP4>(a, t, grid, st) : launch_quantise<uint16_t, FP8MLP_MXFP4>(a, t, grid, st))
                                              : (f32 ? launch_quantise<float, FP8MLP_NVFP4>(a, t, grid, st) : launch_quantise<uint16_t, FP8MLP_NVFP4>(a, t, grid, st));
    FP8MLP_CUDA_CHECK(e);
    count_launch();
    return FP8MLP_OK;
}

extern "C" int fp8mlp_dequantize_fp4(const uint8_t* codes, int64_t ld_codes, const uint8_t* block_scales, const float* scale,
                                     int64_t rows, int64_t cols, int fmt, void* out, int out_dtype, int64_t ld_out, void* stream) {
    if (out_dtype != FP8MLP_BF16 && out_dtype != FP8MLP_F32) return FP8MLP_ERR_ARG;
    if (fmt != FP8MLP_MXFP4 && fmt != FP8MLP_NVFP4) return FP8MLP_ERR_ARG;
    if (fmt == FP8MLP_MXFP4 && scale != nullptr) return FP8MLP_ERR_ARG;
    if (rows < 0 || cols < 0 || rows > kMost || cols > kMost || (rows > 1 && ld_out < cols)) return FP8MLP_ERR_SHAPE;
    if (ld_codes % 16 != 0 || (rows > 0 && ld_codes < (cols + 31) / 32 * 16)) return FP8MLP_ERR_SHAPE;
    const int align = aligned(out, 32) && ld_out * (out_dtype == FP8MLP_F32 ? 4 : 2) % 32 == 0   ? 32
                      : aligned(out, 16) && ld_out * (out_dtype == FP8MLP_F32 ? 4 : 2) % 16 == 0 ? 16
                                                                                                 : 1;
    const int width = align >= 16 ? kColsBack : kCols;
    const int64_t col_tiles = (cols + width - 1) / width;
    // rows on any boundary: few tiles are cut into four (1531 x 509, 48 tiles: 4.9 us, cut 2.5)
    const bool cut = align == 1 && (rows + kTileRows - 1) / kTileRows * col_tiles <= 256;
    const int tile_rows = cut ? kRowStep : kTileRows;
    const int64_t tiles = (rows + tile_rows - 1) / tile_rows * col_tiles;
    if (tiles > INT32_MAX) return FP8MLP_ERR_SHAPE;
    if (rows > 0 && cols > 0 && (codes == nullptr || block_scales == nullptr || out == nullptr)) return FP8MLP_ERR_ARG;
    const int bytes = out_dtype == FP8MLP_F32 ? 4 : 2;
    if (!aligned(codes, 16) || !aligned(block_scales, 16) || !aligned(scale, 4) || !aligned(out, bytes)) return FP8MLP_ERR_ALIGN;
    if (rows == 0 || cols == 0) return FP8MLP_OK;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    DequantArgs a{};
    a.codes = codes; a.scales = block_scales; a.scale = scale; a.out = static_cast<uint8_t*>(out);
    a.ld_codes = ld_codes; a.ld_out = ld_out * bytes; a.rows = rows; a.cols = cols;
    const int per_tile = 4 * (fmt == FP8MLP_MXFP4 ? 32 : 16);
    a.scale_tiles = static_cast<int>((cols + per_tile - 1) / per_tile);
    a.col_tiles = static_cast<int>(col_tiles);
    const dim3 grid(static_cast<unsigned>(tiles));
#define FP8MLP_DEQUANT(D, F)                                                                                  \
    (align == 32 ? launch_chained(dequantise_kernel<D, F, 32>, grid, dim3(kThreads), 0, st, a)                \
     : align == 16 ? launch_chained(dequantise_kernel<D, F, 16>, grid, dim3(kThreads), 0, st, a)              \
     : cut         ? launch_chained(dequantise_narrow_kernel<D, F, 1>, grid, dim3(kThreads), 0, st, a)        \
                   : launch_chained(dequantise_narrow_kernel<D, F, kChunks>, grid, dim3(kThreads), 0, st, a))
    const bool f32 = out_dtype == FP8MLP_F32;
    const cudaError_t e = fmt == FP8MLP_MXFP4 ? (f32 ? FP8MLP_DEQUANT(float, FP8MLP_MXFP4) : FP8MLP_DEQUANT(uint16_t, FP8MLP_MXFP4))
                                              : (f32 ? FP8MLP_DEQUANT(float, FP8MLP_NVFP4) : FP8MLP_DEQUANT(uint16_t, FP8MLP_NVFP4));
#undef FP8MLP_DEQUANT
    FP8MLP_CUDA_CHECK(e);
    count_launch();
    return FP8MLP_OK;
}
