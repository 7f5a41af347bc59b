// Root-mean-square norm with the residual's addition, its output optionally as E4M3 codes, and its gradient.
//
// Both directions are one pass over their rows: a row's units of 32 bytes lie in the registers of the threads that share it
// (as many as the row has units, a power of two; several rows per block where they are short), the row's sums go through
// shuffles and one barrier, and the blocks stay for many rows, so that the gain is read once per block and the next row's
// loads are on their way while the present row is summed and written.
#include "common.cuh"

#include <atomic>
#include <type_traits>

namespace fp8mlp {

namespace {

constexpr uint32_t kAll = 0xffffffffu;
constexpr int kMaxWarps = 32;
constexpr int kCluster = kWideCluster;      // blocks of the one cluster that takes a short batch as a whole

struct NormArgs {
    const uint8_t *x, *residual;
    uint8_t *h, *y;
    const float* gain;
    float *scale, *rstd;
    unsigned int* amax;
    int64_t T, ld_x, ld_res, ld_h, ld_y;      // row strides in bytes
    float eps, inv_d;
    double inv_d64;
    int units, tpr;                           // 32-byte units of a row; threads that share it
    int cluster;                              // the grid is one cluster: it finds the maximum by itself
};

struct NormBackArgs {
    const uint8_t *dy, *h, *dh;
    uint8_t* dx;
    const float *gain, *rstd;
    float* partial;                           // [grid][d], null: no gradient of the gain
    int64_t T, ld_dy, ld_h, ld_dh, ld_dx;
    float inv_d;
    int units, tpr, d;
    float* d_gain;                            // not null: the grid is one cluster, which adds the blocks' sums itself
};

template <typename SRC> struct Unit;          // 32 bytes of a row
template <> struct Unit<float> { static constexpr int kElems = 8; };
template <> struct Unit<uint16_t> { static constexpr int kElems = 16; };

// rows start on 16-byte boundaries; WIDE: all of them on 32-byte ones.  Plain loads, not the read-only path: h may be x.
// ONCE: nobody reads it soon again, so that L2 rather keeps what is written (16384 x 4096 forward: 81 -> 77 us; the gradient's
// time stays the same).
template <bool WIDE, bool ONCE = false>
__device__ __forceinline__ void load_unit(const uint8_t* p, uint32_t (&w)[8]) {
    if constexpr (WIDE && ONCE) {
        asm volatile("ld.global.L1::no_allocate.L2::evict_first.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                     : "l"(p) : "memory");
    } else if constexpr (WIDE) {
        asm volatile("ld.global.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                     : "l"(p) : "memory");
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(w[4 * i]), "=r"(w[4 * i + 1]), "=r"(w[4 * i + 2]), "=r"(w[4 * i + 3])
                         : "l"(p + 16 * i) : "memory");
    }
}
template <bool WIDE>
__device__ __forceinline__ void store_unit(uint8_t* p, const uint32_t (&w)[8]) {
    if constexpr (WIDE) {
        st_global_v8(p, w);
    } else {
        st_global_v4(p, w[0], w[1], w[2], w[3]);
        st_global_v4(p + 16, w[4], w[5], w[6], w[7]);
    }
}

template <typename SRC>
__device__ __forceinline__ float elem(const uint32_t (&w)[8], int i) {
    if constexpr (sizeof(SRC) == 4) return __uint_as_float(w[i]);
    else return (i & 1) ? bf16_hi(w[i >> 1]) : bf16_lo(w[i >> 1]);
}
template <typename SRC>                                       // elements i (even) and i + 1
__device__ __forceinline__ f32x2 elems(const uint32_t (&w)[8], int i) { return pack2(elem<SRC>(w, i), elem<SRC>(w, i + 1)); }
__device__ __forceinline__ float max3_abs(float a, float b, float c) {      // of the sizes; a NaN is not taken
    float r;
    asm("max.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
template <typename SRC>
__device__ __forceinline__ void pack_unit(const float (&v)[Unit<SRC>::kElems], uint32_t (&w)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (sizeof(SRC) == 4) w[i] = __float_as_uint(v[i]);
        else w[i] = cvt_bf16x2(v[2 * i], v[2 * i + 1]);
    }
}
// x + r, rounded once to the type
template <typename SRC>
__device__ __forceinline__ void add_unit(uint32_t (&w)[8], const uint32_t (&r)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (sizeof(SRC) == 4) w[i] = __float_as_uint(__fadd_rn(__uint_as_float(w[i]), __uint_as_float(r[i])));
        else asm("add.rn.bf16x2 %0, %0, %1;" : "+r"(w[i]) : "r"(r[i]));
    }
}
template <int N>
__device__ __forceinline__ void load_gain(const float* gain, int first, float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        const float4 q = gain != nullptr ? __ldg(reinterpret_cast<const float4*>(gain + first + i)) : make_float4(1.0f, 1.0f, 1.0f, 1.0f);
        v[i] = q.x; v[i + 1] = q.y; v[i + 2] = q.z; v[i + 3] = q.w;
    }
}

// Sum of one value (fp32, or 64 bits for norms whose output is codes) over the tpr threads of a row, and with MAX the maximum of another,
// held as an fp32 number >= 0 and what its rounding left off; every thread of the row gets them.  `part`: words for each warp; the
// caller alternates between two such arrays, so that one barrier per call is enough.
template <typename STAT> struct Part {
    STAT sum[kMaxWarps];
    float2 top[kMaxWarps];
};
// the maximum over a warp
__device__ __forceinline__ void warp_top(float& top, float& rest) {
    const float most = warp_max_nonneg(top);
    uint32_t key = __float_as_uint(rest);                 // in the order of whole numbers
    key = top == most ? (key ^ (static_cast<uint32_t>(static_cast<int32_t>(key) >> 31) | 0x80000000u)) : 0u;
    key = __reduce_max_sync(kAll, key);
    rest = __uint_as_float(key ^ (key & 0x80000000u ? 0x80000000u : 0xffffffffu));
    top = most;
}
// LEAN: where several warps have a row, their own sums are in fp32, and only those of the warps are added up in STAT.
template <bool MAX, bool LEAN, typename STAT>
__device__ __forceinline__ void over_row(STAT& sum, float lean_sum, float& top, float& rest, int tpr, Part<STAT>& part) {
    if (LEAN && tpr > 32) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) lean_sum = __fadd_rn(lean_sum, __shfl_xor_sync(kAll, lean_sum, o));
        sum = lean_sum;
    }
    for (int o = min(tpr, 32) >> 1; o > 0; o >>= 1) {
        if (LEAN && tpr > 32) break;
        sum += __shfl_xor_sync(kAll, sum, o);
        if (MAX && tpr < 32) {
            const float other = __shfl_xor_sync(kAll, top, o), other_rest = __shfl_xor_sync(kAll, rest, o);
            rest = other > top || (other == top && other_rest > rest) ? other_rest : rest;
            top = fmaxf(top, other);
        }
    }
    if (MAX && tpr >= 32) warp_top(top, rest);
    if (tpr <= 32) return;
    const int warp = threadIdx.x >> 5, per_row = tpr >> 5, first = warp & ~(per_row - 1);
    if ((threadIdx.x & 31) == 0) {
        part.sum[warp] = sum;
        if (MAX) part.top[warp] = make_float2(top, rest);
    }
    __syncthreads();
    // every warp adds up those of its row, a lane for each
    const int mine = first + (threadIdx.x & (per_row - 1));
    sum = part.sum[mine];
    for (int o = per_row >> 1; o > 0; o >>= 1) sum += __shfl_xor_sync(kAll, sum, o);
    if (MAX) {
        top = part.top[mine].x;
        rest = part.top[mine].y;
        warp_top(top, rest);
    }
}

// The E4M3 code of h * gain * factor (64 bits), rounded once: to fp32 with a last bit that says whether something was cut off, from
// where the conversion rounds to the code.
__device__ __forceinline__ float for_code(float h, float gain, double factor) {
    asm volatile("" : "+f"(gain));                // (the gain's 64-bit values are not to be made ahead of the loop and kept)
    const double v = static_cast<double>(h) * static_cast<double>(gain) * factor;
    const float cut = __double2float_rz(v);
    return static_cast<double>(cut) != v ? __uint_as_float(__float_as_uint(cut) | 1u) : cut;
}

// ---------------------------------------------------------------- forward
// NU: units per thread.  With one (d <= 16384 bf16, 8192 fp32) the next row is fetched ahead and the gain stays in registers.
// Codes (OUT != FP8MLP_RMS_SAME) are those next to the exact value: an fp32 product may land on the other side of a border between two
// codes (one in 10^6 does, each a step of 6 percent).  A row's sums are joined in 64 bits (bf16: those of its warps, of squares that
// have 16 bits), and the factor has a second fp32 number; a unit's codes are converted from its fp32 values a little increased and a
// little decreased, and where the two differ its products are taken again in 64 bits (one unit in 5000).
// Measured, 16384 x 4096 with residual: bf16 to codes 80 us (from fp32 products alone 77; 72 at the copy rate), with a scale per row 81,
// to bf16 88 (82); fp32 to codes 136 (133).  2048 x 16384 bf16 to codes 43 (36), fp32 94 (67: two units a thread, no row ahead).  16384
// rows of 5120, 6144, 7168 bf16 to codes: 111, 121, 133 (90, 108, 125): a row's threads are a power of two.  One token: 2.9 us, 2.5 from
// fp32 products.  What bounds it: DRAM, and the row's chain of reductions.  bf16 to codes spills 20 to 32 bytes a thread.
template <typename SRC, int BLOCK, int NU, bool WIDE, int OUT>
__global__ void __launch_bounds__(BLOCK, 1024 / BLOCK) norm_kernel(const NormArgs p) {
    constexpr int E = Unit<SRC>::kElems;
    constexpr bool kCodes = OUT != FP8MLP_RMS_SAME, kRows = OUT == FP8MLP_RMS_E4M3_ROWS;
    constexpr bool kLean = kCodes && sizeof(SRC) == 2;
    using Stat = typename std::conditional<kCodes, double, float>::type;
    __shared__ Part<Stat> part[2];
    __shared__ float warp_max[kMaxWarps];
    __shared__ float block_max[kCluster];
    if (p.cluster) cluster_begin();
    const int sub = threadIdx.x / p.tpr, u0 = threadIdx.x % p.tpr, rows = BLOCK / p.tpr;
    const int64_t step = static_cast<int64_t>(gridDim.x) * rows;
    int64_t row = static_cast<int64_t>(blockIdx.x) * rows + sub;
    grid_dependency_wait();
    grid_launch_dependents();
    float gain[E];
    if (NU == 1 && u0 < p.units) load_gain<E>(p.gain, u0 * E, gain);
    float scale = 1.0f, run_max = 0.0f;
    if (OUT == FP8MLP_RMS_E4M3) scale = *p.scale;
    uint32_t next[NU][8], next_res[NU][8];
    auto fetch = [&](int64_t r) {
#pragma unroll
        for (int k = 0; k < NU; ++k) {
            const int u = u0 + k * p.tpr;
            if (r < p.T && u < p.units) {
                load_unit<WIDE, true>(p.x + r * p.ld_x + 32 * u, next[k]);
                if (p.residual != nullptr) load_unit<WIDE, true>(p.residual + r * p.ld_res + 32 * u, next_res[k]);
            }
        }
    };
    fetch(row);
    int parity = 0;
    // every thread of the block makes the same number of rounds: rows past the end take part in the barriers only
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * rows; first < p.T; first += step, row += step, parity ^= 1) {
        const bool here = row < p.T;
        uint32_t h[NU][8];
        Stat sum = 0;                                       // of h^2
        float lean_sum = 0.0f;
        float top = 0.0f, top_rest = 0.0f;                  // max |h gain|, and what its rounding left off (a scale for the row)
#pragma unroll
        for (int k = 0; k < NU; ++k) {
            const int u = u0 + k * p.tpr;
            if (!here || u >= p.units) continue;
#pragma unroll
            for (int i = 0; i < 8; ++i) h[k][i] = next[k][i];
            if (p.residual != nullptr) {
                add_unit<SRC>(h[k], next_res[k]);
                if (p.h != nullptr) store_unit<WIDE>(p.h + row * p.ld_h + 32 * u, h[k]);
            }
            if (NU > 1) load_gain<E>(p.gain, u * E, gain);
            float s[E / 4];
#pragma unroll
            for (int j = 0; j < E / 4; ++j) {               // four elements, two an instruction
                const f32x2 a = elems<SRC>(h[k], 4 * j), b = elems<SRC>(h[k], 4 * j + 2);
                if constexpr (!kCodes || sizeof(SRC) == 2) {
                    float lo, hi;
                    unpack2(fma2(b, b, mul2(a, a)), lo, hi);
                    s[j] = __fadd_rn(lo, hi);
                }
                if constexpr (!kRows) {
                    float g[4];
                    unpack2(mul2(a, pack2(gain[4 * j], gain[4 * j + 1])), g[0], g[1]);
                    unpack2(mul2(b, pack2(gain[4 * j + 2], gain[4 * j + 3])), g[2], g[3]);
                    top = max3_abs(max3_abs(top, g[0], g[1]), g[2], g[3]);
                }
            }
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const float v = elem<SRC>(h[k], i);
                if constexpr (kCodes && sizeof(SRC) == 4) sum += static_cast<Stat>(v) * static_cast<Stat>(v);
                if constexpr (kRows) {
                    const float g = __fmul_rn(fabsf(v), fabsf(gain[i])), rest = __fmaf_rn(fabsf(v), fabsf(gain[i]), -g);
                    top_rest = g > top ? rest : top_rest;
                    top = fmaxf(top, g);
                }
            }
            if constexpr (kLean) {
                if (p.tpr > 32) lean_sum = __fadd_rn(lean_sum, __fadd_rn(__fadd_rn(s[0], s[1]), __fadd_rn(s[2], s[3])));
                else sum += (static_cast<Stat>(s[0]) + static_cast<Stat>(s[1])) + (static_cast<Stat>(s[2]) + static_cast<Stat>(s[3]));
            } else if constexpr (!kCodes) {
#pragma unroll
                for (int i = 0; i < E / 4; i += 2) sum += s[i] + s[i + 1];
            }
        }
        if (NU == 1) fetch(row + step);
        over_row<kRows, kLean>(sum, lean_sum, top, top_rest, p.tpr, part[parity]);
        float rstd, factor, factor_rest = 0.0f;             // the factor of codes, and what its rounding left off
        if constexpr (kCodes) {
            // one step of Newton's method for 1 / sqrt(mean), its residual 1 - mean rstd^2 with what the roundings of both left off
            float step;
            auto inverse_root = [&](double mean) {
                const float m = static_cast<float>(mean);
                rstd = __fdiv_rn(1.0f, __fsqrt_rn(m));
                step = 0.0f;
                if (rstd > 0.0f && !isinf(rstd)) {
                    const float square = __fmul_rn(rstd, rstd), square_rest = __fmaf_rn(rstd, rstd, -square), m_rest = static_cast<float>(mean - static_cast<double>(m));
                    step = __fmul_rn(__fmul_rn(0.5f, rstd), __fmaf_rn(-m_rest, square, __fmaf_rn(-m, square_rest, __fmaf_rn(-m, square, 1.0f))));
                }
            };
            const double mean = sum * p.inv_d64 + static_cast<double>(p.eps);
            inverse_root(mean);
            if (rstd > 0x1p50f) {                           // its square may leave fp32, or the mean: of 2^200 times the mean
                inverse_root(mean * 0x1p200);
                rstd = __fmul_rn(rstd, 0x1p100f);
                step = __fmul_rn(step, 0x1p100f);
            }
            // y = (h gain) factor
            factor = __fmul_rn(rstd, scale);
            factor_rest = __fmaf_rn(step, scale, __fmaf_rn(rstd, scale, -factor));
            rstd = __fadd_rn(rstd, step);
        } else {
            rstd = __fdiv_rn(1.0f, __fsqrt_rn(__fmaf_rn(sum, p.inv_d, p.eps)));
            factor = rstd;
        }
        if (here && u0 == 0 && p.rstd != nullptr) p.rstd[row] = rstd;
        if constexpr (kRows) {                              // codes with a scale of the row's own do not depend on rstd, as it cancels
            const float most = __fmul_rn(top, rstd), row_scale = __fdiv_rn(448.0f, most);
            const float to_codes = __fdiv_rn(448.0f, top);
            const bool sound = most > 0.0f && !isinf(most) && !isinf(row_scale) && !isinf(to_codes);
            if (sound) {
                factor = to_codes;
                factor_rest = __fmul_rn(__fmul_rn(to_codes, 1.0f / 448.0f), __fmaf_rn(-to_codes, top_rest, __fmaf_rn(-to_codes, top, 448.0f)));
            }
            if (here && u0 == 0) p.scale[row] = sound ? row_scale : 1.0f;
        } else {
            run_max = fmaxf(run_max, __fmul_rn(top, rstd));
        }
#pragma unroll
        for (int k = 0; k < NU; ++k) {
            const int u = u0 + k * p.tpr;
            if (!here || u >= p.units) continue;
            if (NU > 1) load_gain<E>(p.gain, u * E, gain);
            if constexpr (OUT == FP8MLP_RMS_SAME) {
                float v[E];
#pragma unroll
                for (int i = 0; i < E; i += 2)
                    unpack2(mul2(mul2(elems<SRC>(h[k], i), pack2(gain[i], gain[i + 1])), pack2(factor, factor)), v[i], v[i + 1]);
                uint32_t w[8];
                pack_unit<SRC>(v, w);
                store_unit<WIDE>(p.y + row * p.ld_y + 32 * u, w);
            } else {
                uint8_t* dst = p.y + row * p.ld_y + E * u;
                float v[E];
#pragma unroll
                for (int i = 0; i < E; ++i) v[i] = __fmul_rn(__fmul_rn(elem<SRC>(h[k], i), gain[i]), factor);
                // The exact values lie between these: two products, the factor's product with the scale and 1 / rms (half a rounding of
                // the mean, the root, the division) are 5.5 roundings of 2^-24 off, the products below one more; 2^-21 are eight.
                const f32x2 more = pack2(1.0f + 0x1p-21f, 1.0f + 0x1p-21f), less = pack2(1.0f - 0x1p-21f, 1.0f - 0x1p-21f);
                uint32_t c[E / 4], differ = 0;
#pragma unroll
                for (int i = 0; i < E / 4; ++i) {
                    const f32x2 a = pack2(v[4 * i], v[4 * i + 1]), b = pack2(v[4 * i + 2], v[4 * i + 3]);
                    float hi[4], lo[4];
                    unpack2(mul2(a, more), hi[0], hi[1]);
                    unpack2(mul2(b, more), hi[2], hi[3]);
                    unpack2(mul2(a, less), lo[0], lo[1]);
                    unpack2(mul2(b, less), lo[2], lo[3]);
                    c[i] = cvt_fp8x4<FP8MLP_E4M3>(hi[0], hi[1], hi[2], hi[3]);
                    differ |= c[i] ^ cvt_fp8x4<FP8MLP_E4M3>(lo[0], lo[1], lo[2], lo[3]);
                }
                // (a factor beyond these may bring h gain back from where fp32 has few bits, or none)
                if (differ != 0 || fabsf(factor) > 0x1p60f || fabsf(factor) < 0x1p-60f) {
                    const double exact = static_cast<double>(factor) + static_cast<double>(isnan(factor_rest) ? 0.0f : factor_rest);
#pragma unroll
                    for (int i = 0; i < E / 4; ++i)
                        c[i] = cvt_fp8x4<FP8MLP_E4M3>(for_code(elem<SRC>(h[k], 4 * i), gain[4 * i], exact), for_code(elem<SRC>(h[k], 4 * i + 1), gain[4 * i + 1], exact),
                                                      for_code(elem<SRC>(h[k], 4 * i + 2), gain[4 * i + 2], exact), for_code(elem<SRC>(h[k], 4 * i + 3), gain[4 * i + 3], exact));
                }
                if constexpr (E == 16) st_global_v4(dst, c[0], c[1], c[2], c[3]); else st_global_v2(dst, c[0], c[1]);
            }
        }
        if (NU > 1) fetch(row + step);
    }
    if (OUT != FP8MLP_RMS_E4M3_ROWS && p.amax != nullptr) {
        __syncthreads();
        run_max = warp_max_nonneg(run_max);
        if ((threadIdx.x & 31) == 0) warp_max[threadIdx.x >> 5] = run_max;
        __syncthreads();
        if (threadIdx.x < 32) {
            run_max = warp_max_nonneg(threadIdx.x < BLOCK / 32 ? warp_max[threadIdx.x] : 0.0f);
            // a single block or cluster has the whole maximum (nobody cleared the word for it then)
            if (threadIdx.x == 0 && gridDim.x == 1) *p.amax = __float_as_uint(run_max);
            else if (threadIdx.x == 0 && !p.cluster && run_max > 0.0f) atomicMax(p.amax, __float_as_uint(run_max));
        }
        if (p.cluster) {
            cluster_begun();
            if (threadIdx.x == 0) st_cluster_f32(mapa_shared(smem_u32(&block_max[cluster_ctarank()]), 0), run_max);
            cluster_sync_all();
            if (blockIdx.x == 0 && threadIdx.x < 32) {
                run_max = warp_max_nonneg(threadIdx.x < kCluster ? block_max[threadIdx.x] : 0.0f);
                if (threadIdx.x == 0) *p.amax = __float_as_uint(run_max);
            }
        }
    }
}

// ---------------------------------------------------------------- backward
// A thread keeps the columns of its units through all rows of its block and sums their part of d_gain in registers (NU = 1)
// or in its own words of shared memory; blocks leave one row of partial sums each, which a second kernel
// adds in their order; a cluster that has the whole batch adds them over distributed shared memory.
// Measured with the residual stream's gradient, 16384 x 4096: bf16 88.7 us (82 at the copy rate), fp32 209 (164).  NU > 1: 2048 x 16384
// bf16 89 (41), fp32 160 (82), 4096 x 8192 fp32 119 (82): by count, lanes' words of shared memory share banks (8 or 16 to one);
// no row is fetched ahead, and four units of fp32 spill 332 bytes.  16384 rows of 5120, 6144, 7168 bf16: 143, 152, 165 (102, 123, 143), one block to an SM.
template <typename SRC, int BLOCK, int NU, bool WIDE>
__global__ void __launch_bounds__(BLOCK) norm_backward_kernel(const NormBackArgs p) {
    constexpr int E = Unit<SRC>::kElems;
    __shared__ Part<float> part_sum[2];
    extern __shared__ float d_gain_row[];                        // [d]: NU > 1, or where several rows share a block
    const int sub = threadIdx.x / p.tpr, u0 = threadIdx.x % p.tpr, rows = BLOCK / p.tpr;
    const int64_t step = static_cast<int64_t>(gridDim.x) * rows;
    int64_t row = static_cast<int64_t>(blockIdx.x) * rows + sub;
    const bool together = p.d_gain != nullptr, want = p.partial != nullptr || together;
    float gain[E], acc[E];
#pragma unroll
    for (int i = 0; i < E; ++i) acc[i] = 0.0f;
    if (NU > 1 && want)
        for (int i = threadIdx.x; i < p.d; i += BLOCK) d_gain_row[i] = 0.0f;
    grid_dependency_wait();
    grid_launch_dependents();
    if (NU == 1 && u0 < p.units) load_gain<E>(p.gain, u0 * E, gain);
    if (NU > 1) __syncthreads();
    uint32_t next_dy[NU][8], next_h[NU][8];
    float next_rstd = 0.0f;
    auto fetch = [&](int64_t r) {
#pragma unroll
        for (int k = 0; k < NU; ++k) {
            const int u = u0 + k * p.tpr;
            if (r < p.T && u < p.units) {
                load_unit<WIDE>(p.dy + r * p.ld_dy + 32 * u, next_dy[k]);
                load_unit<WIDE>(p.h + r * p.ld_h + 32 * u, next_h[k]);
            }
        }
        if (r < p.T) next_rstd = __ldg(p.rstd + r);
    };
    fetch(row);
    int parity = 0;
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * rows; first < p.T; first += step, row += step, parity ^= 1) {
        const bool here = row < p.T;
        const float rstd = next_rstd;
        uint32_t dy[NU][8], h[NU][8], dh[NU][8];
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < NU; ++k) {
            const int u = u0 + k * p.tpr;
            if (!here || u >= p.units) continue;
            if (p.dh != nullptr) load_unit<WIDE>(p.dh + row * p.ld_dh + 32 * u, dh[k]);
            if (NU > 1) load_gain<E>(p.gain, u * E, gain);
#pragma unroll
            for (int i = 0; i < 8; ++i) { dy[k][i] = next_dy[k][i]; h[k][i] = next_h[k][i]; }
            float s[2] = {0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const float unit = __fmul_rn(elem<SRC>(h[k], i), rstd), d = elem<SRC>(dy[k], i);
                s[i & 1] = __fmaf_rn(__fmul_rn(d, gain[i]), unit, s[i & 1]);
                if (NU == 1) acc[i] = __fmaf_rn(d, unit, acc[i]);
                else if (want) d_gain_row[u * E + i] = __fmaf_rn(d, unit, d_gain_row[u * E + i]);
            }
            sum = __fadd_rn(sum, __fadd_rn(s[0], s[1]));
        }
        if (NU == 1) fetch(row + step);
        float unused = 0.0f;
        over_row<false, false>(sum, 0.0f, unused, unused, p.tpr, part_sum[parity]);
        const float mean = __fmul_rn(sum, p.inv_d);
#pragma unroll
        for (int k = 0; k < NU; ++k) {
            const int u = u0 + k * p.tpr;
            if (!here || u >= p.units) continue;
            if (NU > 1) load_gain<E>(p.gain, u * E, gain);
            float v[E];
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const float unit = __fmul_rn(elem<SRC>(h[k], i), rstd), g = __fmul_rn(elem<SRC>(dy[k], i), gain[i]);
                v[i] = __fmul_rn(rstd, __fmaf_rn(-unit, mean, g));
                if (p.dh != nullptr) v[i] = __fadd_rn(v[i], elem<SRC>(dh[k], i));
            }
            uint32_t w[8];
            pack_unit<SRC>(v, w);
            store_unit<WIDE>(p.dx + row * p.ld_dx + 32 * u, w);
        }
        if (NU > 1) fetch(row + step);
    }
    if (!want) return;
    float* out = p.partial + static_cast<int64_t>(blockIdx.x) * p.d;
    if (NU == 1) {
        if (rows == 1 && !together) {
            if (u0 < p.units)
#pragma unroll
                for (int i = 0; i < E; i += 4) *reinterpret_cast<float4*>(out + u0 * E + i) = make_float4(acc[i], acc[i + 1], acc[i + 2], acc[i + 3]);
            return;
        }
        // the rows of a warp first, then warp after warp
        for (int o = p.tpr; o < 32; o <<= 1)
#pragma unroll
            for (int i = 0; i < E; ++i) acc[i] = __fadd_rn(acc[i], __shfl_xor_sync(kAll, acc[i], o));
        const bool speaks = p.tpr >= 32 || (threadIdx.x & 31) < p.tpr;
        const int turns = p.tpr >= 32 ? rows : BLOCK / 32, mine = p.tpr >= 32 ? sub : threadIdx.x >> 5;
        for (int turn = 0; turn < turns; ++turn) {
            if (turn == mine && speaks && u0 < p.units)
#pragma unroll
                for (int i = 0; i < E; ++i) d_gain_row[u0 * E + i] = turn == 0 ? acc[i] : __fadd_rn(d_gain_row[u0 * E + i], acc[i]);
            __syncthreads();
        }
    }
    if (together) {
        // every block adds its share of the columns over all blocks' rows of sums, in the order of their ranks
        cluster_sync_all();
        for (int i = blockIdx.x * BLOCK + threadIdx.x; i < p.d; i += kCluster * BLOCK) {
            const uint32_t at = smem_u32(d_gain_row + i);
            float v[kCluster];
#pragma unroll
            for (int b = 0; b < kCluster; ++b) v[b] = ld_cluster_f32(mapa_shared(at, b));
#pragma unroll
            for (int b = 1; b < kCluster; ++b) v[0] = __fadd_rn(v[0], v[b]);
            p.d_gain[i] = v[0];
        }
        cluster_sync_all();                                      // nobody leaves while its sums are read
        return;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < p.d; i += BLOCK) out[i] = d_gain_row[i];
}

// d_gain[i] = sum of the blocks' partial sums: 64 columns a block, 16 lanes to a row; every one of the 64 half-warps takes every 64th
// partial row and has its loads on their way together
constexpr int kGainThreads = 1024, kGainCols = 64, kGainRows = kGainThreads / 16;
__global__ void __launch_bounds__(kGainThreads) norm_gain_kernel(const float* partial, int n_partial, int d, float* d_gain) {
    __shared__ float4 part[kGainRows][16];
    const int lane = threadIdx.x & 15, sub = threadIdx.x >> 4, col = blockIdx.x * kGainCols + 4 * lane;
    grid_dependency_wait();
    grid_launch_dependents();
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    auto add = [](float4& a, const float4& b) {
        a.x = __fadd_rn(a.x, b.x); a.y = __fadd_rn(a.y, b.y); a.z = __fadd_rn(a.z, b.z); a.w = __fadd_rn(a.w, b.w);
    };
    if (col < d) {
        const float* at = partial + col;
        for (int i = sub; i < n_partial; i += 5 * kGainRows) {
            float4 v[5];
#pragma unroll
            for (int k = 0; k < 5; ++k) {
                const int row = min(i + k * kGainRows, n_partial - 1);
                v[k] = __ldcg(reinterpret_cast<const float4*>(at + static_cast<int64_t>(row) * d));
            }
#pragma unroll
            for (int k = 0; k < 5; ++k)
                if (i + k * kGainRows < n_partial) add(sum, v[k]);
        }
    }
    part[sub][lane] = sum;
    __syncthreads();
    if (threadIdx.x < kGainCols && blockIdx.x * kGainCols + threadIdx.x < d) {
        const float* mine = reinterpret_cast<const float*>(part) + threadIdx.x;
        float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < kGainRows; ++k) v[k & 3] = __fadd_rn(v[k & 3], mine[kGainCols * k]);
        d_gain[blockIdx.x * kGainCols + threadIdx.x] = __fadd_rn(__fadd_rn(v[0], v[1]), __fadd_rn(v[2], v[3]));
    }
}

// ---------------------------------------------------------------- host side
bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

int sm_count_of_current(int* sms) {
    int dev = 0;
    FP8MLP_CUDA_CHECK(cudaGetDevice(&dev));
    FP8MLP_CUDA_CHECK(cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev));
    return FP8MLP_OK;
}

struct RowShape { int units, tpr, block, nu; };
// threads and units per row, at most `most` threads (forward 1024, backward 512: its registers)
RowShape row_shape(int64_t d, int elems, int most) {
    RowShape s;
    s.units = static_cast<int>(d / elems);
    s.block = s.units <= 256 ? 256 : s.units <= 512 || most == 512 ? 512 : 1024;
    s.tpr = 1;
    while (s.tpr < s.units && s.tpr < s.block) s.tpr <<= 1;
    const int need = (s.units + s.tpr - 1) / s.tpr;
    s.nu = need <= 2 ? need : 4;
    return s;
}

// Whether one cluster takes the batch, without a launch before (which clears the maximum) or after it (which adds up the gradient of
// the gain): a call takes 1.8 us less, which is the host's time (32 x 4096 bf16: forward 6.2 and 8.0 us, backward 7.2 and 9.0).  On the
// device alone, as a captured graph runs, one round of its blocks takes 3.7 us and two launches 4.1 forward, 5.4 and 4.6 backward; two
// rounds (32 x 4096) 4.8 and 4.2, 6.2 and 4.9; four (64 x 4096) 6.8 and 4.4, 7.8 and 5.4.  Wide rows take longer than a launch already
// in their second round.
bool one_cluster_does(const RowShape& s, int64_t blocks) { return blocks <= (s.nu == 1 ? 2 : 1) * kCluster; }

// a row stride in elements -> bytes; false where it is no multiple of 16 bytes or shorter than the row
bool stride_ok(int64_t T, int64_t ld, int64_t d, int bytes) { return T <= 1 || (ld >= d && ld * bytes % 16 == 0); }

// A chained launch, or (one_cluster) of a grid that is one cluster.
template <typename ARGS>
cudaError_t launch_rows(void (*kernel)(ARGS), bool one_cluster, dim3 grid, int block, size_t smem, cudaStream_t st, const ARGS& a) {
    if (!one_cluster) return launch_chained(kernel, grid, dim3(block), smem, st, a);
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = kCluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, a);
}

template <typename SRC, int BLOCK, int NU, bool WIDE>
cudaError_t launch_norm(const NormArgs& a, int out, dim3 grid, cudaStream_t st) {
    const bool one = a.cluster != 0;
    switch (out) {
        case FP8MLP_RMS_SAME: return launch_rows(norm_kernel<SRC, BLOCK, NU, WIDE, FP8MLP_RMS_SAME>, one, grid, BLOCK, 0, st, a);
        case FP8MLP_RMS_E4M3: return launch_rows(norm_kernel<SRC, BLOCK, NU, WIDE, FP8MLP_RMS_E4M3>, one, grid, BLOCK, 0, st, a);
        default: return launch_rows(norm_kernel<SRC, BLOCK, NU, WIDE, FP8MLP_RMS_E4M3_ROWS>, one, grid, BLOCK, 0, st, a);
    }
}

template <typename SRC, int BLOCK, int NU, bool WIDE>
cudaError_t launch_norm_backward(const NormBackArgs& a, size_t smem, dim3 grid, cudaStream_t st) {
    if (smem + 2 * sizeof(Part<float>) > 48 * 1024) {        // with the kernel's own, more than a launch has without asking
        cudaError_t e = cudaFuncSetAttribute(norm_backward_kernel<SRC, BLOCK, NU, WIDE>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             FP8MLP_MAX_NORM_WIDTH * 4);
        if (e != cudaSuccess) return e;
    }
    return launch_rows(norm_backward_kernel<SRC, BLOCK, NU, WIDE>, a.d_gain != nullptr, grid, BLOCK, smem, st, a);
}

// the instantiation for a shape: F<SRC, BLOCK, NU, WIDE>; a row of bf16 has half as many units as one of fp32
template <typename SRC> constexpr int kMostUnits = FP8MLP_MAX_NORM_WIDTH / Unit<SRC>::kElems;
#define FP8MLP_NORM_TYPES(PICK, F, ...)                                                                                   \
    (dtype == FP8MLP_F32 ? (wide ? PICK(F, float, true, __VA_ARGS__) : PICK(F, float, false, __VA_ARGS__))                 \
                         : (wide ? PICK(F, uint16_t, true, __VA_ARGS__) : PICK(F, uint16_t, false, __VA_ARGS__)))
#define FP8MLP_NORM_FORWARD(F, SRC, WIDE, ...)                                                                            \
    (s.block == 256 ? F<SRC, 256, 1, WIDE>(__VA_ARGS__) : s.block == 512 ? F<SRC, 512, 1, WIDE>(__VA_ARGS__)               \
     : s.nu == 1 ? F<SRC, 1024, 1, WIDE>(__VA_ARGS__) : F<SRC, 1024, kMostUnits<SRC> / 1024, WIDE>(__VA_ARGS__))
#define FP8MLP_NORM_BACKWARD(F, SRC, WIDE, ...)                                                                           \
    (s.block == 256 ? F<SRC, 256, 1, WIDE>(__VA_ARGS__) : s.nu == 1 ? F<SRC, 512, 1, WIDE>(__VA_ARGS__)                    \
     : s.nu == 2 ? F<SRC, 512, 2, WIDE>(__VA_ARGS__) : F<SRC, 512, kMostUnits<SRC> / 512, WIDE>(__VA_ARGS__))

}  // namespace

// Asked once for each device: a part of a GPU may not have that many SMs side by side.  The kernel asked for has 64 registers for
// each of 1024 threads, all of an SM; blocks that take less fit where these do.
int wide_cluster_fits(bool* fits) {
    static std::atomic<int> known[64];                       // 1 + the answer
    int dev = 0;
    FP8MLP_CUDA_CHECK(cudaGetDevice(&dev));
    const int answer = dev < 64 ? known[dev].load(std::memory_order_relaxed) : 0;
    *fits = answer == 2;
    if (answer != 0) return FP8MLP_OK;
    const auto kernel = norm_kernel<uint16_t, 1024, 1, true, FP8MLP_RMS_SAME>;
    FP8MLP_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(kWideCluster);
    cfg.blockDim = dim3(1024);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = kWideCluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int clusters = 0;
    if (cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg) != cudaSuccess) {      // a size that the device does not know: it does not fit
        cudaGetLastError();
        clusters = 0;
    }
    *fits = clusters > 0;
    if (dev < 64) known[dev].store(*fits ? 2 : 1, std::memory_order_relaxed);
    return FP8MLP_OK;
}

}  // namespace fp8mlp

using namespace fp8mlp;

extern "C" int fp8mlp_rmsnorm(int64_t T, int64_t d, int dtype, const void* x, int64_t ld_x, const void* residual,
                              int64_t ld_residual, void* h_out, int64_t ld_h, const float* gain, float eps, int out_kind, void* y,
                              int64_t ld_y, float* scale, float* amax, float* rstd, void* stream) {
    if (dtype != FP8MLP_BF16 && dtype != FP8MLP_F32) return FP8MLP_ERR_ARG;
    if (out_kind < FP8MLP_RMS_SAME || out_kind > FP8MLP_RMS_E4M3_ROWS) return FP8MLP_ERR_ARG;
    if (h_out != nullptr && residual == nullptr) return FP8MLP_ERR_ARG;
    if (out_kind == FP8MLP_RMS_E4M3_ROWS && amax != nullptr) return FP8MLP_ERR_ARG;
    if (!(eps >= 0.0f)) return FP8MLP_ERR_ARG;
    const int bytes = dtype == FP8MLP_F32 ? 4 : 2, out_bytes = out_kind == FP8MLP_RMS_SAME ? bytes : 1;
    if (T < 0 || T > (int64_t(1) << 40) || d < 16 || d % 16 != 0 || d > FP8MLP_MAX_NORM_WIDTH) return FP8MLP_ERR_SHAPE;
    if (!stride_ok(T, ld_x, d, bytes) || !stride_ok(T, ld_y, d, out_bytes)) return FP8MLP_ERR_SHAPE;
    if (residual != nullptr && !stride_ok(T, ld_residual, d, bytes)) return FP8MLP_ERR_SHAPE;
    if (h_out != nullptr && !stride_ok(T, ld_h, d, bytes)) return FP8MLP_ERR_SHAPE;
    if (T > 0 && (x == nullptr || y == nullptr)) return FP8MLP_ERR_ARG;
    if (y != nullptr && (y == x || y == residual || y == h_out)) return FP8MLP_ERR_ARG;
    // in place, a row of the output has to lie over its own row of the input: over another, it is written before that is read, or after
    if (h_out != nullptr && T > 1 && ((h_out == x && ld_h != ld_x) || (h_out == residual && ld_h != ld_residual))) return FP8MLP_ERR_ARG;
    if (out_kind == FP8MLP_RMS_E4M3 && scale == nullptr) return FP8MLP_ERR_ARG;
    if (out_kind == FP8MLP_RMS_E4M3_ROWS && T > 0 && scale == nullptr) return FP8MLP_ERR_ARG;
    if (!aligned(x, 16) || !aligned(residual, 16) || !aligned(h_out, 16) || !aligned(y, 16) || !aligned(gain, 16)) return FP8MLP_ERR_ALIGN;
    if (!aligned(scale, 4) || !aligned(amax, 4) || !aligned(rstd, 4)) return FP8MLP_ERR_ALIGN;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (T == 0) return amax != nullptr ? clear_float(amax, st) : FP8MLP_OK;
    int sms = 0;
    if (int rc = sm_count_of_current(&sms)) return rc;
    const RowShape s = row_shape(d, 32 / bytes, 1024);
    NormArgs a{};
    a.x = static_cast<const uint8_t*>(x); a.residual = static_cast<const uint8_t*>(residual);
    a.h = static_cast<uint8_t*>(h_out); a.y = static_cast<uint8_t*>(y);
    a.gain = gain; a.scale = scale; a.rstd = rstd; a.amax = reinterpret_cast<unsigned int*>(amax);
    a.T = T; a.ld_x = ld_x * bytes; a.ld_res = ld_residual * bytes; a.ld_h = ld_h * bytes; a.ld_y = ld_y * out_bytes;
    a.eps = eps; a.inv_d = 1.0f / static_cast<float>(d); a.inv_d64 = 1.0 / static_cast<double>(d); a.units = s.units; a.tpr = s.tpr;
    auto on32 = [&](const void* q, int64_t ld) { return aligned(q, 32) && (T <= 1 || ld % 32 == 0); };
    const bool wide = on32(x, a.ld_x) && (residual == nullptr || on32(residual, a.ld_res)) && (h_out == nullptr || on32(h_out, a.ld_h)) &&
                      (out_kind != FP8MLP_RMS_SAME || on32(y, a.ld_y));
    const int64_t rows = s.block / s.tpr, blocks = (T + rows - 1) / rows, most = static_cast<int64_t>(sms) * (1024 / s.block);
    bool one_cluster = amax != nullptr && blocks > 1 && one_cluster_does(s, blocks);
    if (one_cluster)
        if (int rc = wide_cluster_fits(&one_cluster)) return rc;
    a.cluster = one_cluster ? 1 : 0;
    const dim3 grid(static_cast<unsigned>(a.cluster ? kCluster : blocks < most ? blocks : most));
    if (amax != nullptr && grid.x > 1 && !a.cluster)
        if (int rc = clear_float(amax, st)) return rc;
    FP8MLP_CUDA_CHECK(FP8MLP_NORM_TYPES(FP8MLP_NORM_FORWARD, launch_norm, a, out_kind, grid, st));
    count_launch();
    return FP8MLP_OK;
}

extern "C" int fp8mlp_rmsnorm_backward(int64_t T, int64_t d, int dtype, const void* dy, int64_t ld_dy, const void* h, int64_t ld_h,
                                       const float* gain, const float* rstd, const void* dh, int64_t ld_dh, void* dx,
                                       int64_t ld_dx, float* d_gain, void* workspace, void* stream) {
    if (dtype != FP8MLP_BF16 && dtype != FP8MLP_F32) return FP8MLP_ERR_ARG;
    if (d_gain != nullptr && workspace == nullptr) return FP8MLP_ERR_ARG;
    const int bytes = dtype == FP8MLP_F32 ? 4 : 2;
    if (T < 0 || T > (int64_t(1) << 40) || d < 16 || d % 16 != 0 || d > FP8MLP_MAX_NORM_WIDTH) return FP8MLP_ERR_SHAPE;
    if (!stride_ok(T, ld_dy, d, bytes) || !stride_ok(T, ld_h, d, bytes) || !stride_ok(T, ld_dx, d, bytes)) return FP8MLP_ERR_SHAPE;
    if (dh != nullptr && !stride_ok(T, ld_dh, d, bytes)) return FP8MLP_ERR_SHAPE;
    if (T > 0 && (dy == nullptr || h == nullptr || rstd == nullptr || dx == nullptr)) return FP8MLP_ERR_ARG;
    if (dx != nullptr && dx == h) return FP8MLP_ERR_ARG;
    if (dx != nullptr && T > 1 && ((dx == dy && ld_dx != ld_dy) || (dx == dh && ld_dx != ld_dh))) return FP8MLP_ERR_ARG;      // (as above)
    if (!aligned(dy, 16) || !aligned(h, 16) || !aligned(dh, 16) || !aligned(dx, 16) || !aligned(gain, 16) || !aligned(workspace, 16))
        return FP8MLP_ERR_ALIGN;
    if (!aligned(rstd, 4) || !aligned(d_gain, 4)) return FP8MLP_ERR_ALIGN;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (T == 0) {
        if (d_gain != nullptr) FP8MLP_CUDA_CHECK(cudaMemsetAsync(d_gain, 0, sizeof(float) * d, st));
        return FP8MLP_OK;
    }
    int sms = 0;
    if (int rc = sm_count_of_current(&sms)) return rc;
    const RowShape s = row_shape(d, 32 / bytes, 512);
    NormBackArgs a{};
    a.dy = static_cast<const uint8_t*>(dy); a.h = static_cast<const uint8_t*>(h); a.dh = static_cast<const uint8_t*>(dh);
    a.dx = static_cast<uint8_t*>(dx);
    a.gain = gain; a.rstd = rstd; a.partial = d_gain != nullptr ? static_cast<float*>(workspace) : nullptr;
    a.T = T; a.ld_dy = ld_dy * bytes; a.ld_h = ld_h * bytes; a.ld_dh = ld_dh * bytes; a.ld_dx = ld_dx * bytes;
    a.inv_d = 1.0f / static_cast<float>(d); a.units = s.units; a.tpr = s.tpr; a.d = static_cast<int>(d);
    auto on32 = [&](const void* q, int64_t ld) { return aligned(q, 32) && (T <= 1 || ld % 32 == 0); };
    const bool wide = on32(dy, a.ld_dy) && on32(h, a.ld_h) && on32(dx, a.ld_dx) && (dh == nullptr || on32(dh, a.ld_dh));
    const int64_t rows = s.block / s.tpr, blocks = (T + rows - 1) / rows;
    int64_t most = static_cast<int64_t>(sms) * (512 / s.block);
    if (most > FP8MLP_RMS_PARTIALS) most = FP8MLP_RMS_PARTIALS;      // a row of the workspace per block
    bool one_cluster = d_gain != nullptr && one_cluster_does(s, blocks);
    if (one_cluster)
        if (int rc = wide_cluster_fits(&one_cluster)) return rc;
    if (one_cluster) { a.d_gain = d_gain; a.partial = nullptr; }
    const dim3 grid(static_cast<unsigned>(one_cluster ? kCluster : blocks < most ? blocks : most));
    const size_t smem = d_gain != nullptr && (s.nu > 1 || rows > 1 || one_cluster) ? sizeof(float) * d : 0;
    FP8MLP_CUDA_CHECK(FP8MLP_NORM_TYPES(FP8MLP_NORM_BACKWARD, launch_norm_backward, a, smem, grid, st));
    count_launch();
    if (d_gain != nullptr && !one_cluster) {
        FP8MLP_CUDA_CHECK(launch_chained(norm_gain_kernel, dim3(static_cast<unsigned>((d + kGainCols - 1) / kGainCols)), dim3(kGainThreads), 0, st,
                                         static_cast<const float*>(workspace), static_cast<int>(grid.x), static_cast<int>(d), d_gain));
        count_launch();
    }
    return FP8MLP_OK;
}
