// fp8.hip -- gfx950 kernels of the block-scaled FP8 matrices: quantisation
// along rows and columns, and the product of two such matrices.
#include "operators.h"

namespace pact {
namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// The same at an element's alignment: global memory is read and written in whole vectors wherever they start.
typedef u32x4 u32x4_at2 __attribute__((aligned(2)));
typedef u32x2 u32x2_at2 __attribute__((aligned(2)));
typedef v4f v4f_at4 __attribute__((aligned(4)));

__device__ __forceinline__ uint32_t bits_of(float x) { return __builtin_bit_cast(uint32_t, x); }
__device__ __forceinline__ float float_of(uint32_t x) { return __builtin_bit_cast(float, x); }

// What is finite, and NaN for what is not (0 * x is; the conversion would take an infinity to
// the largest number).  NaN has no part in a block's scale: it is never the larger of two.
__device__ __forceinline__ float finite(float x) { return __builtin_fmaf(x, 0.0f, x); }
__device__ __forceinline__ float larger(float most, float x) { return __builtin_fmaxf(most, __builtin_fabsf(x)); }

// The biased exponent b of the least scale 2^(b - 127) with which a block whose largest
// finite element has the bits `amax` stays within 448 = 1.75 * 2^8: one more than the
// element's own exponent less 8 where its significand is over 1.75.
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax) {
    const uint32_t e = (amax + 0x1fffffu) >> 23;
    return e > 8u ? e - 8u : 0u;
}

// 2^(127 - b), by which the block's elements are multiplied exactly (or to less than half
// of E4M3's smallest step).
__device__ __forceinline__ float inverse_scale(uint32_t b) { return float_of((254u - b) << 23); }

// A value that is the same in all lanes, in a scalar register (a division leaves it in a vector's).
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); }

// Four elements as E4M3 bytes, rounded to nearest even.
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}

// Largest of the 16 lanes of a DPP row.
template <int Ror>
__device__ __forceinline__ uint32_t row_ror(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x120 + Ror, 0xf, 0xf, false);
}
__device__ __forceinline__ uint32_t max_of_16_lanes(uint32_t x) {
    x = max(x, row_ror<8>(x));
    x = max(x, row_ror<4>(x));
    x = max(x, row_ror<2>(x));
    return max(x, row_ror<1>(x));
}
__device__ __forceinline__ uint32_t max_over_16_lane_groups(uint32_t x) {
    x = max(x, (uint32_t)__shfl_xor((int)x, 16));
    return max(x, (uint32_t)__shfl_xor((int)x, 32));
}

// Eight neighbouring elements of a row as they lie in memory.
template <typename T>
struct Eight;

template <>
struct Eight<uint16_t> {
    u32x4 raw = {0, 0, 0, 0};
    __device__ __forceinline__ void load(const uint16_t* p) { raw = *reinterpret_cast<const u32x4_at2*>(p); }
    __device__ __forceinline__ void set(const uint16_t (&x)[8], int64_t left) {
#pragma unroll
        for (int j = 0; j < 8; ++j) raw[j / 2] |= (j < left ? (uint32_t)x[j] : 0u) << (16 * (j & 1));
    }
    __device__ __forceinline__ float operator[](int j) const {
        return float_of(j & 1 ? raw[j / 2] & 0xffff0000u : raw[j / 2] << 16);
    }
};

template <>
struct Eight<float> {
    v4f lo = {0.0f, 0.0f, 0.0f, 0.0f}, hi = {0.0f, 0.0f, 0.0f, 0.0f};
    __device__ __forceinline__ void load(const float* p) {
        lo = *reinterpret_cast<const v4f_at4*>(p);
        hi = *reinterpret_cast<const v4f_at4*>(p + 4);
    }
    __device__ __forceinline__ void set(const float (&x)[8], int64_t left) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            lo[j] = j < left ? x[j] : 0.0f;
            hi[j] = j + 4 < left ? x[j + 4] : 0.0f;
        }
    }
    __device__ __forceinline__ float operator[](int j) const { return j < 4 ? lo[j & 3] : hi[j & 3]; }
};

// Columns col.. of the first `rows` of N rows `ld` elements apart, zero from `left` columns on and in the other rows.  All
// loads start before any is waited for: they are widened where they are used, and what a branch
// touches of a load it waits for (a row after the other: 0.7 us more for 512 x 4096).
template <int N, typename T>
__device__ __forceinline__ void load_eights(Eight<T> (&x)[N], const char* first, uint64_t ld, int64_t rows, uint64_t col,
                                            int64_t left) {
    const T* p = reinterpret_cast<const T*>(first) + col;
    if (left >= 8) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (i < rows) x[i].load(p + i * ld);
        }
    } else if (left > 0 && rows > 0) {
        T e[N][8];
#pragma unroll
        for (int i = 0; i < N; ++i) {
#pragma unroll
            for (int j = 0; j < 8; ++j) e[i][j] = p[(uint64_t)min((int64_t)i, rows - 1) * ld + min((int64_t)j, left - 1)];
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (i < rows) x[i].set(e[i], left);
        }
    }
}

// ---------------------------------------------------------------------------
// quantisation
//
// A workgroup takes a square of 128 x 128 elements, so that one reading serves
// both directions; a thread holds 4 x 8 of them. Sixteen neighbouring lanes have
// four rows of the square between them, and the 32 groups of sixteen lanes
// its columns. Along the rows a thread's bytes are written as they lie (sixteen
// lanes fill a line of 128 bytes); along the columns they go through LDS first.
//
// Large matrices are bound by memory: 32768 x 4096 in bf16, read from memory, takes 110 us both
// ways (4.9 TB/s of what is read and written, a copy's rate), 74 along the rows, 82 along the
// columns. Small ones are bound by the instructions of a thread's elements, and their loads' and exchanges'
// time: 512 x 4096 takes 3.9, 4.3 and 5.4 us, a single square 4.0. So an element is made NaN where it is not
// finite once for both directions, and then costs a maximum and a product for each. (A thread with
// 8 x 8: 117, 77 and 92 us, and two more of a small matrix.)
// ---------------------------------------------------------------------------
constexpr uint32_t kTall = 4;  // rows of a thread
static_assert(kBlockK / kTall * 16 == kQuantizeThreads, "a thread for each 4 x 8 elements");

struct Quantize {
    Plain x;
    Fp8 rows, cols;
    uint32_t tiles_c;
};

template <bool kStream>
__device__ __forceinline__ void store8(uint8_t* at, u32x2 x) {
    if constexpr (kStream) {
        __builtin_nontemporal_store(x, reinterpret_cast<u32x2*>(at));
    } else {
        *reinterpret_cast<u32x2*>(at) = x;
    }
}

// The largest of `x` in a word of LDS that began as zero.
__device__ __forceinline__ void largest(uint32_t* seen, uint32_t x) {
    __hip_atomic_fetch_max(seen, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
}

template <typename T, bool kRows, bool kCols, bool kSquare, bool kStream>
__global__ __launch_bounds__(kQuantizeThreads) void quantize_kernel(const Quantize q) {
    __shared__ __attribute__((aligned(16))) uint32_t seen[kBlockK];
    __shared__ __attribute__((aligned(8))) uint8_t turned[kCols ? kBlockK * kBlockK : 8];
    const uint32_t t = threadIdx.x, cg = t & 15, rg = t >> 4;
    const uint32_t tr = blockIdx.x / q.tiles_c, tc = blockIdx.x % q.tiles_c;
    const uint32_t r0 = tr * kBlockK + rg * kTall, c0 = tc * kBlockK + cg * 8;
    const char* base = q.x.data + (uint64_t)r0 * q.x.ld * sizeof(T);
    const int64_t left = (int64_t)q.x.cols - c0;

    Eight<T> x[kTall];
    load_eights(x, base, q.x.ld, (int64_t)q.x.rows - r0, c0, left);
    if (kSquare || kCols) {
        if (t < kBlockK) seen[t] = 0;
        __syncthreads();
    }
    float v[kTall][8];
#pragma unroll
    for (uint32_t i = 0; i < kTall; ++i) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = finite(x[i][j]);
    }
    float most_of_row[kTall] = {}, most_of_col[8] = {};
#pragma unroll
    for (uint32_t i = 0; i < kTall; ++i) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if constexpr (kSquare || kRows) most_of_row[i] = larger(most_of_row[i], v[i][j]);
            if constexpr (!kSquare && kCols) most_of_col[j] = larger(most_of_col[j], v[i][j]);
        }
    }
    uint32_t square = 0;
    if constexpr (kSquare) {
#pragma unroll
        for (uint32_t i = 0; i < kTall; ++i) square = max(square, bits_of(most_of_row[i]));
        square = max_over_16_lane_groups(max_of_16_lanes(square));
        if ((t & 63) == 0) largest(&seen[0], square);
        __syncthreads();
        square = seen[0];
    } else if constexpr (kCols) {
        uint32_t most[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) most[j] = max_over_16_lane_groups(bits_of(most_of_col[j]));
        if ((t & 48) == 0) {
#pragma unroll
            for (int j = 0; j < 8; ++j) largest(&seen[cg * 8 + j], most[j]);
        }
    }

    if constexpr (kRows) {
        // zeros behind the last block, up to a whole group of scales
        const uint32_t pad = tc + 1 == q.tiles_c ? (0u - q.tiles_c) % kScaleGroup : 0u;
#pragma unroll
        for (uint32_t i = 0; i < kTall; ++i) {
            const uint32_t b = scale_byte(kSquare ? square : max_of_16_lanes(bits_of(most_of_row[i])));
            const float inv = inverse_scale(b);
            float y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = v[i][j] * inv;
            if (r0 + i < q.x.rows) {
                const u32x2 out = {encode4(y[0], y[1], y[2], y[3]), encode4(y[4], y[5], y[6], y[7])};
                store8<kStream>(q.rows.data + (uint64_t)(r0 + i) * q.rows.ld + c0, out);
                if (cg == 0) {
                    uint8_t* s = q.rows.scale + (uint64_t)(r0 + i) * q.rows.scale_ld + tc;
                    s[0] = (uint8_t)b;
                    for (uint32_t k = 1; k <= pad; ++k) s[k] = 0;
                }
            }
        }
    }
    if constexpr (kCols) {
        const uint32_t tiles_r = (q.x.rows + kBlockK - 1) / kBlockK;
        const uint32_t pad = tr + 1 == tiles_r ? (0u - tiles_r) % kScaleGroup : 0u;
        if constexpr (!kSquare) __syncthreads();
        if (t < kBlockK && tc * kBlockK + t < q.x.cols) {
            uint8_t* const to = q.cols.scale + (uint64_t)(tc * kBlockK + t) * q.cols.scale_ld + tr;
            to[0] = (uint8_t)scale_byte(kSquare ? square : seen[t]);
            for (uint32_t k = 1; k <= pad; ++k) to[k] = 0;
        }
        const u32x4* const sizes = reinterpret_cast<const u32x4*>(seen + cg * 8);
        const u32x4 lo = sizes[0], hi = sizes[1];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t c = cg * 8 + j;
            const float inv = inverse_scale(scale_byte(kSquare ? square : j < 4 ? lo[j & 3] : hi[j & 3]));
            float y[kTall];
#pragma unroll
            for (uint32_t i = 0; i < kTall; ++i) y[i] = v[i][j] * inv;
            // eight-byte places of a column in an order that spreads sixteen lanes over the banks
            uint32_t* const to = reinterpret_cast<uint32_t*>(turned + c * kBlockK + ((rg * kTall) ^ (cg * 8)));
            *to = encode4(y[0], y[1], y[2], y[3]);
        }
        __syncthreads();
#pragma unroll
        for (uint32_t p = 0; p < kTall; ++p) {
            const uint32_t c = p * (kQuantizeThreads / 16) + rg;
            if (tc * kBlockK + c < q.x.cols) {
                const u32x2 out = *reinterpret_cast<const u32x2*>(turned + c * kBlockK + (cg ^ (c >> 3)) * 8);
                store8<kStream>(q.cols.data + (uint64_t)(tc * kBlockK + c) * q.cols.ld + tr * kBlockK + cg * 8, out);
            }
        }
    }
}

template <typename T, bool kRows, bool kCols, bool kSquare>
void quantize(const Quantize& q, uint32_t grid, hipStream_t stream) {
    // Results too large for the caches go past them: us, 32768 x 4096 in bf16, through / past: both ways, square
    // 119 / 101; rows 81 / 67; columns 93 / 77. What is smaller is wanted there by the product that follows.
    if ((uint64_t)q.x.rows * q.x.cols >= 16u << 20) {
        quantize_kernel<T, kRows, kCols, kSquare, true><<<grid, kQuantizeThreads, 0, stream>>>(q);
    } else {
        quantize_kernel<T, kRows, kCols, kSquare, false><<<grid, kQuantizeThreads, 0, stream>>>(q);
    }
}

template <typename T, bool kSquare>
void quantize(const Quantize& q, bool rows, bool cols, uint32_t grid, hipStream_t stream) {
    if (rows && cols) {
        quantize<T, true, true, kSquare>(q, grid, stream);
    } else if (rows) {
        quantize<T, true, false, kSquare>(q, grid, stream);
    } else {
        quantize<T, false, true, kSquare>(q, grid, stream);
    }
}

template <typename T>
void quantize(const Quantize& q, bool rows, bool cols, bool square, uint32_t grid, hipStream_t stream) {
    if (square) {
        quantize<T, true>(q, rows, cols, grid, stream);
    } else {
        quantize<T, false>(q, rows, cols, grid, stream);
    }
}

// ---------------------------------------------------------------------------
// bytes the other way round
//
// Squares of 128 x 128: a thread turns 8 x 8 bytes in registers, and the
// square's columns are written as whole lines by way of LDS. Bound by memory:
// 4096 x 4096 in 7.5 us (4.5 TB/s), 14336 x 4096 in 26.
// ---------------------------------------------------------------------------
typedef u32x2 u32x2_at1 __attribute__((aligned(1)));

// Bytes 0, 2 (or 1, 3) of two words between each other, then their halves.
__device__ __forceinline__ void turn4(const uint32_t (&x)[4], uint32_t (&y)[4]) {
    const uint32_t ab_lo = __builtin_amdgcn_perm(x[1], x[0], 0x05010400u), ab_hi = __builtin_amdgcn_perm(x[1], x[0], 0x07030602u);
    const uint32_t cd_lo = __builtin_amdgcn_perm(x[3], x[2], 0x05010400u), cd_hi = __builtin_amdgcn_perm(x[3], x[2], 0x07030602u);
    y[0] = __builtin_amdgcn_perm(cd_lo, ab_lo, 0x05040100u);
    y[1] = __builtin_amdgcn_perm(cd_lo, ab_lo, 0x07060302u);
    y[2] = __builtin_amdgcn_perm(cd_hi, ab_hi, 0x05040100u);
    y[3] = __builtin_amdgcn_perm(cd_hi, ab_hi, 0x07060302u);
}

__global__ __launch_bounds__(256) void transpose_kernel(const Bytes b) {
    __shared__ u32x2 turned[kBlockK * 16];
    const uint32_t t = threadIdx.x, cg = t & 15, rg = t >> 4;
    const uint32_t tiles_c = (b.cols + kBlockK - 1) / kBlockK;
    const uint32_t tr = blockIdx.x / tiles_c, tc = blockIdx.x % tiles_c;
    const uint32_t r0 = tr * kBlockK + rg * 8, c0 = tc * kBlockK + cg * 8;
    u32x2 x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = u32x2{0, 0};
    const uint8_t* from = b.in + (uint64_t)r0 * b.ld + c0;
    if (c0 < b.cols && b.cols >= 8) {
        // the last bytes of a row with those before them, which are then shifted out
        const uint32_t over = c0 + 8 <= b.cols ? 0 : c0 + 8 - b.cols;
        from -= over;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (r0 + i < b.rows) x[i] = *reinterpret_cast<const u32x2_at1*>(from + i * b.ld);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] = __builtin_bit_cast(u32x2, __builtin_bit_cast(uint64_t, x[i]) >> (8 * over));
        }
    } else {
        for (int i = 0; i < 8; ++i) {
            for (uint32_t j = 0; r0 + i < b.rows && c0 + j < b.cols; ++j) {
                x[i][j / 4] |= (uint32_t)from[i * b.ld + j] << (8 * (j % 4));
            }
        }
    }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const uint32_t up[4] = {x[0][half], x[1][half], x[2][half], x[3][half]};
        const uint32_t down[4] = {x[4][half], x[5][half], x[6][half], x[7][half]};
        uint32_t lo[4], hi[4];
        turn4(up, lo);
        turn4(down, hi);
#pragma unroll
        for (int j = 0; j < 4; ++j) turned[(cg * 8 + half * 4 + j) * 16 + (rg ^ cg)] = u32x2{lo[j], hi[j]};
    }
    __syncthreads();
#pragma unroll
    for (int p = 0; p < 8; ++p) {
        const uint32_t c = p * 16 + rg, at = tr * kBlockK + cg * 8;
        if (tc * kBlockK + c >= b.cols) continue;
        const u32x2 y = turned[c * 16 + (cg ^ (c >> 3))];
        uint8_t* out = b.out + (uint64_t)(tc * kBlockK + c) * b.out_ld + at;
        if (at + 8 <= b.rows) {
            *reinterpret_cast<u32x2_at1*>(out) = y;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (at + j < b.rows) out[j] = (uint8_t)(y[j / 4] >> (8 * (j % 4)));
            }
        }
    }
}

// ---------------------------------------------------------------------------
// product
//
// v_mfma_scale_f32_16x16x128_f8f6f4 contracts one block of 128: its scale operands
// take a byte per row and 32 elements, here the block's byte four times, so that the
// matrix unit applies both scales exactly (powers of two) before it adds to the
// binary32 sums. Its first operand takes rows of b and its second rows of a, so that
// a lane ends with four neighbouring elements of a row of C. Which 32 of a block's
// elements a lane holds makes no difference as long as it is the same for a and b.
//
// That instruction holds the sum of a block's products in fewer than 24 bits: 1.3e-5 off in the
// 2-norm at any K for normally distributed elements (the 8-bit instructions without scales
// likewise), a hundredth of what rounding to bf16 costs. Where C is binary32 the bytes are
// therefore widened to bf16 with their scale, exactly, and go through the bf16 instruction at
// half the rate, whose sums are binary32: 8e-8 off at K = 4096.  (Exactly where bf16 has the number: scale
// bytes of 3 to 246. Beside those the least bits of an element end at 2^-133, and 2^128 is infinite; the scaled
// instruction takes every scale.)
// ---------------------------------------------------------------------------
template <int Sb, int Sa>
__device__ __forceinline__ v4f mfma(v8i b, v8i a, v4f c, uint32_t scale_b, uint32_t scale_a) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, c, 0, 0, Sb, (int)scale_b, Sa, (int)scale_a);
}

// 16 bytes of a row as bf16 numbers with the scale whose exponent bits are in `scale`.
struct Wide {
    v4i lo, hi;  // eight numbers each
    __device__ __forceinline__ void set(int pair, int two) { (pair < 4 ? lo : hi)[pair & 3] = two; }
};
__device__ __forceinline__ Wide widen16(v4i x, uint32_t scale) {
    const float s = float_of(scale);
    Wide w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        w.set(2 * i, __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)x[i], s, false)));
        w.set(2 * i + 1, __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)x[i], s, true)));
    }
    return w;
}
__device__ __forceinline__ v4f mfma_wide(const Wide& b, const Wide& a, v4f c) {
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, b.lo), __builtin_bit_cast(v8bf, a.lo), c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, b.hi), __builtin_bit_cast(v8bf, a.hi), c, 0, 0, 0);
}
// One block from 32 bytes a lane of either.
template <bool kWide>
__device__ __forceinline__ v4f mfma_block(v8i b, v8i a, v4f c, uint32_t scale_b, uint32_t scale_a) {
    if constexpr (kWide) {
        const v4i b0 = __builtin_shufflevector(b, b, 0, 1, 2, 3), b1 = __builtin_shufflevector(b, b, 4, 5, 6, 7);
        const v4i a0 = __builtin_shufflevector(a, a, 0, 1, 2, 3), a1 = __builtin_shufflevector(a, a, 4, 5, 6, 7);
        c = mfma_wide(widen16(b0, scale_b << 23), widen16(a0, scale_a << 23), c);
        return mfma_wide(widen16(b1, scale_b << 23), widen16(a1, scale_a << 23), c);
    } else {
        return mfma<0, 0>(b, a, c, scale_b, scale_a);
    }
}

__device__ __forceinline__ uint16_t round_bf16(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

// Four neighbouring elements of row m of C, from column n on.
__device__ __forceinline__ void store4(const Product& p, uint32_t m, uint32_t n, v4f x) {
    const uint32_t N = p.b.rows;
    if (m >= p.a.rows || n >= N) return;
    const uint64_t at = (uint64_t)m * p.ldc + n;
    if (p.out == Out::Bf16) {
        uint16_t* c = reinterpret_cast<uint16_t*>(p.c) + at;
        uint16_t h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = round_bf16(x[i]);
        if (n + 4 <= N) {
            const u32x2 two = {h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16};
            *reinterpret_cast<u32x2_at2*>(c) = two;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (n + i < N) c[i] = h[i];
            }
        }
        return;
    }
    float* c = reinterpret_cast<float*>(p.c) + at;
    if (n + 4 <= N) {
        v4f_at4* to = reinterpret_cast<v4f_at4*>(c);
        if (p.out == Out::AddF32) {
            const v4f was = *to;
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = was[i] + x[i];
        }
        *to = x;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (n + i < N) c[i] = p.out == Out::AddF32 ? c[i] + x[i] : x[i];
        }
    }
}

// Memory from `base` on as a buffer of `bytes` bytes: a load takes a 32-bit offset of the lane's, one of
// the wave's, and checks the range.
typedef __amdgpu_buffer_rsrc_t Buffer;
__device__ __forceinline__ Buffer buffer_of(const uint8_t* base, uint64_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base), (short)0,
                                             (int)(uint32_t)(bytes < 0xffffffffu ? bytes : 0xffffffffu), 0x00020000);
}
__device__ __forceinline__ void buffer16_to_lds(Buffer from, uint32_t at, uint32_t uniform_at, void* to) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)to, 16, (int)at,
                                             (int)uniform_at, 0, 0);
}
__device__ __forceinline__ void buffer4_to_lds(Buffer from, uint32_t at, uint32_t uniform_at, void* to) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)to, 4, (int)at,
                                             (int)uniform_at, 0, 0);
}

// The places of a 128-byte row's 16-byte chunks in LDS.
__device__ __forceinline__ uint32_t swizzle(uint32_t row) { return row & 7; }

// The tile of C that is workgroup id's.
struct Place {
    uint32_t m0, n0;
};
template <int BM, int BN>
__device__ __forceinline__ Place place_of(const Product& p, uint32_t id) {
    // A workgroup's XCD is its number modulo 8: each XCD takes a run of neighbouring tiles,
    // eight tiles of rows high, so that what its workgroups read at a time fits its L2.
    const uint32_t tiles = p.tiles_m * p.tiles_n;
    Place at;
    if (tiles >= 8) {
        const uint32_t per = tiles / 8, whole = per * 8;
        if (id < whole) id = id % 8 * per + id / 8;
    }
    constexpr uint32_t kBand = 8;
    const uint32_t band = uniform(id / (kBand * p.tiles_n)), in_band = id - band * kBand * p.tiles_n;
    const uint32_t high = min(kBand, p.tiles_m - band * kBand);
    const uint32_t across = uniform(in_band / high);
    at.m0 = (band * kBand + in_band - across * high) * BM;
    at.n0 = across * BN;
    return at;
}

// A workgroup's tile of C is BM x BN, a wave's BM / WM x BN / WN of it in accumulators.  Blocks of
// a and b come into LDS by direct loads, kDeep buffers deep, and four blocks' scales a row at a time.
// (Behind the last block the last one is loaded again and not used: loops without branches.)  Two buffers
// leave a load about a block's time to arrive: enough where two workgroups share a CU or the tile is large.
// Where a CU has one tile of 128 x 128, which is done with a block in a third of the time that memory takes,
// four buffers: 1024 x 4096 x 4096 in 24 us for 34 (1440 and 1020 TFLOP/s; binary32 result 38 and 49).
// The large tile's two buffers fill the LDS, and what bounds it is a load's time to arrive: there the rows of b, which
// are all in registers early in a block, make room for the next block but one's long before those of a do (kApart).
template <int BM, int BN, int WM, int WN, int kDeep>
struct Stage {
    static constexpr int kThreads = WM * WN * 64;
    static constexpr int kFM = BM / WM / 16, kFN = BN / WN / 16;
    static constexpr int kRows = BM + BN, kTileM = BM;
    static constexpr bool kApart = BM == 256;  // a thread's loads of a and of b start at times of their own
    static constexpr int kLoads = kRows * 8 / kThreads;
    static constexpr int kScaleLoads = (kRows + kThreads - 1) / kThreads;
    // (a whole power of two: BN is BM, or half of it with as much left free)
    static constexpr uint32_t kTileBytes = 2 * BM * kBlockK, kScaleBytes = kRows * 4;
    static constexpr uint32_t kLdsBytes = kDeep * kTileBytes + 2 * kScaleBytes;
    static_assert((kTileBytes & (kTileBytes - 1)) == 0 && (kDeep & (kDeep - 1)) == 0, "a buffer is some bits of an address");
    static_assert(BN <= BM && kRows % 64 == 0 && BM % 64 == 0 && BM % (kThreads / 8) == 0 && kRows % (kThreads / 8) == 0,
                  "a load's rows are of one matrix");
    static_assert(!kApart || BM == BN, "half of the loads are of each matrix");

    uint8_t* lds;
    Buffer buf_a, buf_b, buf_sa, buf_sb;  // from the tile's first row on
    uint32_t from[kLoads], scale_from[kScaleLoads];  // offsets of this thread's loads
    uint32_t wave;
    uint32_t at0, at1;        // where the two halves of a lane's fragments start in the buffer in use,
    uint32_t rows_a, rows_b;  // counted from the wave's first rows of a and of b
    uint32_t at_sa, at_sb;
    uint32_t sa[kFM], sb[kFN], next_sa[kFM], next_sb[kFN];
    v4f acc[kFM][kFN];

    __device__ __forceinline__ void set_up(const Product& p, const Place& at, uint8_t* shared) {
        lds = shared;
        const uint32_t tid = threadIdx.x, lane = tid & 63, row = lane & 15, g = lane >> 4;
        wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        buf_a = buffer_of(p.a.data + (uint64_t)at.m0 * p.a.ld, (uint64_t)(p.a.rows - at.m0) * p.a.ld);
        buf_b = buffer_of(p.b.data + (uint64_t)at.n0 * p.b.ld, (uint64_t)(p.b.rows - at.n0) * p.b.ld);
        buf_sa = buffer_of(p.a.scale + (uint64_t)at.m0 * p.a.scale_ld, (uint64_t)(p.a.rows - at.m0) * p.a.scale_ld);
        buf_sb = buffer_of(p.b.scale + (uint64_t)at.n0 * p.b.scale_ld, (uint64_t)(p.b.rows - at.n0) * p.b.scale_ld);
        // rows behind the last are read as the last one; what comes of them is not stored
        const uint32_t last_a = p.a.rows - 1 - at.m0, last_b = p.b.rows - 1 - at.n0;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const uint32_t r = i * (kThreads / 8) + tid / 8;
            from[i] = (r < BM ? min(r, last_a) * p.a.ld : min(r - BM, last_b) * p.b.ld) + ((tid & 7) ^ swizzle(r)) * 16;
        }
#pragma unroll
        for (int i = 0; i < kScaleLoads; ++i) {
            const uint32_t r = i * kThreads + tid;
            scale_from[i] = r < BM ? min(r, last_a) * p.a.scale_ld : min(r - BM, last_b) * p.b.scale_ld;
        }
        rows_a = wave / WN * (BM / WM);
        rows_b = BM + wave % WN * (BN / WN);
        at0 = row * kBlockK + (g ^ swizzle(row)) * 16;
        at1 = row * kBlockK + ((g + 4) ^ swizzle(row)) * 16;
        at_sa = (rows_a + row) * 4;
        at_sb = (rows_b + row) * 4;
#pragma unroll
        for (int i = 0; i < kFM; ++i) {
#pragma unroll
            for (int j = 0; j < kFN; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        }
    }

    // The i-th of a thread's loads of a block.
    __device__ __forceinline__ void load(int i, uint32_t block, uint32_t buffer) {
        buffer16_to_lds(i * (kThreads / 8) < BM ? buf_a : buf_b, from[i], block * kBlockK,
                        lds + buffer % kDeep * kTileBytes + wave * 1024 + i * kThreads * 16);
    }
    __device__ __forceinline__ void load_scales(uint32_t group) {
#pragma unroll
        for (int i = 0; i < kScaleLoads; ++i) {
            if (i * kThreads + wave * 64 >= (uint32_t)kRows) break;  // (waves behind the last row)
            buffer4_to_lds(i * kThreads + wave * 64 < BM ? buf_sa : buf_sb, scale_from[i], group * kScaleGroup,
                           lds + kDeep * kTileBytes + (group & 1) * kScaleBytes + wave * 256 + i * kThreads * 4);
        }
    }
    // In block kb, before anything else: the scales of a group that is read from the block after the next three
    // on; by then they are there, however few loads are waited for.  (A branch further down would have
    // matrix instructions sunk behind it.)
    __device__ __forceinline__ void load_next_scales(uint32_t kb, uint32_t blocks) {
        if ((kb + 5) % kScaleGroup == 0 && kb + 5 < blocks) load_scales((kb + 5) / kScaleGroup);
    }
    // What is loaded before the first block: all buffers but the last.
    __device__ __forceinline__ void load_first(uint32_t blocks) {
        load_scales(0);
        if (blocks > kScaleGroup) load_scales(1);
#pragma unroll
        for (uint32_t b = 0; b + 1 < kDeep; ++b) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) load(i, uniform(min(b, blocks - 1)), b);
        }
    }
    // All waves meet, each with its LDS reads done and at most `under_way` of its vector loads, which end in their
    // order, not.  (A fence would wait for every one.)
    template <int under_way>
    static __device__ __forceinline__ void meet() {
        static_assert(under_way < 64, "what the instruction counts to");
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0070 | (under_way & 15) | (under_way >> 4) << 14);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    }
    // The scales of a block, with the others of its group.
    __device__ __forceinline__ void read_scales_a(uint32_t block) {
        const uint8_t* from = lds + kDeep * kTileBytes + (block / kScaleGroup & 1) * kScaleBytes;
#pragma unroll
        for (int i = 0; i < kFM; ++i) next_sa[i] = *reinterpret_cast<const uint32_t*>(from + at_sa + i * 64);
    }
    __device__ __forceinline__ void read_scales_b(uint32_t block) {
        const uint8_t* from = lds + kDeep * kTileBytes + (block / kScaleGroup & 1) * kScaleBytes;
#pragma unroll
        for (int j = 0; j < kFN; ++j) next_sb[j] = *reinterpret_cast<const uint32_t*>(from + at_sb + j * 64);
    }
    // The fragments that are read from here on are those of a block `blocks` further.
    __device__ __forceinline__ void next_buffer(uint32_t blocks = 1) {
        if constexpr (kDeep == 2) {
            at0 ^= kTileBytes;
            at1 ^= kTileBytes;
        } else {
            at0 = (at0 + blocks * kTileBytes) & (kDeep * kTileBytes - 1);
            at1 = (at1 + blocks * kTileBytes) & (kDeep * kTileBytes - 1);
        }
    }
    __device__ __forceinline__ v4i half0(uint32_t row) const {
        return *reinterpret_cast<const v4i*>(lds + at0 + row * kBlockK);
    }
    __device__ __forceinline__ v4i half1(uint32_t row) const {
        return *reinterpret_cast<const v4i*>(lds + at1 + row * kBlockK);
    }
};

// The product with the 8-bit instruction.  A block is used in rounds, one for each 16 of the wave's
// rows of a; the fragments of a round are read one round ahead.  Before the last round every wave
// has read all of its buffer: there the waves meet, the load of the next block but one starts
// into that buffer, and the next block's first fragments are read behind the round's instructions.
//
// Bound by the matrix unit at the clock that power leaves it (1.8 GHz; it is busy in two thirds of the cycles), and by
// the time that a block's loads take to arrive: 8192 x 14336 x 4096 in 393 us (2450 TFLOP/s), 8192 x 8192 x 8192 in 386
// (2850), 512 x 32768 x 4096 in 57; 401, 416 and 62 with one time for the loads of a and b, half of them in the last
// round and half in the next first one. Three quarters of a's rows behind the second meeting as well: 8% slower, for all
// loads then start at once; loads spread over all rounds: no difference. The instruction of 32 x 32 x 64: 11%
// slower, on whole blocks as on halves, four of them under way. Waves of 2 x 2, 2 x 4 or 4 x 2: within 3%.
// Scales that are loaded a block at a time instead of four: 480 us for 398.
// (With kDeep buffers: the next block but kDeep - 1.)  With kApart the waves meet once more, when a round has used all
// rows of b, and the load of the next block but one's rows of b starts there, that of a's before the last round.
template <int BM, int BN, int WM, int WN, int kDeep>
struct Tiled : Stage<BM, BN, WM, WN, kDeep> {
    using St = Stage<BM, BN, WM, WN, kDeep>;
    using St::kFM, St::kFN, St::kLoads, St::kApart;
    using St::load, St::acc, St::sa, St::sb, St::next_sa, St::next_sb, St::rows_a, St::rows_b;
    v8i a[2], b[kFN];

    __device__ __forceinline__ v8i fragment(uint32_t row) const {
        return __builtin_shufflevector(this->half0(row), this->half1(row), 0, 1, 2, 3, 4, 5, 6, 7);
    }
    __device__ __forceinline__ void read_a(int i) { a[i & 1] = fragment(rows_a + i * 16); }
    __device__ __forceinline__ void read_b(int j) { b[j] = fragment(rows_b + j * 16); }

    // What is done behind matrix instruction (i, j) of block kb, a little at a time: the matrix unit
    // takes 32 cycles for each.
    __device__ __forceinline__ void beside(int i, int j, uint32_t kb, uint32_t blocks) {
        constexpr int kLast = kFM - 1, kHalf = kLoads / 2, kPer = (kHalf + kFN - 1) / kFN;
        const uint32_t one = uniform(min(kb + kDeep - 1, blocks - 1)), two = uniform(min(kb + kDeep, blocks - 1));
        const uint32_t shift = (kb + 1) % kScaleGroup * 8;
        if (i < kLast && j == 0) read_a(i + 1);
        if (i == (kApart ? 1 : 0)) {
#pragma unroll
            for (int k = j * kPer; k < (j + 1) * kPer && k < kHalf; ++k) {
                load(kHalf + k, kApart ? two : one, kApart ? kb : kb + kDeep - 1);
            }
        }
        if (i == 1 && j == 1) this->read_scales_a(kb + 1);
        if (i == 1 && j == (kFN > 2 ? 2 : 1)) this->read_scales_b(kb + 1);
        if (i >= 2 && j == 1) {
            if (i == 2) sa[0] = next_sa[0] >> shift;
            sa[i - 1] = next_sa[i - 1] >> shift;
        }
        if (i == kLast) {
            if (j == 0) read_a(0);
            read_b(j);
#pragma unroll
            for (int k = j * kPer; k < (j + 1) * kPer && k < kHalf; ++k) load(k, two, kb);
            sb[j] = next_sb[j] >> shift;
            if (j == kFN - 1) sa[kLast] = next_sa[kLast] >> shift;
        }
    }

    __device__ __forceinline__ void run(uint32_t blocks) {
        static_assert(kFM % 2 == 0, "a block's first rows take the place of the last but one's of the block before");
        static_assert(kFM >= 4 && kFN >= 2, "a place beside for everything");
        if (blocks == 0) return;
        this->load_first(blocks);
        constexpr int kMore = kApart ? kLoads : kLoads / 2;  // loads of the block behind those
#pragma unroll
        for (int i = 0; i < kMore; ++i) load(i, uniform(min(kDeep - 1u, blocks - 1)), kDeep - 1);
        St::template meet<(kDeep - 2) * kLoads + kMore>();
        read_a(0);
#pragma unroll
        for (int j = 0; j < kFN; ++j) read_b(j);
        this->read_scales_a(0);
        this->read_scales_b(0);
#pragma unroll
        for (int i = 0; i < kFM; ++i) sa[i] = next_sa[i];
#pragma unroll
        for (int j = 0; j < kFN; ++j) sb[j] = next_sb[j];
#pragma unroll 1
        for (uint32_t kb = 0; kb < blocks; ++kb) {
            this->load_next_scales(kb, blocks);
#pragma unroll
            for (int i = 0; i < kFM; ++i) {
                if (kApart && i == 1) St::template meet<63>();  // all rows of b have been read
                if (i == kFM - 1) {
                    // the next block is there
                    St::template meet<(kDeep - 2) * kLoads + (kApart ? kLoads / 2 : 0)>();
                    this->next_buffer();
                }
#pragma unroll
                for (int j = 0; j < kFN; ++j) {
                    __builtin_amdgcn_sched_barrier(0);
                    acc[i][j] = mfma<0, 0>(b[j], a[i & 1], acc[i][j], sb[j], sa[i]);
                    __builtin_amdgcn_sched_barrier(0);
                    beside(i, j, kb, blocks);
                }
            }
        }
    }
};

// The product with the bf16 instruction: the same bytes in LDS, widened in registers, half a block at a
// time.  In each round (16 rows of a, half a block) a slot of two matrix instructions, 32 cycles,
// goes with each 16 rows of b; beside it run a part of the widening of the next round's
// rows of a, which were read a round before, and a part of that of the other half's rows of b.
// The next block's bytes are there from the second half on, and the buffer in use is free at its end (of b's rows
// from the second half on: with kApart their loads start there).
//
// Bound by the matrix unit, whose bf16 rate is half the 8-bit one: 8192 x 14336 x 4096 in 644 us
// (1490 TFLOP/s; 670 with a's and b's loads at one time), 4096 x 4096 x 4096 in 94. A wave has 128 x 128 of the larger tile, so that a widened
// fragment serves eight products and the conversions fit beside the matrix instructions.
template <int BM, int BN, int WM, int WN, int kDeep>
struct TiledWide : Stage<BM, BN, WM, WN, kDeep> {
    using St = Stage<BM, BN, WM, WN, kDeep>;
    using St::kFM, St::kFN, St::kLoads, St::kApart;
    using St::load, St::acc, St::sa, St::sb, St::next_sa, St::next_sb, St::rows_a, St::rows_b;
    static constexpr int kParts = 8 / kFN;  // pairs of elements of 16 bytes that a slot widens
    static_assert(kFM == kFN && (kFN == 4 || kFN == 8), "a round of a widens a fragment of b");

    Wide a[2], b[2][kFN];
    v4i raw_a[2], raw_b[3];

    // Round r of a block's 2 * kFM; the next block's follow.
    __device__ __forceinline__ void read_a(int r) {
        const uint32_t row = rows_a + r % kFM * 16;
        raw_a[r & 1] = r / kFM & 1 ? this->half1(row) : this->half0(row);
    }
    __device__ __forceinline__ void read_b(int half, int j, int to) {
        raw_b[to] = half ? this->half1(rows_b + j * 16) : this->half0(rows_b + j * 16);
    }
    static __device__ __forceinline__ void widen(Wide& to, v4i from, int part, uint32_t scale) {
        const uint32_t w = (uint32_t)from[part >> 1];
        const v2bf two = part & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, float_of(scale), true)
                                  : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, float_of(scale), false);
        to.set(part, __builtin_bit_cast(int, two));
    }

    template <int H>
    __device__ __forceinline__ void half(uint32_t kb, uint32_t blocks) {
        // with kApart the first half starts a's loads of a block and the second b's of the one behind it
        constexpr int kCount = kApart ? kLoads / 2 : H == 0 ? kLoads : 0, kPer = (kCount + kFN - 1) / kFN;
        const uint32_t ahead = uniform(min(kb + kDeep - 1 + H, blocks - 1));
        const uint32_t shift = (kb + 1) % kScaleGroup * 8;
#pragma unroll
        for (int i = 0; i < kFM; ++i) {
#pragma unroll
            for (int j = 0; j < kFN; ++j) {
                const int r = H * kFM + i;
                __builtin_amdgcn_sched_barrier(0);
                acc[i][j] = mfma_wide(b[H][j], a[r & 1], acc[i][j]);
                __builtin_amdgcn_sched_barrier(0);
                if (i == 0) {
#pragma unroll
                    for (int k = j * kPer; k < (j + 1) * kPer && k < kCount; ++k) load(H * kCount + k, ahead, kb + kDeep - 1 + H);
                }
                // the rows of a of the round after the next one; the next block's are in the other buffer
                if (j == 0) {
                    if (r + 2 >= 2 * kFM) this->next_buffer();
                    read_a((r + 2) % (2 * kFM));
                    if (r + 2 >= 2 * kFM) this->next_buffer(kDeep - 1);
                }
                // the rows of b of the other half (the second half: of the next block)
                if (j == 1 && i < kFM - 1) {
                    if (H == 1) this->next_buffer();
                    read_b(H ^ 1, i, i & 1);
                    if (i == kFM - 2) read_b(H ^ 1, kFM - 1, 2);
                    if (H == 1) this->next_buffer(kDeep - 1);
                }
                if (H == 0 && i == 1 && j == 2) this->read_scales_a(kb + 1);
                if (H == 0 && i == 2 && j == 2) this->read_scales_b(kb + 1);
                // scales of the next block as soon as the block's own has been used
                if (H == 1 && i == 0) sb[j] = exponent(next_sb[j] >> shift);
                if (H == 1 && i >= 1 && j == 0) sa[i - 1] = exponent(next_sa[i - 1] >> shift);
#pragma unroll
                for (int k = j * kParts; k < (j + 1) * kParts; ++k) {
                    widen(a[(r + 1) & 1], raw_a[(r + 1) & 1], k, sa[(i + 1) % kFM]);
                    if (i >= 1) widen(b[H ^ 1][i - 1], raw_b[(i - 1) & 1], k, sb[i - 1]);
                    if (i == kFM - 1) widen(b[H ^ 1][i], raw_b[2], k, sb[i]);
                }
                if (H == 1 && i == kFM - 1 && j == kFN - 1) sa[i] = exponent(next_sa[i] >> shift);
            }
        }
    }
    static __device__ __forceinline__ uint32_t exponent(uint32_t scale) { return (scale & 0xffu) << 23; }

    __device__ __forceinline__ void run(uint32_t blocks) {
        if (blocks == 0) return;
        this->load_first(blocks);
        constexpr int kMore = kApart ? kLoads / 2 : 0;  // b's loads of the block behind those
#pragma unroll
        for (int i = kLoads - kMore; i < kLoads; ++i) load(i, uniform(min(kDeep - 1u, blocks - 1)), kDeep - 1);
        St::template meet<(kDeep - 2) * kLoads + kMore>();
        this->read_scales_a(0);
        this->read_scales_b(0);
#pragma unroll
        for (int i = 0; i < kFM; ++i) sa[i] = exponent(next_sa[i]);
#pragma unroll
        for (int j = 0; j < kFN; ++j) sb[j] = exponent(next_sb[j]);
        read_a(0);
#pragma unroll
        for (int k = 0; k < 8; ++k) widen(a[0], raw_a[0], k, sa[0]);
        read_a(1);
#pragma unroll
        for (int j = 0; j < kFN; ++j) {
            read_b(0, j, 0);
#pragma unroll
            for (int k = 0; k < 8; ++k) widen(b[0][j], raw_b[0], k, sb[j]);
        }
#pragma unroll 1
        for (uint32_t kb = 0; kb < blocks; ++kb) {
            this->load_next_scales(kb, blocks);
            half<0>(kb, blocks);
            St::template meet<(kDeep - 2) * kLoads>();  // the next block is there
            half<1>(kb, blocks);
            St::template meet<63>();  // the block's buffer has been read
            this->next_buffer();
        }
    }
};

// What the lanes of a wave have stored in LDS and what they read of each other's from here on, in that order (no
// instruction: LDS serves a wave's in turn, the compiler has to keep them so).
__device__ __forceinline__ void lanes_meet() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
}

// LDS of a wave for what follows: 16 rows of its tile, a little more than their elements apart.
template <int kFN>
constexpr uint32_t kRowRoom = kFN * 64 + 16;

// A wave's accumulators into C, rows m.. and columns n.. of it, 16 rows at a time by way of LDS of the
// wave's own: neighbouring lanes hold neighbouring rows, and a store of theirs would touch a line for
// each lane; from LDS they take 16 bytes next to each other.
template <int kFM, int kFN>
__device__ __forceinline__ void store_wave(const Product& p, uint32_t m, uint32_t n, const v4f (&acc)[kFM][kFN],
                                           uint8_t* room) {
    const uint32_t lane = threadIdx.x & 63, row = lane & 15, g = lane >> 4;
    const bool whole = m + kFM * 16 <= p.a.rows && n + kFN * 16 <= p.b.rows;
    const bool half = whole && p.out == Out::Bf16;
    // lanes of a row, and the rows of a store
    constexpr uint32_t kLanes16 = kFN * 2, kLanes32 = kFN * 4;
    const uint32_t shift = half ? 1 : 2, lanes = half ? kLanes16 : kLanes32;
    const uint32_t r = lane / lanes, at = lane % lanes * 16;
    char* to = p.c + (((uint64_t)(m + r) * p.ldc + n) << shift) + at;
    const uint64_t ld = p.ldc << shift;
#pragma unroll
    for (int i = 0; i < kFM; ++i) {
        uint8_t* const in = room + row * kRowRoom<kFN>;
#pragma unroll
        for (int j = 0; j < kFN; ++j) {
            if (half) {
                const v4f x = acc[i][j];
                *reinterpret_cast<u32x2*>(in + j * 32 + g * 8) =
                    u32x2{round_bf16(x[0]) | (uint32_t)round_bf16(x[1]) << 16,
                          round_bf16(x[2]) | (uint32_t)round_bf16(x[3]) << 16};
            } else {
                *reinterpret_cast<v4f*>(in + j * 64 + g * 16) = acc[i][j];
            }
        }
        lanes_meet();
        if (half) {
#pragma unroll
            for (uint32_t q = 0; q < kLanes16 / 4; ++q) {
                const u32x4 x = *reinterpret_cast<const u32x4*>(room + (q * (64 / kLanes16) + r) * kRowRoom<kFN> + at);
                *reinterpret_cast<u32x4_at2*>(to + (i * 16 + q * (64 / kLanes16)) * ld) = x;
            }
        } else if (whole) {
#pragma unroll
            for (uint32_t q = 0; q < kLanes32 / 4; ++q) {
                v4f x = *reinterpret_cast<const v4f*>(room + (q * (64 / kLanes32) + r) * kRowRoom<kFN> + at);
                v4f_at4* const c = reinterpret_cast<v4f_at4*>(to + (i * 16 + q * (64 / kLanes32)) * ld);
                if (p.out == Out::AddF32) {
                    const v4f was = *c;
#pragma unroll
                    for (int k = 0; k < 4; ++k) x[k] = was[k] + x[k];
                }
                *c = x;
            }
        } else {
#pragma unroll 1
            for (uint32_t c = lane; c < 16 * kLanes32; c += 64) {
                const uint32_t k = c / kLanes32, q = c % kLanes32;
                store4(p, m + i * 16 + k, n + q * 4, *reinterpret_cast<const v4f*>(room + k * kRowRoom<kFN> + q * 16));
            }
        }
        lanes_meet();
    }
}

template <typename Tl>
__device__ __forceinline__ void product_tile(const Product& p, const Place& at, uint8_t* lds) {
    Tl t;
    t.set_up(p, at, lds);
    static_assert(Tl::kThreads / 64 * 16 * kRowRoom<Tl::kFN> <= Tl::kLdsBytes, "a store's rows fit the loads' LDS");
    t.run(p.kblocks);
    Tl::template meet<0>();  // no load into LDS is under way, and no wave reads it
    store_wave(p, at.m0 + t.rows_a, at.n0 + t.rows_b - Tl::kTileM, t.acc,
               lds + t.wave * (16 * kRowRoom<Tl::kFN>));
}

// The workgroup's tile; with four buffers, of its part of K.
template <typename Tl, int BM, int BN, int kDeep>
__device__ __forceinline__ void product_part(Product p, uint8_t* lds) {
    uint32_t id = blockIdx.x;
    if constexpr (kDeep == 4) {
        if (p.part_blocks != 0) {
            const uint32_t tiles = p.tiles_m * p.tiles_n, part = uniform(id / tiles), first = part * p.part_blocks;
            id -= part * tiles;
            p.a.data += first * kBlockK;
            p.b.data += first * kBlockK;
            p.a.scale += first;
            p.b.scale += first;
            p.kblocks = min(p.part_blocks, p.kblocks - first);
            p.c = reinterpret_cast<char*>(p.sums + (uint64_t)part * p.a.rows * p.ld_sums);
            p.ldc = p.ld_sums;
            p.out = Out::F32;
        }
    }
    product_tile<Tl>(p, place_of<BM, BN>(p, id), lds);
}

template <int BM, int BN, int WM, int WN, int kDeep>
__global__ __launch_bounds__(WM* WN * 64, 1) void product_kernel(const Product p) {
    using Tl = Tiled<BM, BN, WM, WN, kDeep>;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[Tl::kLdsBytes];
    product_part<Tl, BM, BN, kDeep>(p, lds);
}

template <int BM, int BN, int WM, int WN, int kDeep>
__global__ __launch_bounds__(WM* WN * 64, 1) void wide_product_kernel(const Product p) {
    using Tl = TiledWide<BM, BN, WM, WN, kDeep>;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[Tl::kLdsBytes];
    product_part<Tl, BM, BN, kDeep>(p, lds);
}

// C from the sums of the parts of K, added in their order.
__global__ __launch_bounds__(256) void join_kernel(const Product p, uint32_t parts) {
    const uint32_t fours = p.ld_sums / 4;
    const uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (uint64_t)p.a.rows * fours) return;
    const uint32_t m = (uint32_t)(i / fours), n = (uint32_t)(i - (uint64_t)m * fours) * 4;
    const float* from = p.sums + (uint64_t)m * p.ld_sums + n;
    v4f x = *reinterpret_cast<const v4f*>(from);
#pragma unroll 4
    for (uint32_t s = 1; s < parts; ++s) {
        const v4f y = *reinterpret_cast<const v4f*>(from + (uint64_t)s * p.a.rows * p.ld_sums);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = x[e] + y[e];
    }
    store4(p, m, n, x);
}

// ---------------------------------------------------------------------------
// products whose tiles are too few to fill the GPU
//
// Here the waves of a workgroup share a small tile of C and have the blocks of K between them. A wave
// loads whole lines (eight lanes a row) into registers, one block ahead, and turns them into
// fragments in LDS of its own, so that it waits for nobody until the sums of all waves are
// added, in the order of the waves.  (Fragments loaded as they are used would be 16 rows a load, a
// line for each lane.)  Bound by the time that a block takes from memory, of which each wave has one under way:
// 32 x 4096 x 4096 in 8.5 us, 64 rows 9.2, 256 rows 15, weights read from memory.
// ---------------------------------------------------------------------------

// The blocks of K of one of `waves` waves: runs of up to four neighbours, whose scales are one load
// where there are enough of them to go round.
struct Runs {
    uint32_t run, stride, at, left;  // at: the block in use; left: blocks of its run behind it
    bool words;
    __device__ __forceinline__ Runs(uint32_t blocks, uint32_t waves, uint32_t wave) {
        words = blocks >= waves * kScaleGroup;
        run = words ? kScaleGroup : uniform(max((blocks + waves - 1) / waves, 1u));  // (of no blocks too)
        stride = run * (waves - 1) + 1;
        at = wave * run;
        left = run - 1;
    }
    __device__ __forceinline__ void next() {
        const bool over = left == 0;
        at += over ? stride : 1;
        left = over ? run - 1 : left - 1;
    }
    // the first block of a run
    __device__ __forceinline__ bool fresh() const { return left == run - 1; }
};

// Rows of a matrix in FP8 as a lane loads them: two rows (eight apart) of each of `kTiles` groups of 16.
template <int kTiles>
struct Lines {
    Buffer data, scale;
    uint32_t from[kTiles][2], scale_from[kTiles];

    __device__ __forceinline__ void set_up(const Fp8& x, uint32_t first) {
        const uint32_t lane = threadIdx.x & 63, last = x.rows - 1 - first;
        data = buffer_of(x.data + (uint64_t)first * x.ld, (uint64_t)(x.rows - first) * x.ld);
        scale = buffer_of(x.scale + (uint64_t)first * x.scale_ld, (uint64_t)(x.rows - first) * x.scale_ld);
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                from[t][q] = min((uint32_t)(t * 16 + q * 8) + lane / 8, last) * x.ld + (lane & 7) * 16;
            }
            scale_from[t] = min(t * 16 + (lane & 15), last) * x.scale_ld;
        }
    }
    __device__ __forceinline__ void load(uint32_t block, v4i (&to)[kTiles][2]) const {
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                to[t][q] = __builtin_bit_cast(
                    v4i, __builtin_amdgcn_raw_buffer_load_b128(data, (int)from[t][q], (int)(block * kBlockK), 0));
            }
        }
    }
    // The scales of a run's blocks, the first in the lowest byte.
    __device__ __forceinline__ void load_scales(const Runs& k, uint32_t blocks, uint32_t (&to)[kTiles]) const {
        if (k.words) {
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                to[t] = __builtin_amdgcn_raw_buffer_load_b32(scale, (int)scale_from[t], (int)k.at, 0);
            }
            return;
        }
#pragma unroll
        for (int t = 0; t < kTiles; ++t) to[t] = 0;
        for (uint32_t u = 0; u < k.run && k.at + u < blocks; ++u) {
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                to[t] |= (uint32_t)__builtin_amdgcn_raw_buffer_load_b8(scale, (int)scale_from[t], (int)(k.at + u), 0)
                         << (8 * u);
            }
        }
    }
};

// 16 rows of a block between a wave's lines and its fragments, by way of 2 KB of LDS.
struct Turn {
    uint32_t in0, in1, out0, out1;
    __device__ __forceinline__ Turn() {
        const uint32_t lane = threadIdx.x & 63, line = lane / 8, row = lane & 15, g = lane >> 4;
        in0 = line * kBlockK + ((lane & 7) ^ swizzle(line)) * 16;
        in1 = in0 + 8 * kBlockK;
        out0 = row * kBlockK + (g ^ swizzle(row)) * 16;
        out1 = row * kBlockK + ((g + 4) ^ swizzle(row)) * 16;
    }
    __device__ __forceinline__ void put(uint8_t* room, const v4i (&lines)[2]) const {
        *reinterpret_cast<v4i*>(room + in0) = lines[0];
        *reinterpret_cast<v4i*>(room + in1) = lines[1];
    }
    __device__ __forceinline__ v8i get(const uint8_t* room) const {
        return __builtin_shufflevector(*reinterpret_cast<const v4i*>(room + out0),
                                       *reinterpret_cast<const v4i*>(room + out1), 0, 1, 2, 3, 4, 5, 6, 7);
    }
};

template <int MT, int NT, int kWaves, bool kWide>
__global__ __launch_bounds__(kWaves * 64, 2) void shared_tile_kernel(const Product p) {
    constexpr uint32_t kRoom = (MT + NT) * 2048, kSums = MT * NT * 64;
    constexpr uint32_t kBytes = kWaves * (kRoom > kSums * 16 ? kRoom : kSums * 16);
    __shared__ __attribute__((aligned(1024))) uint8_t lds[kBytes];
    const uint32_t lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const Place at = place_of<MT * 16, NT * 16>(p, blockIdx.x);
    Lines<MT> a;
    Lines<NT> b;
    a.set_up(p.a, at.m0);
    b.set_up(p.b, at.n0);
    const Turn turn;
    uint8_t* room = lds + wave * kRoom;
    v4f acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    }
    Runs k(p.kblocks, kWaves, wave);
    v4i line_a[MT][2], line_b[NT][2];
    uint32_t next_sa[MT], next_sb[NT], sa[MT], sb[NT];
    if (k.at < p.kblocks) {
        b.load(k.at, line_b);
        a.load(k.at, line_a);
        b.load_scales(k, p.kblocks, next_sb);
        a.load_scales(k, p.kblocks, next_sa);
    }
    while (k.at < p.kblocks) {
#pragma unroll
        for (int j = 0; j < NT; ++j) turn.put(room + j * 2048, line_b[j]);
#pragma unroll
        for (int i = 0; i < MT; ++i) turn.put(room + (NT + i) * 2048, line_a[i]);
        const bool fresh = k.fresh();
#pragma unroll
        for (int i = 0; i < MT; ++i) sa[i] = fresh ? next_sa[i] : sa[i] >> 8;
#pragma unroll
        for (int j = 0; j < NT; ++j) sb[j] = fresh ? next_sb[j] : sb[j] >> 8;
        k.next();
        if (k.at < p.kblocks) {
            b.load(k.at, line_b);
            a.load(k.at, line_a);
            if (k.fresh()) {
                b.load_scales(k, p.kblocks, next_sb);
                a.load_scales(k, p.kblocks, next_sa);
            }
        }
        lanes_meet();
        v8i y[NT];
#pragma unroll
        for (int j = 0; j < NT; ++j) y[j] = turn.get(room + j * 2048);
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const v8i x = turn.get(room + (NT + i) * 2048);
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                acc[i][j] = mfma_block<kWide>(y[j], x, acc[i][j], kWide ? sb[j] & 0xffu : sb[j], kWide ? sa[i] & 0xffu : sa[i]);
            }
        }
        lanes_meet();
    }
    __syncthreads();
    v4f* sums = reinterpret_cast<v4f*>(lds);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
#pragma unroll
        for (int j = 0; j < NT; ++j) sums[(wave * MT * NT + i * NT + j) * 64 + lane] = acc[i][j];
    }
    __syncthreads();
    for (uint32_t f = wave; f < MT * NT; f += kWaves) {
        v4f x = sums[f * 64 + lane];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) {
            const v4f y = sums[(w * MT * NT + f) * 64 + lane];
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = x[i] + y[i];
        }
        store4(p, at.m0 + f / NT * 16 + (lane & 15), at.n0 + f % NT * 16 + (lane >> 4) * 4, x);
    }
}

// The product of up to 16 rows of binary32 or bf16 elements. Every workgroup quantises them for itself, into
// LDS, while its first lines of b are on their way, and then takes one 16 rows of b after the
// other, the lines of the next four blocks always under way.  Bound by the reading of b: one row, 32768 x 4096
// in 22 us (6.1 TB/s), 14336 x 4096 in 11, 4096 x 4096 in 5.4 (7.3 out of memory), where a quantisation
// of its own and the product would take 2.3 and 4.2.
constexpr int kFewWaves = 8;

// LDS of the rows of a (blocks, then scales), of the waves' fragments of b and of two sets of sums.
constexpr uint32_t few_rows_lds(uint32_t rows, uint32_t blocks) {
    return (rows * blocks * (kBlockK + 1) + 1023) / 1024 * 1024 + kFewWaves * (2048 + 2 * 1024);
}

template <typename T, bool kWide>
__global__ __launch_bounds__(kFewWaves * 64) void few_rows_kernel(const Plain x, const Product p) {
    extern __shared__ __attribute__((aligned(1024))) uint8_t few_lds[];
    constexpr int kAhead = kScaleGroup;
    const uint32_t lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const uint32_t rows = x.rows, blocks = p.kblocks;
    uint8_t* const held = few_lds;                          // block k, row m: 128 bytes at (k * rows + m) * 128
    uint8_t* const held_scale = held + rows * blocks * kBlockK;  // one byte at m * blocks + k
    uint8_t* const rest = few_lds + (rows * blocks * (kBlockK + 1) + 1023) / 1024 * 1024;
    uint8_t* const room = rest + wave * 2048;
    v4f* const sums = reinterpret_cast<v4f*>(rest + kFewWaves * 2048);
    const Turn turn;
    const uint32_t row = min(lane & 15, rows - 1), g = lane >> 4;

    // a wave's runs of blocks for one tile are `batches` loads
    const Runs runs(blocks, kFewWaves, wave);
    const uint32_t batches = uniform((blocks + runs.run * kFewWaves - 1) / (runs.run * kFewWaves));
    v4i line[kAhead][2], next_line[kAhead][2];
    uint32_t scales = 0, next_scales = 0;
    auto load = [&](uint32_t tile, uint32_t batch) {
        Lines<1> b;
        b.set_up(p.b, tile * 16);
        Runs k = runs;
        k.at += batch * runs.run * kFewWaves;
        v4i one[1][2];
        uint32_t s[1] = {0};
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if ((uint32_t)u < k.run && k.at + u < blocks) {
                b.load(k.at + u, one);
                next_line[u][0] = one[0][0];
                next_line[u][1] = one[0][1];
            }
        }
        if (k.at < blocks) b.load_scales(k, blocks, s);
        next_scales = s[0];
    };
    load(blockIdx.x, 0);

    // sixteen lanes a block
    for (uint32_t c = threadIdx.x / 16; c < rows * blocks; c += kFewWaves * 4) {
        const uint32_t m = c / blocks, k = c - m * blocks, part = threadIdx.x % 16, col = k * kBlockK + part * 8;
        Eight<T> eight[1];
        load_eights(eight, x.data + (uint64_t)m * x.ld * sizeof(T), 0, 1, col, (int64_t)x.cols - col);
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = finite(eight[0][j]);
        float most = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) most = larger(most, v[j]);
        const uint32_t s = scale_byte(max_of_16_lanes(bits_of(most)));
        const float inv = inverse_scale(s);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = v[j] * inv;
        const u32x2 out = {encode4(v[0], v[1], v[2], v[3]), encode4(v[4], v[5], v[6], v[7])};
        *reinterpret_cast<u32x2*>(held + (k * rows + m) * kBlockK + ((part / 2) ^ swizzle(m)) * 16 + part % 2 * 8) = out;
        if (part == 0) held_scale[m * blocks + k] = (uint8_t)s;
    }
    __syncthreads();

    uint32_t turns = 0;
    for (uint32_t tile = blockIdx.x; tile < p.tiles_n; tile += gridDim.x, ++turns) {
        v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
        for (uint32_t batch = 0; batch < batches; ++batch) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                line[u][0] = next_line[u][0];
                line[u][1] = next_line[u][1];
            }
            scales = next_scales;
            if (batch + 1 < batches) {
                load(tile, batch + 1);
            } else if (tile + gridDim.x < p.tiles_n) {
                load(tile + gridDim.x, 0);
            }
            const uint32_t first = runs.at + batch * runs.run * kFewWaves;
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const uint32_t k = first + u;
                if ((uint32_t)u < runs.run && k < blocks) {
                    turn.put(room, line[u]);
                    lanes_meet();
                    const uint8_t* a = held + (k * rows + row) * kBlockK;
                    const v8i xa = __builtin_shufflevector(*reinterpret_cast<const v4i*>(a + (g ^ swizzle(row)) * 16),
                                                           *reinterpret_cast<const v4i*>(a + ((g + 4) ^ swizzle(row)) * 16),
                                                           0, 1, 2, 3, 4, 5, 6, 7);
                    const v8i xb = turn.get(room);
                    lanes_meet();
                    acc = mfma_block<kWide>(xb, xa, acc, scales >> (8 * u) & 0xffu, held_scale[row * blocks + k]);
                }
            }
        }
        v4f* at = sums + (turns & 1) * kFewWaves * 64;
        at[wave * 64 + lane] = acc;
        __syncthreads();
        // one wave after the other has the joining, the rest go on (and write the other set)
        if (turns % kFewWaves == wave) {
            v4f y = at[lane];
#pragma unroll
            for (int w = 1; w < kFewWaves; ++w) {
                const v4f z = at[w * 64 + lane];
#pragma unroll
                for (int i = 0; i < 4; ++i) y[i] = y[i] + z[i];
            }
            store4(p, lane & 15, tile * 16 + g * 4, y);
        }
    }
}

}  // namespace

hipError_t launch_quantize(const Plain& x, const Fp8* along_rows, const Fp8* along_cols, bool square,
                           hipStream_t stream) {
    Quantize q = {};
    q.x = x;
    if (along_rows != nullptr) q.rows = *along_rows;
    if (along_cols != nullptr) q.cols = *along_cols;
    q.tiles_c = (x.cols + kBlockK - 1) / kBlockK;
    const uint32_t grid = q.tiles_c * ((x.rows + kBlockK - 1) / kBlockK);
    if (x.dtype == kF32) {
        quantize<float>(q, along_rows != nullptr, along_cols != nullptr, square, grid, stream);
    } else {
        quantize<uint16_t>(q, along_rows != nullptr, along_cols != nullptr, square, grid, stream);
    }
    return hipGetLastError();
}

hipError_t launch_transpose(const Bytes& b, hipStream_t stream) {
    const uint32_t grid = ((b.cols + kBlockK - 1) / kBlockK) * ((b.rows + kBlockK - 1) / kBlockK);
    transpose_kernel<<<grid, 256, 0, stream>>>(b);
    return hipGetLastError();
}

template <bool kWide>
static void product(Tile tile, const Product& p, hipStream_t stream) {
    const uint32_t parts = p.part_blocks != 0 ? (p.kblocks + p.part_blocks - 1) / p.part_blocks : 1;
    const uint32_t grid = p.tiles_m * p.tiles_n * parts;
    switch (tile) {
        case Tile::Shared16: shared_tile_kernel<1, 1, 8, kWide><<<grid, 512, 0, stream>>>(p); break;
        case Tile::Shared32: shared_tile_kernel<2, 2, 8, kWide><<<grid, 512, 0, stream>>>(p); break;
        case Tile::Shared64: shared_tile_kernel<4, 4, 4, kWide><<<grid, 256, 0, stream>>>(p); break;
        case Tile::Shared64Long:
            if constexpr (kWide) shared_tile_kernel<4, 4, 8, true><<<grid, 512, 0, stream>>>(p);
            break;
        case Tile::Deep128:
            if constexpr (kWide) {
                wide_product_kernel<128, 128, 2, 2, 4><<<grid, 256, 0, stream>>>(p);
            } else {
                product_kernel<128, 128, 2, 2, 4><<<grid, 256, 0, stream>>>(p);
            }
            break;
        case Tile::Narrow128:
            if constexpr (!kWide) product_kernel<128, 64, 2, 2, 4><<<grid, 256, 0, stream>>>(p);
            break;
        case Tile::Square128:
            if constexpr (kWide) {
                wide_product_kernel<128, 128, 2, 2, 2><<<grid, 256, 0, stream>>>(p);
            } else {
                product_kernel<128, 128, 2, 2, 2><<<grid, 256, 0, stream>>>(p);
            }
            break;
        case Tile::Square256:
            if constexpr (kWide) {
                wide_product_kernel<256, 256, 2, 2, 2><<<grid, 256, 0, stream>>>(p);
            } else {
                product_kernel<256, 256, 4, 2, 2><<<grid, 512, 0, stream>>>(p);
            }
            break;
    }
}

hipError_t launch_product(Tile tile, const Product& p, hipStream_t stream) {
    if (p.wide) {
        product<true>(tile, p, stream);
    } else {
        product<false>(tile, p, stream);
    }
    if (p.part_blocks != 0) {
        const uint64_t fours = (uint64_t)p.a.rows * (p.ld_sums / 4);
        join_kernel<<<(uint32_t)((fours + 255) / 256), 256, 0, stream>>>(p, (p.kblocks + p.part_blocks - 1) / p.part_blocks);
    }
    return hipGetLastError();
}

uint32_t few_rows_bytes(uint32_t rows, uint32_t blocks) { return few_rows_lds(rows, blocks); }

template <typename T>
static void few_rows(const Plain& x, const Product& p, hipStream_t stream) {
    // two workgroups a CU, each with as many of the tiles as the others
    const uint32_t turns = (p.tiles_n + 511) / 512, grid = (p.tiles_n + turns - 1) / turns;
    const uint32_t lds = few_rows_lds(x.rows, p.kblocks);
    if (p.wide) {
        few_rows_kernel<T, true><<<grid, kFewWaves * 64, lds, stream>>>(x, p);
    } else {
        few_rows_kernel<T, false><<<grid, kFewWaves * 64, lds, stream>>>(x, p);
    }
}

hipError_t launch_few_rows(const Plain& x, const Product& p, hipStream_t stream) {
    if (x.dtype == kF32) {
        few_rows<float>(x, p, stream);
    } else {
        few_rows<uint16_t>(x, p, stream);
    }
    return hipGetLastError();
}

}  // namespace pact
