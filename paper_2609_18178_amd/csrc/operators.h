// operators.h -- internal interface between the host side of the training
// operators (operators.hip) and their gfx950 kernels (fp8.hip, distill.hip).
// Not installed.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace pact {

// Records a failed HIP call for pact_last_hip_error(); returns PACT_EHIP.
int fail_hip(hipError_t e);

constexpr uint32_t kF32 = 0, kBf16 = 1;  // element types (PACT_F32, PACT_BF16)

constexpr uint32_t kBlockK = 128;     // elements that share a scale
constexpr uint32_t kScaleGroup = 4;   // scales that a kernel loads at once

// A matrix of binary32 or bf16 elements.
struct Plain {
    char* data;
    uint32_t rows, cols;
    uint64_t ld;    // elements between rows
    uint32_t dtype;
};

// A matrix in FP8 with its scales.
struct Fp8 {
    uint8_t* data;
    uint8_t* scale;
    uint32_t rows, cols;
    uint32_t ld, scale_ld;  // bytes between rows
};

// How a product ends: the binary32 sums go to C as they are, rounded to bf16, or added to C.
enum class Out : uint32_t { F32 = 0, Bf16 = 1, AddF32 = 2 };

struct Product {
    Fp8 a, b;         // C[m, n] = sum over k of a[m, k] * b[n, k]
    char* c;
    uint64_t ldc;     // elements
    Out out;
    bool wide;        // sums of binary32 all through: C is binary32
    uint32_t kblocks; // of 128
    uint32_t tiles_m, tiles_n;
    // In parts of K (Tile::Deep128): blocks of each, a multiple of kScaleGroup, and their sums, part after
    // part, rows of `ld_sums` elements.  0: not.
    uint32_t part_blocks, ld_sums;
    float* sums;
};

// The tiles that a product can be cut into: of a square of C for a workgroup whose waves share
// the blocks of K, or whose waves have a part of the tile each.
enum class Tile : int { Shared16, Shared32, Shared64, Shared64Long, Deep128, Narrow128, Square128, Square256 };

constexpr uint32_t kQuantizeThreads = 512;  // of a workgroup, which takes 128 x 128 elements
hipError_t launch_quantize(const Plain& x, const Fp8* along_rows, const Fp8* along_cols, bool square,
                           hipStream_t stream);
// out[j, i] = in[i, j] of rows x cols bytes.
struct Bytes {
    const uint8_t* in;
    uint8_t* out;
    uint64_t ld, out_ld;
    uint32_t rows, cols;
};
hipError_t launch_transpose(const Bytes& b, hipStream_t stream);
hipError_t launch_product(Tile tile, const Product& p, hipStream_t stream);
// The product of up to 16 rows that are quantised on the way, in tiles of 16 rows of b, with
// few_rows_bytes() bytes of LDS a workgroup.
uint32_t few_rows_bytes(uint32_t rows, uint32_t blocks);
hipError_t launch_few_rows(const Plain& x, const Product& p, hipStream_t stream);

// The distillation loss of `rows` rows of logits against a teacher's top ones.
constexpr uint32_t kMaxTop = 1024;
enum class Distill : int { Loss = 0, Grad = 1, Step = 2 };
struct DistillArgs {
    const char* logits;
    char* grad;
    const char* top_logits;
    const char* top_index;
    const float* row_weight;  // or null: ones
    float* loss;
    float* lse;               // written by Loss, read by Grad; Step: written unless null
    uint64_t ld_logits, ld_grad, ld_top_logits, ld_top_index;  // elements
    uint32_t rows, vocab, top;
    float to_log2;            // log2(e) / temperature
    float inv_temperature;
    uint32_t dtype, top_dtype;
    bool wide_index;          // 64-bit indices
};
hipError_t launch_distill(Distill kind, const DistillArgs& d, hipStream_t stream);

}  // namespace pact
