// operators.hip -- host side of the training operators: argument validation,
// the choice of tiles, and the launches.  The C ABI and its contract are in
// include/pactshard.h.
#include "operators.h"

#include <algorithm>
#include <cmath>

#include "pactshard.h"

static_assert(pact::kF32 == PACT_F32 && pact::kBf16 == PACT_BF16, "element types");
static_assert(pact::kBlockK == PACT_FP8_BLOCK && pact::kMaxTop == PACT_DISTILL_MAX_TOP, "the header's figures");

namespace {

using pact::Tile;

// Rows and columns stay in 32-bit arithmetic with tiles to spare, and a row of FP8 bytes
// within the offsets that a tile adds to its base.
constexpr uint64_t kMaxRows = 1ull << 31;
constexpr uint64_t kMaxCols = 1ull << 31;
// A dispatch counts its work-items in 32 bits.
constexpr uint64_t kMaxItems = UINT32_MAX;
constexpr uint64_t kCus = 256;
// A row of FP8 bytes: 256 of them are counted in 32 bits.
constexpr uint64_t kMaxFp8Row = 1ull << 24;
// A product of up to so many rows can quantise them on the way, with this LDS a workgroup: two fit a CU.
constexpr uint64_t kFewRows = 16;
constexpr uint64_t kFewLds = 64 * 1024;
constexpr double kLog2e = 1.4426950408889634074;

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }
uint64_t round_up(uint64_t a, uint64_t b) { return ceil_div(a, b) * b; }
uint32_t esize(uint32_t dtype) { return dtype == PACT_F32 ? 4 : 2; }

// The buffers of one call. Inputs may share memory with each other, an output with nothing; rows of one matrix beside
// those of another, as column slices of a larger one are, share none.
class Spans {
public:
    // rows x width bytes, `stride` bytes apart; false if that wraps the address space
    bool add(const void* p, uint64_t rows, uint64_t stride, uint64_t width, bool written) {
        if (p == nullptr || rows == 0 || width == 0) return true;
        const unsigned __int128 bytes = (unsigned __int128)(rows - 1) * stride + width;
        const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
        if (bytes > UINTPTR_MAX - lo) return false;
        s_[n_++] = {lo, lo + (uintptr_t)bytes, rows > 1 ? stride : 0, width, written};
        return true;
    }
    bool overlap() const {
        for (int i = 0; i < n_; ++i) {
            for (int j = i + 1; j < n_; ++j) {
                const Span &a = s_[i], &b = s_[j];
                if ((a.written || b.written) && a.lo < b.hi && b.lo < a.hi && !beside(a, b)) return true;
            }
        }
        return false;
    }

private:
    struct Span {
        uintptr_t lo, hi;
        uint64_t stride, width;  // stride 0: one row
        bool written;
    };
    // Whether no row of either meets one of the other, however many there are: the same distance between rows, and
    // the one's bytes of it are not the other's. (A single row is taken to be one of rows so far apart.)
    static bool beside(const Span& a, const Span& b) {
        const uint64_t stride = a.stride != 0 ? a.stride : b.stride;
        if (stride == 0 || (b.stride != 0 && b.stride != stride)) return false;
        const uint64_t ahead = b.lo >= a.lo ? (b.lo - a.lo) % stride : (stride - (a.lo - b.lo) % stride) % stride;
        return ahead >= a.width && b.width <= stride && ahead <= stride - b.width;
    }
    Span s_[10];
    int n_ = 0;
};

int check(const pact_matrix& x) {
    if (x.dtype > PACT_BF16 || x.reserved != 0) return PACT_EINVAL;
    if (x.rows > 0 && x.cols > 0 && x.data == nullptr) return PACT_EINVAL;
    if (x.rows >= kMaxRows || x.cols >= kMaxCols || x.ld > (1ull << 40)) return PACT_ERANGE;
    if (x.rows > 1 && x.ld < x.cols) return PACT_EINVAL;
    return aligned(x.data, esize(x.dtype)) ? PACT_OK : PACT_EALIGN;
}

int check(const pact_fp8& x) {
    if (x.rows >= kMaxRows || x.ld >= kMaxFp8Row || x.scale_ld >= kMaxFp8Row) return PACT_ERANGE;
    if (x.cols > x.ld) return PACT_EINVAL;
    const uint64_t blocks = ceil_div(x.cols, PACT_FP8_BLOCK);
    if (x.rows > 0 && x.cols > 0 && (x.data == nullptr || x.scale == nullptr)) return PACT_EINVAL;
    if (x.ld < blocks * PACT_FP8_BLOCK || x.ld % PACT_FP8_BLOCK != 0) return PACT_EINVAL;
    if (x.scale_ld < round_up(blocks, pact::kScaleGroup) || x.scale_ld % pact::kScaleGroup != 0) return PACT_EINVAL;
    return aligned(x.data, 16) && aligned(x.scale, 4) ? PACT_OK : PACT_EALIGN;
}

bool add(Spans& s, const pact_matrix& x, bool written) {
    return s.add(x.data, x.rows, x.ld * esize(x.dtype), x.cols * esize(x.dtype), written);
}

bool add(Spans& s, const pact_fp8& x, bool written) {
    const uint64_t blocks = ceil_div(x.cols, PACT_FP8_BLOCK);
    return s.add(x.data, x.rows, x.ld, blocks * PACT_FP8_BLOCK, written) &&
           s.add(x.scale, x.rows, x.scale_ld, round_up(blocks, pact::kScaleGroup), written);
}

pact::Plain plain(const pact_matrix& x) {
    pact::Plain p;
    p.data = static_cast<char*>(x.data);
    p.rows = (uint32_t)x.rows;
    p.cols = (uint32_t)x.cols;
    p.ld = x.ld;
    p.dtype = x.dtype;
    return p;
}

pact::Fp8 fp8(const pact_fp8& x) {
    return {x.data, x.scale, (uint32_t)x.rows, (uint32_t)x.cols, (uint32_t)x.ld, (uint32_t)x.scale_ld};
}

// Workgroups of a quantisation.
uint64_t squares(const pact_matrix& x) {
    return ceil_div(x.rows, pact::kBlockK) * ceil_div(x.cols, pact::kBlockK);
}

// ---------------------------------------------------------------------------
// how a product is cut
// ---------------------------------------------------------------------------
struct Cut {
    Tile tile;
    uint32_t side;     // of its squares of C
    uint32_t threads;  // of a workgroup
    uint32_t part_blocks = 0;  // of K, if it is cut too
    uint32_t side_n = 0;       // along C's rows, if they are no squares
};

// The parts that K is cut into, each a square of 128's for a workgroup of its own, so that there is one for nearly
// every CU.  The sums of the parts go through memory and a second kernel, which takes as long as ten to fifteen blocks:
// so K has to be long, or, where the squares of 128 are the choice already but half of the CUs or more are without
// one, of 40 blocks (at 32, inputs that are in the caches take 2 us more in parts).  A square has to be half
// full at least, and is cut into four parts or more if it is no fuller.  us, uncut / cut, inputs out of memory, with bf16 and with binary32 result:
//                     K = 4096                     K = 8192                     K = 14336
//    512 x  4096   22.4 / 21.1   30.7 / 27.7    41.0 / 31.3   53.6 / 42.3    71.1 / 47.5   85.0 / 63.9
//    512 x  2048   13.8 / 17.8   18.9 / 21.4    22.6 / 21.2   30.8 / 27.8    36.3 / 30.4   45.3 / 39.8
//    256 x  4096   14.8 / 18.4   20.2 / 21.9    24.8 / 22.5   32.0 / 27.9    37.8 / 30.8   46.7 / 38.9
//    256 x  2048   12.0 / 16.3   12.9 / 19.6    20.8 / 17.3   21.5 / 20.8    31.8 / 22.2   32.8 / 27.2
//    256 x  1024    7.1 / 12.2    7.8 / 15.5    12.6 / 16.6   13.0 / 18.6    19.6 / 17.7   19.7 / 20.5
//    128 x 14336   25.0 / 22.2   33.8 / 27.4    46.3 / 40.9   59.6 / 45.8    82.2 / 60.8   98.6 / 67.3
//    128 x  2048    8.1 / 14.1    8.4 / 16.1    13.3 / 17.3   13.4 / 19.1    20.4 / 17.8   20.7 / 20.4
//     64 x 14336   18.3 / 19.0   23.9 / 25.3    34.1 / 36.3   39.9 / 42.5    55.2 / 52.1   64.7 / 64.8
//     64 x  8192   15.3 / 16.0   15.5 / 18.7    26.1 / 21.9   26.1 / 26.1    39.8 / 31.5   40.3 / 38.6
//     32 x  8192   10.7 / 15.1   10.8 / 18.5    16.8 / 20.5   17.0 / 25.3    28.4 / 29.2   28.9 / 37.6
struct Parts {
    uint64_t count;
    uint32_t blocks;  // of each, of 128
};
Parts parts_of(uint64_t m, uint64_t n, uint64_t k) {
    auto tiles = [&](uint64_t side) { return ceil_div(m, side) * ceil_div(n, side); };
    const uint64_t blocks = ceil_div(k, pact::kBlockK), all = tiles(128), less = std::min(m, n);
    if (less < 64 || 2 * all > kCus || blocks < 40) return {1, 0};
    const uint64_t most = std::min(kCus / all, blocks / 8);
    const bool is_long = blocks >= 64 && tiles(32) * blocks > 64 * kCus;
    if (!(is_long || tiles(64) > kCus) || (less == 64 && most < 4)) return {1, 0};
    const uint64_t each = round_up(ceil_div(blocks, most), pact::kScaleGroup);
    return {ceil_div(blocks, each), (uint32_t)each};
}

// The smallest square of which there are few enough, its waves sharing K: two for each CU, or one for each
// where a bf16 result's squares of 128 do as well.  Beyond those, a part of the tile for each wave: squares of 128,
// with their LDS full of blocks to come where a CU has one of them at most; squares of 256 where the
// squares of 128 would take a second turn and the edges waste no more than a fifth.  A binary32 result has more to
// store behind its last block, which goes on beside another square of 128: there the squares of 256 have to save an
// eighth of the turns, and, where they take more than one, more than a few blocks.
// Squares of 64 have four waves, so that a CU holds two, and eight where a CU has one of them and the bytes are
// widened, which is what they wait for: with binary32 result, 256 x 4096, four / eight waves: K = 512 7.1 / 7.4 us,
// 1024 9.3 / 8.8, 4096 23.9 / 20.2, 8192 41 / 33; with bf16 result 6.0 / 6.2, 7.2 / 7.1, 14.9 / 14.6, 24.7 / 23.5.
// A bf16 result whose squares of 128 are for half of the CUs at most, those of 64 for more than all: halves of 128 x 64,
// one for each CU.  us, deep squares of 128 (K in parts from 5000 on) / halves: 512 x 4096, K = 512 6.5 / 6.0, 1024 8.1 / 6.9,
// 2048 11.1 / 9.4, 4096 18.0 / 15.1, 5000 21.3 / 17.4, 14336 37.8 / 40.5; 500 x 3000 x 8192 25.0 / 24.6; 1024 x 2048 x 4096 17.2 / 14.4,
// 300 x 4096 x 4096 17.7 / 14.7.  From 64 blocks on the parts are left.  Outside of those sizes: 256 x 4096 x 4096 in squares of 64 /
// halves 12.8 / 14.0; 600 x 4096 x 2048, of 320 halves, in squares of 128 / halves 12.1 / 16.6.
// Up to 16 rows of a are in squares of 16 however many there are: their waves add in the order of the product that quantises
// its rows on the way, so that both give the same bits, and the larger squares would be empty in most of their rows.  us, weights out of
// memory, in the larger squares / of 16, with bf16 and with binary32 result: 1 x 17000 x 4096 23.3 / 16.4, 30.9 / 16.3; 1 x 140000 x 4096 148 / 93,
// 165 / 94; 16 x 140000 x 4096 154 / 114, 171 / 121; 1 x 140000 x 520 30.1 / 28.3, 36.3 / 33.2; 1 x 65536 x 520 13.3 / 14.9, 16.2 / 17.6.
// us per product of inputs out of memory, in squares of 16 / 32 / 64 / 128, deep / 128 / 256, with bf16 result:
//                 K = 1024                               K = 4096
//     16 x  4096    4.3   4.9   7.0   8.8     -     -     6.8   8.2  13.0  18.3     -     -
//     64 x  4096    6.1   5.2   8.1   8.9     -     -    11.9   9.0  15.4  19.9     -     -
//    128 x  4096    9.4   6.6   7.9   9.2     -     -    18.7  12.5  15.0  22.9     -     -
//    256 x  4096   15.1  10.6   8.1   9.2  11.7     -    33.0  19.9  14.8  22.6  33.9     -
//    512 x  4096      -  18.2  10.2   9.5  11.9  16.2       -  33.8  22.1  22.7  33.8  43.1
//   1024 x  4096      -  33.5  17.7  10.8  12.7  16.7       -  59.6  36.4  24.4  34.6  43.0
//    512 x 14336      -     -  29.5  19.2  16.0  18.4       -     -  62.6  47.4  42.7  46.3
//   2500 x  4096      -     -  34.9  24.6  22.4  19.6       -     -  78.5  58.7  60.9  47.3
//   4096 x  4096      -     -  55.8  35.0  29.3  22.5       -     -   125  88.8  77.3  56.6
//   6000 x  4096      -     -     -  48.2  40.0  39.3       -     -     -   116   103  97.6
//  14336 x  4096      -     -     -  99.3  78.3  78.3       -     -     -   261   232   200
// and with binary32 result:
//    256 x  4096   18.8  11.7  10.2  12.7  15.7     -    36.9  22.0  23.6  33.6  46.5     -
//    512 x  4096      -  19.9  14.0  13.3  16.2  28.0       -  38.8  32.3  34.7  47.1  81.9
//   1024 x  4096      -  35.7  23.6  15.1  17.6  29.0       -  66.3  54.3  36.6  46.9  81.8
//    512 x 14336      -     -  39.8  26.7  20.8  30.0       -     -  97.1  71.3  58.8  84.5
//   2500 x  4096      -     -  45.9  36.5  31.7  33.6       -     -   120  99.9  91.1  90.1
//   4096 x  4096      -     -  76.8  52.4  41.9  36.6       -     -   195   138   117  99.0
//   6000 x  4096      -     -     -  71.1  59.7  66.3       -     -     -   201   168   179
//  14336 x  4096      -     -     -   154   123   124       -     -     -   468   398   361
Cut cut(uint64_t m, uint64_t n, uint64_t k, bool wide) {
    auto tiles = [&](uint64_t side) { return ceil_div(m, side) * ceil_div(n, side); };
    const Parts parts = parts_of(m, n, k);
    const bool halves = !wide && tiles(64) > kCus && ceil_div(m, 128) * ceil_div(n, 64) <= kCus;
    if (halves && (parts.count <= 1 || k <= 63 * pact::kBlockK)) return {Tile::Narrow128, 128, 256, 0, 64};
    if (parts.count > 1) return {Tile::Deep128, 128, 256, parts.blocks};
    if ((m <= kFewRows && tiles(16) <= kMaxItems / 512) || tiles(16) <= 2 * kCus) return {Tile::Shared16, 16, 512};
    if (tiles(32) <= 2 * kCus) return {Tile::Shared32, 32, 512};
    if (wide && tiles(64) <= kCus && k >= 1024) return {Tile::Shared64Long, 64, 512};
    if (tiles(64) <= (wide ? 2 : 1) * kCus) return {Tile::Shared64, 64, 256};
    const uint64_t all = tiles(128), large = tiles(256), turns = ceil_div(large, kCus);
    if (all <= kCus) return {Tile::Deep128, 128, 256};
    if (wide ? all * 2 >= turns * 7 * kCus && (turns == 1 || k > 1024) : all > 2 * kCus && all * 5 >= large * 16) {
        return {Tile::Square256, 256, 512};
    }
    return {Tile::Square128, 128, 256};
}

// A long product in squares of 256 whose last turn would be part of one is cut along one side of C: squares of 256 for
// the turns that are full (to seven eighths), then the rest, of at most 512 squares of 128, in a launch of its own: one
// deep square a CU, or two.  That saves a part of a turn: K has to be long, and for a binary32 result, whose squares
// of 128 wait for less, longer where only one turn is full; and the second launch has to be well filled.
// Of two ways to cut, rows of C or its columns, the one that leaves more squares to the second launch (8192 x 4800 x 4096 by
// rows / columns 145 / 147 us and 245 / 243, 8192 x 8900 x 4096 258 / 258 and 443 / 443).
// us uncut / cut, inputs out of memory, with bf16 and with binary32 result (within 3%; for K = 1024 and one turn of a binary32 result
// of K = 2048, 1300 x 14336 x 4096 among them, the cut that the rule does not make):
//                       K = 1024                     K = 2048                     K = 4096
//   4300 x  4096   34.6 / 32.0   49.9 / 50.4   52.8 / 46.8   79.9 / 77.9   89.8 / 77.0    142 /  130
//   5000 x  4096   35.4 / 33.3   49.2 / 54.7   53.0 / 48.5   79.6 / 83.3   91.5 / 80.7    144 /  136
//   6000 x  4096   38.8 / 39.6   55.3 / 59.2   57.8 / 57.8   94.5 / 95.6   97.3 / 95.6    174 /  158
//   1300 x 14336   37.6 / 34.9   54.0 / 52.8   56.8 / 51.7   85.0 / 85.7   94.0 / 86.2    156 /  148
//   3000 x 11008   55.8 / 51.5   77.4 / 82.2   83.0 / 75.3    132 /  125    141 /  127    240 /  216
//   8192 x  4800   60.1 / 58.2    100 / 90.7   88.3 / 85.7    158 /  141    148 /  146    281 /  243
//   8192 x  5120   58.7 / 57.8   99.1 / 92.8   87.1 / 86.7    159 /  144    151 /  148    289 /  249
//  14336 x  4096   78.5 / 79.8    126 /  129    118 /  119    200 /  196    195 /  199    364 /  351
//   8192 x  8900    109 /  104    188 /  166    157 /  153    267 /  253    259 /  258    460 /  437
struct Split {
    bool rows;    // of C, or its columns
    uint64_t at;  // where; 0: not cut
    Cut rest;
};
Split split_of(uint64_t m, uint64_t n, uint64_t k, bool wide) {
    const uint64_t tiles_m = ceil_div(m, 256), tiles_n = ceil_div(n, 256), turns = tiles_m * tiles_n / kCus;
    Split best = {};
    if (turns == 0 || k < 2048 || (wide && turns == 1 && k < 4096)) return best;
    uint64_t most = 0;
    for (const bool rows : {true, false}) {
        const uint64_t length = rows ? m : n, strips = turns * kCus / (rows ? tiles_n : tiles_m);
        if (strips == 0 || strips * 256 >= length) continue;
        const uint64_t across = ceil_div(rows ? n : m, 128), rest = ceil_div(length - strips * 256, 128) * across;
        const bool one_a_cu = rest <= kCus;
        if (rest > 2 * kCus || strips * 2 * across * 2 < turns * 7 * kCus) continue;
        if (wide && turns == 1 && !one_a_cu && rest <= 400) continue;
        // the rest in one square a CU if either side allows it, and then as much of it as there can be
        const uint64_t worth = one_a_cu ? 2 * kCus + rest : rest;
        if (worth <= most) continue;
        most = worth;
        best = {rows, strips * 256, {one_a_cu ? Tile::Deep128 : Tile::Square128, 128, 256}};
    }
    return best;
}

// Bytes of x quantised along its rows, both parts in whole multiples of 256.
uint64_t held_bytes(uint64_t m, uint64_t k) { return round_up(m * round_up(k, PACT_FP8_BLOCK), 256); }
uint64_t held_scale_bytes(uint64_t m, uint64_t k) {
    return round_up(m * round_up(ceil_div(k, PACT_FP8_BLOCK), pact::kScaleGroup), 256);
}
// Whether a product of x (m x k) with n rows quantises it on its way, in every workgroup: where it would be in squares of 16.
bool on_the_way(uint64_t m, uint64_t n, uint64_t k) {
    return m <= kFewRows && ceil_div(n, 16) <= kMaxItems / 512 && k < kMaxFp8Row && pact::few_rows_bytes((uint32_t)m, (uint32_t)ceil_div(k, pact::kBlockK)) <= kFewLds;
}

// C = a b^T in one launch (and the joining of the parts of K); with x, of x on the way and no more of `a` than its size.
int product(const pact_fp8& a, const pact_fp8& b, const pact_matrix& c, bool add, const Cut& how, const pact_matrix* x,
            uint8_t* sums, hipStream_t stream) {
    const uint64_t m = c.rows, n = c.cols, k = b.cols;
    pact::Product p = {};
    p.a = fp8(a);
    p.b = fp8(b);
    p.c = static_cast<char*>(c.data);
    p.ldc = c.ld;
    p.out = c.dtype == PACT_BF16 ? pact::Out::Bf16 : add ? pact::Out::AddF32 : pact::Out::F32;
    p.wide = c.dtype == PACT_F32;
    p.kblocks = (uint32_t)ceil_div(k, pact::kBlockK);
    p.part_blocks = how.part_blocks;
    p.ld_sums = (uint32_t)round_up(n, 4);
    p.sums = reinterpret_cast<float*>(sums);
    const uint64_t side_n = how.side_n != 0 ? how.side_n : how.side;
    p.tiles_m = (uint32_t)ceil_div(m, how.side);
    p.tiles_n = (uint32_t)ceil_div(n, side_n);
    if (ceil_div(m, how.side) * ceil_div(n, side_n) > kMaxItems / how.threads) return PACT_ERANGE;
    const hipError_t e =
        x != nullptr ? pact::launch_few_rows(plain(*x), p, stream) : pact::launch_product(how.tile, p, stream);
    return e == hipSuccess ? PACT_OK : pact::fail_hip(e);
}

// Rows from..to of a matrix in FP8.
pact_fp8 rows_of(const pact_fp8& x, uint64_t from, uint64_t to) {
    return {x.data + from * x.ld, x.scale + from * x.scale_ld, to - from, x.cols, x.ld, x.scale_ld};
}

// C = a b^T, the arguments already checked.
int product(const pact_fp8& a, const pact_fp8& b, const pact_matrix& c, bool add, const pact_matrix* x, uint8_t* sums,
            hipStream_t stream) {
    const uint64_t m = c.rows, n = c.cols, k = b.cols;
    const bool wide = c.dtype == PACT_F32;
    if (m == 0 || n == 0) return PACT_OK;
    if (x != nullptr) return product(a, b, c, add, {Tile::Shared16, 16, 512}, x, sums, stream);
    const Split split = split_of(m, n, k, wide);
    if (split.at == 0) return product(a, b, c, add, cut(m, n, k, wide), nullptr, sums, stream);
    const uint64_t at = split.at;
    char* const data = static_cast<char*>(c.data);
    pact_fp8 a1 = a, a2 = a, b1 = b, b2 = b;
    pact_matrix c1 = c, c2 = c;
    if (split.rows) {
        a1 = rows_of(a, 0, at), a2 = rows_of(a, at, m);
        c1.rows = at, c2.rows = m - at, c2.data = data + at * c.ld * esize(c.dtype);
    } else {
        b1 = rows_of(b, 0, at), b2 = rows_of(b, at, n);
        c1.cols = at, c2.cols = n - at, c2.data = data + at * esize(c.dtype);
    }
    const int rc = product(a1, b1, c1, add, {Tile::Square256, 256, 512}, nullptr, nullptr, stream);
    return rc != PACT_OK ? rc : product(a2, b2, c2, add, split.rest, nullptr, nullptr, stream);
}

// Scratch memory of a product whose K is cut, for either type of C (a bf16 result may leave it alone).
uint64_t sums_bytes(uint64_t m, uint64_t n, uint64_t k) {
    const Parts parts = parts_of(m, n, k);
    return parts.count <= 1 ? 0 : parts.count * m * round_up(n, 4) * 4;
}

// x quantised in scratch memory, at its start.
struct Held {
    pact_fp8 x;
    uint64_t bytes;
};
Held held_at(uint8_t* at, uint64_t rows, uint64_t cols) {
    const uint64_t blocks = ceil_div(cols, PACT_FP8_BLOCK), data = held_bytes(rows, cols);
    return {{at, at + data, rows, cols, blocks * PACT_FP8_BLOCK, round_up(blocks, pact::kScaleGroup)},
            data + held_scale_bytes(rows, cols)};
}

int check_workspace(Spans& spans, void* workspace, uint64_t bytes) {
    if (workspace == nullptr) return PACT_OK;
    if (!aligned(workspace, 256)) return PACT_EALIGN;
    return spans.add(workspace, 1, 0, bytes, true) ? PACT_OK : PACT_ERANGE;
}

int distill(pact::Distill kind, const pact_distill* s) {
    using pact::Distill;
    if (s == nullptr) return PACT_EINVAL;
    if (s->dtype > PACT_BF16 || s->top_dtype > PACT_BF16 || s->reserved != 0) return PACT_EINVAL;
    if (s->index_bytes != 4 && s->index_bytes != 8) return PACT_EINVAL;
    const float to_log2 = (float)(kLog2e / (double)s->temperature);
    // (below 2^-127.5 or so a difference of zero times an infinity would be NaN)
    if (!(s->temperature > 0.0f) || !std::isfinite(s->temperature) || !std::isfinite(to_log2)) return PACT_EINVAL;
    if (s->top > PACT_DISTILL_MAX_TOP) return PACT_EINVAL;
    // a workgroup of up to 1024 threads a row
    if (s->rows > kMaxItems / 1024 || s->vocab >= kMaxCols || s->ld_logits > (1ull << 40) || s->ld_grad > (1ull << 40) ||
        s->ld_top_logits > (1ull << 40) || s->ld_top_index > (1ull << 40)) {
        return PACT_ERANGE;
    }
    if (s->rows == 0) return PACT_OK;
    const bool writes_loss = kind != Distill::Grad, writes_grad = kind != Distill::Loss;
    if ((s->vocab > 0 && s->logits == nullptr) || (writes_loss && s->loss == nullptr) ||
        (writes_grad && s->vocab > 0 && s->grad == nullptr) || (kind != Distill::Step && s->lse == nullptr) ||
        (s->top > 0 && (s->top_logits == nullptr || s->top_index == nullptr))) {
        return PACT_EINVAL;
    }
    const uint64_t size = esize(s->dtype), tsize = esize(s->top_dtype);
    if (s->rows > 1 && (s->ld_logits < s->vocab || (writes_grad && s->ld_grad < s->vocab) || s->ld_top_logits < s->top ||
                        s->ld_top_index < s->top)) {
        return PACT_EINVAL;
    }
    if (!aligned(s->logits, size) || (writes_grad && !aligned(s->grad, size)) || !aligned(s->top_logits, tsize) ||
        !aligned(s->top_index, s->index_bytes) || !aligned(s->row_weight, 4) || !aligned(s->loss, 4) ||
        !aligned(s->lse, 4)) {
        return PACT_EALIGN;
    }
    const bool in_place = writes_grad && s->grad == s->logits;
    if (in_place && s->rows > 1 && s->ld_grad != s->ld_logits) return PACT_EOVERLAP;
    Spans spans;
    if (!spans.add(s->logits, s->rows, s->ld_logits * size, s->vocab * size, in_place) ||
        !(!writes_grad || in_place || spans.add(s->grad, s->rows, s->ld_grad * size, s->vocab * size, true)) ||
        !spans.add(s->top_logits, s->rows, s->ld_top_logits * tsize, s->top * tsize, false) ||
        !spans.add(s->top_index, s->rows, s->ld_top_index * s->index_bytes, s->top * s->index_bytes, false) ||
        !spans.add(s->row_weight, 1, 0, s->rows * 4, false) ||
        !(!writes_loss || spans.add(s->loss, 1, 0, s->rows * 4, true)) ||
        !spans.add(s->lse, 1, 0, s->rows * 4, writes_loss)) {
        return PACT_ERANGE;
    }
    if (spans.overlap()) return PACT_EOVERLAP;
    pact::DistillArgs d = {};
    d.logits = static_cast<const char*>(s->logits);
    d.grad = static_cast<char*>(s->grad);
    d.top_logits = static_cast<const char*>(s->top_logits);
    d.top_index = static_cast<const char*>(s->top_index);
    d.row_weight = s->row_weight;
    d.loss = s->loss;
    d.lse = s->lse;
    d.ld_logits = s->ld_logits;
    d.ld_grad = s->ld_grad;
    d.ld_top_logits = s->ld_top_logits;
    d.ld_top_index = s->ld_top_index;
    d.rows = (uint32_t)s->rows;
    d.vocab = (uint32_t)s->vocab;
    d.top = (uint32_t)s->top;
    d.inv_temperature = (float)(1.0 / (double)s->temperature);
    d.to_log2 = to_log2;
    d.dtype = s->dtype;
    d.top_dtype = s->top_dtype;
    d.wide_index = s->index_bytes == 8;
    const hipError_t e = pact::launch_distill(kind, d, static_cast<hipStream_t>(s->stream));
    return e == hipSuccess ? PACT_OK : pact::fail_hip(e);
}

}  // namespace

extern "C" {

int pact_fp8_quantize(const pact_matrix* x, const pact_fp8* along_rows, const pact_fp8* along_cols, uint32_t flags,
                      void* stream) {
    if (x == nullptr || (along_rows == nullptr && along_cols == nullptr) || (flags & ~PACT_FP8_SQUARE) != 0) {
        return PACT_EINVAL;
    }
    int rc = check(*x);
    if (rc != PACT_OK) return rc;
    Spans spans;
    bool fits = add(spans, *x, false);
    for (const pact_fp8* o : {along_rows, along_cols}) {
        if (o == nullptr) continue;
        rc = check(*o);
        if (rc != PACT_OK) return rc;
        fits = fits && add(spans, *o, true);
    }
    if (along_rows != nullptr && (along_rows->rows != x->rows || along_rows->cols != x->cols)) return PACT_EINVAL;
    if (along_cols != nullptr && (along_cols->rows != x->cols || along_cols->cols != x->rows)) return PACT_EINVAL;
    if (!fits || squares(*x) * pact::kQuantizeThreads > kMaxItems) return PACT_ERANGE;
    if (spans.overlap()) return PACT_EOVERLAP;
    if (x->rows == 0 || x->cols == 0) return PACT_OK;
    pact::Fp8 rows = {}, cols = {};
    if (along_rows != nullptr) rows = fp8(*along_rows);
    if (along_cols != nullptr) cols = fp8(*along_cols);
    const hipError_t e =
        pact::launch_quantize(plain(*x), along_rows ? &rows : nullptr, along_cols ? &cols : nullptr,
                              (flags & PACT_FP8_SQUARE) != 0, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? PACT_OK : pact::fail_hip(e);
}

int pact_fp8_transpose(const uint8_t* in, uint64_t rows, uint64_t cols, uint64_t ld, uint8_t* out, uint64_t out_ld,
                       void* stream) {
    if (rows >= kMaxRows || cols >= kMaxRows || ld > (1ull << 40) || out_ld > (1ull << 40)) return PACT_ERANGE;
    if (rows == 0 || cols == 0) return PACT_OK;
    if (in == nullptr || out == nullptr || (rows > 1 && ld < cols) || (cols > 1 && out_ld < rows)) return PACT_EINVAL;
    Spans spans;
    if (!spans.add(in, rows, ld, cols, false) || !spans.add(out, cols, out_ld, rows, true)) return PACT_ERANGE;
    if (spans.overlap()) return PACT_EOVERLAP;
    if (ceil_div(rows, pact::kBlockK) * ceil_div(cols, pact::kBlockK) * 256 > kMaxItems) return PACT_ERANGE;
    const pact::Bytes b = {in, out, ld, out_ld, (uint32_t)rows, (uint32_t)cols};
    const hipError_t e = pact::launch_transpose(b, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? PACT_OK : pact::fail_hip(e);
}

int64_t pact_fp8_matmul_workspace_bytes(uint64_t m, uint64_t n, uint64_t k) {
    if (m >= kMaxRows || n >= kMaxRows || k >= kMaxFp8Row) return PACT_ERANGE;
    return (int64_t)sums_bytes(m, n, k);
}

int pact_fp8_matmul(const pact_fp8* a, const pact_fp8* b, const pact_matrix* c, uint32_t flags, void* workspace,
                    uint64_t workspace_bytes, void* stream) {
    if (a == nullptr || b == nullptr || c == nullptr || (flags & ~PACT_FP8_ACCUMULATE) != 0) return PACT_EINVAL;
    int rc = PACT_OK;
    if ((rc = check(*a)) != PACT_OK || (rc = check(*b)) != PACT_OK || (rc = check(*c)) != PACT_OK) return rc;
    const bool add_to = (flags & PACT_FP8_ACCUMULATE) != 0;
    if (a->cols != b->cols || c->rows != a->rows || c->cols != b->rows || (add_to && c->dtype != PACT_F32)) {
        return PACT_EINVAL;
    }
    Spans spans;
    if (!add(spans, *a, false) || !add(spans, *b, false) || !add(spans, *c, true)) return PACT_ERANGE;
    if ((rc = check_workspace(spans, workspace, workspace_bytes)) != PACT_OK) return rc;
    if (spans.overlap()) return PACT_EOVERLAP;
    const uint64_t need = sums_bytes(c->rows, c->cols, a->cols);
    if (workspace_bytes < need || (need > 0 && workspace == nullptr)) return PACT_EINVAL;
    return product(*a, *b, *c, add_to, nullptr, static_cast<uint8_t*>(workspace), static_cast<hipStream_t>(stream));
}

int64_t pact_fp8_linear_workspace_bytes(uint64_t m, uint64_t n, uint64_t k) {
    if (m >= kMaxRows || n >= kMaxRows || k >= kMaxFp8Row) return PACT_ERANGE;
    return on_the_way(m, n, k) ? 0 : (int64_t)(held_at(nullptr, m, k).bytes + sums_bytes(m, n, k));
}

int pact_fp8_linear(const pact_matrix* x, const pact_fp8* w, const pact_matrix* y, void* workspace,
                    uint64_t workspace_bytes, void* stream) {
    if (x == nullptr || w == nullptr || y == nullptr) return PACT_EINVAL;
    int rc = PACT_OK;
    if ((rc = check(*x)) != PACT_OK || (rc = check(*w)) != PACT_OK || (rc = check(*y)) != PACT_OK) return rc;
    if (x->cols != w->cols || y->rows != x->rows || y->cols != w->rows) return PACT_EINVAL;
    Spans spans;
    if (!add(spans, *x, false) || !add(spans, *w, false) || !add(spans, *y, true)) return PACT_ERANGE;
    if ((rc = check_workspace(spans, workspace, workspace_bytes)) != PACT_OK) return rc;
    if (spans.overlap()) return PACT_EOVERLAP;
    const uint64_t m = x->rows, k = x->cols;
    if (on_the_way(m, y->cols, k)) {
        const pact_fp8 size = {nullptr, nullptr, m, k, 0, 0};
        return product(size, *w, *y, false, x, nullptr, static_cast<hipStream_t>(stream));
    }
    uint8_t* at = static_cast<uint8_t*>(workspace);
    const Held held = held_at(at, m, k);
    const uint64_t need = held.bytes + sums_bytes(m, y->cols, k);
    if (workspace_bytes < need || (need > 0 && workspace == nullptr)) return PACT_EINVAL;
    if (y->cols == 0) return PACT_OK;
    if (squares(*x) * pact::kQuantizeThreads > kMaxItems || held.x.ld >= kMaxFp8Row) return PACT_ERANGE;
    if (k > 0) {
        const pact::Fp8 rows = fp8(held.x);
        const hipError_t e = pact::launch_quantize(plain(*x), &rows, nullptr, false, static_cast<hipStream_t>(stream));
        if (e != hipSuccess) return pact::fail_hip(e);
    }
    return product(held.x, *w, *y, false, nullptr, at + held.bytes, static_cast<hipStream_t>(stream));
}

int64_t pact_fp8_linear_backward_workspace_bytes(uint64_t m, uint64_t n, uint64_t k) {
    if (m >= kMaxFp8Row || n >= kMaxFp8Row || k >= kMaxRows) return PACT_ERANGE;
    return (int64_t)(held_at(nullptr, m, n).bytes + held_at(nullptr, n, m).bytes +
                     std::max(sums_bytes(m, k, n), sums_bytes(n, k, m)));
}

int pact_fp8_linear_backward(const pact_matrix* dy, const pact_fp8* w_cols, const pact_fp8* x_cols,
                             const pact_matrix* dx, const pact_matrix* dw, uint32_t flags, void* workspace,
                             uint64_t workspace_bytes, void* stream) {
    if (dy == nullptr || w_cols == nullptr || x_cols == nullptr || dw == nullptr || (flags & ~PACT_FP8_ACCUMULATE) != 0) {
        return PACT_EINVAL;
    }
    int rc = PACT_OK;
    if ((rc = check(*dy)) != PACT_OK || (rc = check(*w_cols)) != PACT_OK || (rc = check(*x_cols)) != PACT_OK ||
        (dx != nullptr && (rc = check(*dx)) != PACT_OK) || (rc = check(*dw)) != PACT_OK) {
        return rc;
    }
    const uint64_t m = dy->rows, n = dy->cols, k = w_cols->rows;
    if (w_cols->cols != n || x_cols->rows != k || x_cols->cols != m || dw->rows != n || dw->cols != k ||
        dw->dtype != PACT_F32 || (dx != nullptr && (dx->rows != m || dx->cols != k))) {
        return PACT_EINVAL;
    }
    Spans spans;
    if (!add(spans, *dy, false) || !add(spans, *w_cols, false) || !add(spans, *x_cols, false) ||
        (dx != nullptr && !add(spans, *dx, true)) || !add(spans, *dw, true)) {
        return PACT_ERANGE;
    }
    if ((rc = check_workspace(spans, workspace, workspace_bytes)) != PACT_OK) return rc;
    if (spans.overlap()) return PACT_EOVERLAP;
    uint8_t* at = static_cast<uint8_t*>(workspace);
    const Held rows = held_at(at, m, n), cols = held_at(at + rows.bytes, n, m);
    const uint64_t held = rows.bytes + cols.bytes, need = held + std::max(sums_bytes(m, k, n), sums_bytes(n, k, m));
    if (workspace_bytes < need || (need > 0 && workspace == nullptr)) return PACT_EINVAL;
    uint8_t* const sums = at + held;  // the one product's, then the other's
    if (squares(*dy) * pact::kQuantizeThreads > kMaxItems || rows.x.ld >= kMaxFp8Row || cols.x.ld >= kMaxFp8Row) return PACT_ERANGE;
    if (m > 0 && n > 0) {
        const pact::Fp8 r = fp8(rows.x), c = fp8(cols.x);
        const hipError_t e =
            pact::launch_quantize(plain(*dy), dx != nullptr ? &r : nullptr, &c, false, static_cast<hipStream_t>(stream));
        if (e != hipSuccess) return pact::fail_hip(e);
    }
    if (dx != nullptr) {
        rc = product(rows.x, *w_cols, *dx, false, nullptr, sums, static_cast<hipStream_t>(stream));
        if (rc != PACT_OK) return rc;
    }
    return product(cols.x, *x_cols, *dw, (flags & PACT_FP8_ACCUMULATE) != 0, nullptr, sums,
                   static_cast<hipStream_t>(stream));
}

int pact_distill_loss(const pact_distill* d) { return distill(pact::Distill::Loss, d); }
int pact_distill_grad(const pact_distill* d) { return distill(pact::Distill::Grad, d); }
int pact_distill_step(const pact_distill* d) { return distill(pact::Distill::Step, d); }

}  // extern "C"
