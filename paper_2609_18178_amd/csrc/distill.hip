// distill.hip -- gfx950 kernels of the distillation loss against a teacher's
// top logits: a workgroup per row of logits.
#include "operators.h"

namespace pact {
namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint32_t bits_of(float x) { return __builtin_bit_cast(uint32_t, x); }
__device__ __forceinline__ float float_of(uint32_t x) { return __builtin_bit_cast(float, x); }

constexpr float kLog2e = 1.44269504088896341f;
constexpr float kNan = __builtin_nanf(""), kInf = __builtin_inff();

// The elements of a 16-byte vector: eight of bf16, four of binary32.
template <typename T>
struct Elems;
template <>
struct Elems<uint16_t> {
    static constexpr int kCount = 8;
    static __device__ __forceinline__ float get(const u32x4& v, int i) {
        const uint32_t w = v[i >> 1];
        return float_of(i & 1 ? w & 0xffff0000u : w << 16);
    }
    static __device__ __forceinline__ float widen(uint16_t x) { return float_of((uint32_t)x << 16); }
    static __device__ __forceinline__ uint16_t narrow(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
    static __device__ __forceinline__ u32x4 pack(const float (&x)[8]) {
        u32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = narrow(x[2 * i]) | (uint32_t)narrow(x[2 * i + 1]) << 16;
        return v;
    }
    static constexpr uint16_t kLowest = 0xff80u;  // -infinity
    static constexpr uint32_t kLowestWord = 0xff80ff80u;
};
template <>
struct Elems<float> {
    static constexpr int kCount = 4;
    static __device__ __forceinline__ float get(const u32x4& v, int i) { return float_of(v[i]); }
    static __device__ __forceinline__ float widen(float x) { return x; }
    static __device__ __forceinline__ float narrow(float x) { return x; }
    static __device__ __forceinline__ u32x4 pack(const float (&x)[4]) {
        return u32x4{bits_of(x[0]), bits_of(x[1]), bits_of(x[2]), bits_of(x[3])};
    }
    static constexpr float kLowest = -kInf;
    static constexpr uint32_t kLowestWord = 0xff800000u;
};

template <typename Op>
__device__ __forceinline__ float over_wave(float x, Op op) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x = op(x, __shfl_xor(x, d));
    return x;
}

struct Max {
    __device__ __forceinline__ float operator()(float a, float b) const { return __builtin_fmaxf(a, b); }
};
struct Sum {
    __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};

// One value per workgroup, the same in every thread: over the lanes of each wave, then over the
// waves in order.
template <int Threads, typename Op>
__device__ __forceinline__ float over_block(float x, Op op, float* scratch) {
    x = over_wave(x, op);
    __syncthreads();  // the last use of scratch is over
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = x;
    __syncthreads();
    x = scratch[0];
#pragma unroll
    for (int w = 1; w < Threads / 64; ++w) x = op(x, scratch[w]);
    return x;
}

// A row of T: the 16-byte vectors that lie in it whole, and the few elements before and behind them,
// one for each of as many threads.
template <typename T>
struct Row {
    static constexpr int kCount = Elems<T>::kCount;
    T* first;  // element 0
    uint32_t lead, vectors, vocab;

    __device__ __forceinline__ Row(const char* at, uint32_t n) {
        first = reinterpret_cast<T*>(const_cast<char*>(at));
        lead = min((0u - (uint32_t)(reinterpret_cast<uintptr_t>(at) / sizeof(T))) % kCount, n);
        vectors = (n - lead) / kCount;
        vocab = n;
    }
    __device__ __forceinline__ uint32_t at(uint32_t i) const { return lead + i * kCount; }
    // The element beside the vectors that is thread t's, or `vocab`.
    __device__ __forceinline__ uint32_t beside(uint32_t t) const {
        return t < lead ? t : min(t - lead, vocab) < vocab - at(vectors) ? at(vectors) + t - lead : vocab;
    }
    // Vector i; behind the last -infinity, which counts for nothing.
    __device__ __forceinline__ u32x4 load(uint32_t i) const {
        const uint32_t low = Elems<T>::kLowestWord;
        u32x4 v = {low, low, low, low};
        if (i < vectors) v = *reinterpret_cast<const u32x4*>(first + at(i));
        return v;
    }
    // (As it lies in memory: widened in the branch it would be waited for there.)
    __device__ __forceinline__ T load_beside(uint32_t t) const {
        T x = Elems<T>::kLowest;
        const uint32_t i = beside(t);
        if (i < vocab) x = first[i];
        return x;
    }
};

// x in the places of elements from.. of a row, wherever that is: past the caches (the gradient of 1024 x 65536
// in bf16 55.0 -> 45.0 us, of 512 x 32768 16.3 -> 12.0).
typedef u32x4 u32x4_at2 __attribute__((aligned(2)));
template <typename T>
__device__ __forceinline__ void store_vector(T* first, uint32_t from, const float (&x)[Elems<T>::kCount]) {
    __builtin_nontemporal_store(Elems<T>::pack(x), reinterpret_cast<u32x4_at2*>(first + from));
}

// 2^((z - from) * to_log2): the difference first, so that logits of any size (masks of the
// type's lowest number among them) cancel exactly.
__device__ __forceinline__ float power(float z, float from, float to_log2) {
    return __builtin_amdgcn_exp2f((z - from) * to_log2);
}

// Largest logit, and the sum of exp((z - most) / T) relative to it.
struct Softmax {
    float most, sum;
};

// The same relative to the largest of several, of all lanes of a wave.
__device__ __forceinline__ Softmax over_wave(Softmax x, float to_log2) {
    const float most = over_wave(x.most, Max());
    const float from = most == -kInf ? 0.0f : most;
    // (a lane that saw no number has a sum of zero, or NaN if it saw one of those)
    const float sum = x.most == -kInf ? x.sum : x.sum * power(x.most, from, to_log2);
    return {most, over_wave(sum, Sum())};
}

// One more vector's logits.
template <typename T>
__device__ __forceinline__ void add_vector(Softmax& x, const u32x4& v, float to_log2) {
    float most = x.most;
#pragma unroll
    for (int j = 0; j < Elems<T>::kCount; ++j) most = __builtin_fmaxf(most, Elems<T>::get(v, j));
    const float from = most == -kInf ? 0.0f : most;
    float sum = x.most == -kInf ? x.sum : x.sum * power(x.most, from, to_log2);
#pragma unroll
    for (int j = 0; j < Elems<T>::kCount; ++j) sum += power(Elems<T>::get(v, j), from, to_log2);
    x = {most, sum};
}

// A log-sum-exp up to this size says what a probability is to 2^-18 of itself; where it is
// larger (or not finite) the gradient reads the row twice instead of going by it.
constexpr float kMostLse = 64.0f;

// Teacher logits up to this number are one wave's.
constexpr uint32_t kWaveTop = 64;

// Loss, gradient or both of one row: a workgroup's.
//
// The row is read once where it fits: Held vectors a thread stay in registers (Held == 0: it
// is read again). Each thread sums its powers of 2 relative to its own largest logit, so that one
// exchange through LDS gives the softmax; the teacher's, of up to 64 logits, is the first wave's
// alone, and comes with the same exchange. The gradient is written for all entries as if the teacher
// listed none, and the few that it lists once more behind a barrier.
//
// With p the teacher's probabilities, q = exp(z / T - lse) the student's and w the row's weight: loss
// w sum p (log p - log q), gradient w (q - p) / T. Bound by the reading and writing of logits that come
// from memory: bf16, 64 listed: loss of 4096 x 32768 in 53 us (5.1 TB/s), gradient of 2047 x 32003 in 52
// (5.0), both of 512 x 32768 in 15 (4.4). A few rows are bound by one workgroup's own rate: one row of 32003
// takes 5.0, 6.3 and 7.9 us, one of 131072 10.5, 13.9 and 22 (64 rows of those 11, 15 and 23).
template <typename T, Distill Kind, int Threads, int Held>
__global__ __launch_bounds__(Threads, Held <= 4 ? 8 : 4) void distill_kernel(const DistillArgs d) {
    constexpr int kCount = Elems<T>::kCount, kWaves = Threads / 64;
    constexpr bool kLoss = Kind != Distill::Grad, kGrad = Kind != Distill::Loss;
    __shared__ float scratch[kWaves];
    __shared__ Softmax part[kWaves];
    __shared__ float prob[kMaxTop], logit[kMaxTop], excess[kMaxTop];  // excess: over the largest, divided by T
    __shared__ int32_t place[kMaxTop];
    __shared__ float total_of_teacher;  // NaN: an index outside of the vocabulary; 0: nothing is listed
    __shared__ uint32_t twice;          // some entry is listed twice
    const uint32_t r = blockIdx.x, t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const Row<T> row(d.logits + (uint64_t)r * d.ld_logits * sizeof(T), d.vocab);
    // A slot of the teacher's, as it lies in memory; what it lists.
    struct Slot {
        int32_t lo, hi;  // of its index
        uint32_t value;
    };
    struct Listed {
        float x;       // the teacher's; -infinity: nothing
        T logit;       // the student's
        int32_t place;
        bool outside;  // of the vocabulary
    };
    auto read = [&](uint32_t j) {
        const uint64_t it = (uint64_t)r * d.ld_top_index + j, lt = (uint64_t)r * d.ld_top_logits + j;
        const int32_t* index = reinterpret_cast<const int32_t*>(d.top_index);
        Slot s;
        s.lo = index[d.wide_index ? 2 * it : it];
        s.hi = d.wide_index ? index[2 * it + 1] : 0;
        s.value = d.top_dtype == kF32 ? reinterpret_cast<const uint32_t*>(d.top_logits)[lt]
                                      : (uint32_t) reinterpret_cast<const uint16_t*>(d.top_logits)[lt];
        return s;
    };
    auto listed = [&](const Slot& s) {
        const int64_t i = d.wide_index ? (int64_t)((uint64_t)(uint32_t)s.hi << 32 | (uint32_t)s.lo) : (int64_t)s.lo;
        const float x = float_of(d.top_dtype == kF32 ? s.value : s.value << 16);
        const bool some = i >= 0 && !(x == -kInf);
        Listed l;
        l.outside = some && i >= (int64_t)d.vocab;
        l.place = some && !l.outside ? (int32_t)i : -1;
        l.logit = T(0);
        if (l.place >= 0) l.logit = row.first[l.place];
        l.x = some ? x : -kInf;
        return l;
    };
    // (Loads are under way in the order of their use: the teacher's slots, the row, the student's logits in them.)
    Slot first_slot = {0, 0, 0};
    if (d.top <= kWaveTop && t < d.top) first_slot = read(t);
    const float weight = d.row_weight ? d.row_weight[r] : 1.0f;
    auto nothing = [&]() {
        if (kLoss && t == 0) {
            d.loss[r] = 0.0f;
            if (d.lse) d.lse[r] = 0.0f;
        }
        if constexpr (kGrad) {
            const Row<T> out(d.grad + (uint64_t)r * d.ld_grad * sizeof(T), d.vocab);
            const float zeros[kCount] = {};
            for (uint32_t i = t; i < out.vectors; i += Threads) store_vector<T>(out.first, out.at(i), zeros);
            if (out.beside(t) < d.vocab) out.first[out.beside(t)] = Elems<T>::narrow(0.0f);
        }
    };
    if (weight == 0.0f) return nothing();

    u32x4 held[Held > 0 ? Held : 1];
    if constexpr (Held > 0) {
#pragma unroll
        for (int k = 0; k < Held; ++k) held[k] = row.load(t + k * Threads);
    }
    const T beside = row.load_beside(t);

    // the teacher's softmax over its listed slots: as the student's, the difference first, so that logits near the
    // type's largest or lowest number stay finite at any temperature
    if (t == 0) twice = 0;
    // (NaN counts as the largest: the row is NaN)
    auto size = [](float x) { return x == x ? x : kInf; };
    Listed first = {-kInf, T(0), -1, false};
    if (d.top <= kWaveTop) {
        if (wave == 0) {
            if (lane < d.top) first = listed(first_slot);
            const float x = first.x;
            const float most = over_wave(size(x), Max());
            const float over = (x - most) * d.inv_temperature;
            const float e = x == -kInf ? 0.0f : __expf(over);
            float total = over_wave(e, Sum());
            if (__builtin_amdgcn_ballot_w64(first.outside) != 0) total = kNan;
            if (lane < d.top) {
                prob[lane] = x == -kInf ? 0.0f : e / total;
                excess[lane] = over;
                place[lane] = first.place;
            }
            if (lane == 0) total_of_teacher = total;
        }
    } else {
        float most = -kInf;
        bool wrong = false;
        for (uint32_t j = t; j < d.top; j += Threads) {
            const Listed l = listed(read(j));
            wrong |= l.outside;
            excess[j] = l.x;
            place[j] = l.place;
            logit[j] = Elems<T>::widen(l.logit);
            most = __builtin_fmaxf(most, size(l.x));
        }
        most = over_block<Threads>(most, Max(), scratch);
        float total = 0.0f;
        for (uint32_t j = t; j < d.top; j += Threads) {
            const float x = excess[j], over = (x - most) * d.inv_temperature, e = x == -kInf ? 0.0f : __expf(over);
            prob[j] = e;
            excess[j] = over;
            total += e;
        }
        total = over_block<Threads>(total, Sum(), scratch);
        if (over_block<Threads>(wrong ? 1.0f : 0.0f, Max(), scratch) != 0.0f) total = kNan;
        for (uint32_t j = t; j < d.top; j += Threads) prob[j] = prob[j] == 0.0f ? 0.0f : prob[j] / total;
        if (t == 0) total_of_teacher = total;
    }

    // the student's: q = 2^((z - from) * to_log2 - less)
    const float held_beside = Elems<T>::widen(beside);
    auto own = [&]() {
        Softmax x = {held_beside, 0.0f};
        if constexpr (Held > 0) {
#pragma unroll
            for (int k = 0; k < Held; ++k) {
#pragma unroll
                for (int j = 0; j < kCount; ++j) x.most = __builtin_fmaxf(x.most, Elems<T>::get(held[k], j));
                __builtin_amdgcn_sched_barrier(0);  // (else all of the row is widened at once, in registers)
            }
            const float from = x.most == -kInf ? 0.0f : x.most;
            x.sum = power(held_beside, from, d.to_log2);
#pragma unroll
            for (int k = 0; k < Held; ++k) {
#pragma unroll
                for (int j = 0; j < kCount; ++j) x.sum += power(Elems<T>::get(held[k], j), from, d.to_log2);
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            x.sum = held_beside == -kInf ? 0.0f : power(held_beside, held_beside, d.to_log2);
            for (uint32_t i = t; i < row.vectors; i += Threads) add_vector<T>(x, row.load(i), d.to_log2);
        }
        x = over_wave(x, d.to_log2);
        if (lane == 0) part[wave] = x;
    };
    auto joined = [&]() {
        Softmax x = over_wave(lane < kWaves ? part[lane] : Softmax{-kInf, 0.0f}, d.to_log2);
        if (x.most == -kInf) x.most = 0.0f;
        return x;
    };
    float from = 0.0f, less, log_sum = 0.0f;
    float lse = 0.0f;
    bool by_reading = kLoss;
    if constexpr (!kLoss) {
        lse = d.lse[r];
        by_reading = !(__builtin_fabsf(lse) <= kMostLse);
    }
    if (by_reading) own();
    if (d.top <= kWaveTop && t < d.top) logit[t] = Elems<T>::widen(first.logit);
    __syncthreads();
    const float total = total_of_teacher;
    if (total == 0.0f) return nothing();
    if (by_reading) {
        const Softmax x = joined();
        from = x.most;
        less = __builtin_amdgcn_logf(x.sum);
        log_sum = __logf(x.sum);
    } else {
        less = lse * kLog2e;
    }
    const float spoilt = total == total ? 0.0f : kNan;  // (an infinite or NaN teacher logit, or an index outside)
    if constexpr (kLoss) {
        const float log_total = __logf(total);
        float loss = 0.0f;
        for (uint32_t j = t; j < d.top; j += Threads) {
            const float p = prob[j];
            if (!(p == 0.0f)) {
                const float z = logit[j];
                const float log_q = z == -kInf ? -kInf : (z - from) * d.inv_temperature - log_sum;
                loss += p * (excess[j] - log_total - log_q);
            }
        }
        loss = d.top <= kWaveTop ? over_wave(loss, Sum()) : over_block<Threads>(loss, Sum(), scratch);
        if (t == 0) {
            d.loss[r] = (loss + spoilt) * weight;
            if (d.lse) d.lse[r] = from * d.inv_temperature + log_sum;
        }
    }
    if constexpr (kGrad) {
        // is an entry listed twice? each wave compares every slot with its share of the others
        bool again = false;
        for (uint32_t j = lane; j < d.top; j += 64) {
            const int32_t i = place[j];
            for (uint32_t k = wave; k < d.top; k += kWaves) again |= i >= 0 && k != j && place[k] == i;
        }
        if (__builtin_amdgcn_ballot_w64(again) != 0 && lane == 0) twice = 1;

        T* const grad = reinterpret_cast<T*>(d.grad + (uint64_t)r * d.ld_grad * sizeof(T));
        const float by = weight * d.inv_temperature;
        less += spoilt;
        auto student = [&](float z) {
            const float q = __builtin_amdgcn_exp2f((z - from) * d.to_log2 - less);
            return z == -kInf ? 0.0f : q;
        };
        auto emit = [&](uint32_t i, const u32x4& v) {
            float g[kCount];
#pragma unroll
            for (int j = 0; j < kCount; ++j) g[j] = student(Elems<T>::get(v, j)) * by;
            store_vector<T>(grad, row.at(i), g);
        };
        if constexpr (Held > 0) {
            uint32_t from_t = t;
            // (the vectors' numbers are formed again where, kept from the loads on, some are spilled: 512 x 32768 18.2 -> 16.3 us)
            if constexpr (kLoss && sizeof(T) == 2) asm("" : "+v"(from_t));
#pragma unroll
            for (int k = 0; k < Held; ++k) {
                const uint32_t i = from_t + k * Threads;
                if (i < row.vectors) emit(i, held[k]);
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            for (uint32_t i = t; i < row.vectors; i += Threads) emit(i, row.load(i));
        }
        if (row.beside(t) < d.vocab) grad[row.beside(t)] = Elems<T>::narrow(student(held_beside) * by);
        __syncthreads();
        for (uint32_t j = t; j < d.top; j += Threads) {
            const int32_t i = place[j];
            if (i < 0) continue;
            float p = prob[j];
            if (twice != 0) {
                p = 0.0f;
                for (uint32_t k = 0; k < d.top; ++k) {
                    if (place[k] == i) p += prob[k];
                }
            }
            grad[i] = Elems<T>::narrow((student(logit[j]) - p) * by);
        }
    }
}

template <typename T, Distill Kind>
void distill(const DistillArgs& d, hipStream_t stream) {
    // The threads, and the vectors a thread, that hold a row. Rows of more than 4096 vectors (64 KB) are read
    // twice instead, the second time mostly from the caches, by all but the step on binary32 logits:
    // more in registers costs waves, and bf16 widens to more. us held / read twice: 2048 x 50257 bf16
    // loss 52 / 40, gradient 108 / 90, step 121 / 117; 1024 x 65536 binary32 loss 48 / 44, step 98 / 151.
    constexpr bool kLong = Kind == Distill::Step && sizeof(T) == 4;
    const uint32_t vectors = d.vocab / Elems<T>::kCount;
    if (vectors <= 256) {
        distill_kernel<T, Kind, 256, 1><<<d.rows, 256, 0, stream>>>(d);
    } else if (vectors <= 256 * 4) {
        distill_kernel<T, Kind, 256, 4><<<d.rows, 256, 0, stream>>>(d);
    } else if (vectors <= 512 * 4) {
        distill_kernel<T, Kind, 512, 4><<<d.rows, 512, 0, stream>>>(d);
    } else if (vectors <= 1024 * 4) {
        distill_kernel<T, Kind, 1024, 4><<<d.rows, 1024, 0, stream>>>(d);
    } else {
        if constexpr (kLong) {
            if (vectors <= 1024 * 8) {
                distill_kernel<T, Kind, 1024, 8><<<d.rows, 1024, 0, stream>>>(d);
                return;
            }
            if (vectors <= 1024 * 16) {
                distill_kernel<T, Kind, 1024, 16><<<d.rows, 1024, 0, stream>>>(d);
                return;
            }
        }
        distill_kernel<T, Kind, 1024, 0><<<d.rows, 1024, 0, stream>>>(d);
    }
}

template <typename T>
void distill(Distill kind, const DistillArgs& d, hipStream_t stream) {
    switch (kind) {
        case Distill::Loss: distill<T, Distill::Loss>(d, stream); break;
        case Distill::Grad: distill<T, Distill::Grad>(d, stream); break;
        case Distill::Step: distill<T, Distill::Step>(d, stream); break;
    }
}

}  // namespace

hipError_t launch_distill(Distill kind, const DistillArgs& d, hipStream_t stream) {
    if (d.dtype == kF32) {
        distill<float>(kind, d, stream);
    } else {
        distill<uint16_t>(kind, d, stream);
    }
    return hipGetLastError();
}

}  // namespace pact
