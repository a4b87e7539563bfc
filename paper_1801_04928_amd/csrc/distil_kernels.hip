// The distillation loss from a teacher's top logits, and its gradient: softmax of a row of logits against a softmax of a few.  Bound by
// memory: a row is read once, held in registers, and its gradient written once.
#include "chunks.h"

#include <algorithm>
#include <type_traits>

namespace lf {
namespace ops {
namespace {

constexpr int kMostRowsAGrid = 1 << 20;   // a grid has fewer than 2^32 threads

__host__ __device__ constexpr int ceil_div(int a, int b) { return a / b + (a % b != 0); }

// The larger one; of a NaN and a number the number.  (fmaxf would first make quiet NaN of signalling ones: an instruction for each value.)
__device__ __forceinline__ float larger(float a, float b) {
    float r;
    asm("v_max_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}
__device__ __forceinline__ float wave_max(float v) {
    v = fmaxf(v, row_rotate<1>(v));
    v = fmaxf(v, row_rotate<2>(v));
    v = fmaxf(v, row_rotate<4>(v));
    v = fmaxf(v, row_rotate<8>(v));
    const auto of = [&](int lane) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane)); };
    return fmaxf(fmaxf(of(0), of(16)), fmaxf(of(32), of(48)));
}
__device__ __forceinline__ double wave_sum_double(double v) {
#pragma unroll
    for (int step = 32; step > 0; step /= 2) v += __shfl_xor(v, step);
    return v;
}

// Past the row's end the values become minus infinity, which adds nothing to either sum: n (0..8) of the chunk's are in the row.
template <bool NARROW>
__device__ __forceinline__ void settle(Chunk<BF16>& c, int n) {
    if (n >= kChunk) return;
    if constexpr (!NARROW) shift_down(c.a, kChunk - max(n, 0));
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if (2 * w >= n) c.a[w] = (c.a[w] & 0xffff0000u) | 0xff80u;
        if (2 * w + 1 >= n) c.a[w] = (c.a[w] & 0xffffu) | 0xff800000u;
    }
}
template <bool NARROW>
__device__ __forceinline__ void settle(Chunk<F32>& c, int n) {
    if (n >= kChunk) return;
    if constexpr (!NARROW) shift_down(c.a, kChunk - max(n, 0));
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i >= n) c.a[i / 4][i % 4] = -__builtin_inff();
}
// (what a register held is read again: the compiler would rather keep the eight values from pass to pass, in memory)
__device__ __forceinline__ void values(Chunk<BF16>& c, float (&v)[8]) {
    asm volatile("" : "+v"(c.a));
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        v[2 * w] = __uint_as_float(c.a[w] << 16);
        v[2 * w + 1] = __uint_as_float(c.a[w] & 0xffff0000u);
    }
}
__device__ __forceinline__ void values(Chunk<F32>& c, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = c.a[i / 4][i % 4];
}

// A workgroup of THREADS walks rows; a thread holds NCH chunks of eight logits of one as they lie in memory (all of the row; AGAIN: rows that are
// longer are read again for every pass).  e^((z - most) / T) is 2^((z - most) c) with c = log2(e) / T: off by 3 |(z - most) c| 2^-24 of itself,
// which no sum feels, for where that is large the term is small.  (z c - most c in one fused operation would be an instruction less,
// and nothing at all where logits are large: most c is rounded.)  What the loss subtracts is subtracted in 64 bits: the difference
// of two logarithms that nearly agree is what a student near its teacher has.
//
// Entries: each of the teacher's is read once into LDS with the student's logit of its class, before anything is written (dlogits
// may be the logits).  The gradient q T weight is written from the registers by whoever holds it; after a barrier the
// entries' classes are written again, less p: by the first of the entries that name a class, for all of them, so that nothing
// depends on an order.
template <int T, int THREADS, int NCH, bool AGAIN, bool NARROW, int BLOCKS>
__global__ __launch_bounds__(THREADS) __attribute__((amdgpu_waves_per_eu(BLOCKS * THREADS / 256 > 0 ? BLOCKS * THREADS / 256 : 1))) void k_distil(const Distil a) {
    constexpr int kWaves = THREADS / kWave;
    __shared__ float wave_most[kWaves], wave_total[kWaves];
    __shared__ float entry_t[kMostTop], entry_z[kMostTop];
    __shared__ int entry_class[kMostTop];
    const int t = threadIdx.x, lane = t % kWave, wave = t / kWave;
    const float c = 1.44269504088896341f / a.temperature;
    typedef typename Stored<T>::type Value;
    const int turns = AGAIN ? ceil_div(a.classes, kChunk * THREADS * NCH) : 1;

    for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const float weight = a.weight ? a.weight[row] : 1.0f;
        Chunk<T> raw[NCH];
        int mine = t;                                      // (what follows from it is not worth registers from row to row)
        asm volatile("" : "+v"(mine));
        const auto col_of = [&](int turn, int j) { return ((turn * NCH + j) * THREADS + mine) * kChunk; };
        const auto load = [&](int turn) {
#pragma unroll
            for (int j = 0; j < NCH; ++j) {
                if constexpr (NARROW) {
                    fetch_chunk<T, true>(raw[j], a.logits, row, col_of(turn, j), a.classes);
                } else {                                   // (a row's address is scalar, and 32 bits hold what is added to it)
                    const Value* from = (const Value*)((const uint8_t*)a.logits.p + row * a.logits.ld * (int)sizeof(Value)
                                                       + (unsigned)min(col_of(turn, j), a.classes - kChunk) * (unsigned)sizeof(Value));
                    if constexpr (T == F32) {
                        raw[j].a[0] = load_vector(from);
                        raw[j].a[1] = load_vector(from + 4);
                    } else {
                        raw[j].a = __builtin_bit_cast(v4u, load_vector(from));
                    }
                }
            }
        };
        const auto settle_all = [&](int turn) {
#pragma unroll
            for (int j = 0; j < NCH; ++j) settle<NARROW>(raw[j], a.classes - col_of(turn, j));
        };
        const auto write = [&](auto&& value) {
            for (int turn = 0; turn < turns; ++turn) {
                if constexpr (AGAIN) {
                    load(turn);
                    settle_all(turn);
                }
#pragma unroll
                for (int j = 0; j < NCH; ++j) {
                    const int n = a.classes - col_of(turn, j);
                    float v[8];
                    values(raw[j], v);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = value(v[i]);
                    if (n > 0)
                        store_values((Value*)((uint8_t*)a.dlogits.p + row * a.dlogits.ld * (int)sizeof(Value)
                                              + (unsigned)col_of(turn, j) * (unsigned)sizeof(Value)), n, v);
                }
            }
        };
        if (weight == 0.0f) {                              // (the whole workgroup's)
            if (t == 0 && a.loss) a.loss[row] = 0.0f;
            if (a.dlogits.p) {
                for (int col = t * kChunk; col < a.classes; col += THREADS * kChunk) {
                    const float zeros[8] = {};
                    store_values((Value*)a.dlogits.p + row * a.dlogits.ld + col, a.classes - col, zeros);
                }
            }
            continue;
        }
        if constexpr (!AGAIN) load(0);
        bool wrong = false;                                // a class that is none
#pragma unroll 1
        for (int i = t; i < a.top; i += THREADS) {
            const int k = a.top_classes[row * a.top_classes_ld + i];
            const long long at = row * a.top_logits.ld + i;
            const float v = a.top_logits.kind == F32 ? ((const float*)a.top_logits.p)[at] : (float)((const __bf16*)a.top_logits.p)[at];
            const bool there = k >= 0 && k < a.classes;
            wrong |= k >= a.classes;
            entry_class[i] = there ? k : -1;
            entry_t[i] = there ? v : -__builtin_inff();
            entry_z[i] = there ? (float)((const Value*)a.logits.p)[row * a.logits.ld + k] : 0.0f;
        }
        // the largest logit (NaN are looked at by the sum)
        float most = -__builtin_inff();
        for (int turn = 0; turn < turns; ++turn) {
            if constexpr (AGAIN) load(turn);
            settle_all(turn);
#pragma unroll
            for (int j = 0; j < NCH; ++j) {
                float v[8];
                values(raw[j], v);
#pragma unroll
                for (int i = 0; i < 8; ++i) most = larger(most, v[i]);
            }
        }
        most = wave_max(most);
        if (lane == 0) wave_most[wave] = most;
        wrong = __syncthreads_or(wrong);
        most = wave_most[0];
#pragma unroll
        for (int i = 1; i < kWaves; ++i) most = fmaxf(most, wave_most[i]);
        float total = 0.0f;
        for (int turn = 0; turn < turns; ++turn) {
            if constexpr (AGAIN) {
                load(turn);
                settle_all(turn);
            }
#pragma unroll
            for (int j = 0; j < NCH; ++j) {
                float v[8];
                values(raw[j], v);
#pragma unroll
                for (int i = 0; i < 8; ++i) total += __builtin_amdgcn_exp2f((v[i] - most) * c);
            }
        }
        total = wave_sum(total);
        if (lane == 0) wave_total[wave] = total;
        __syncthreads();
        total = wave_total[0];
#pragma unroll
        for (int i = 1; i < kWaves; ++i) total += wave_total[i];

        // the teacher's softmax: every wave takes it for itself
        float top_most = -__builtin_inff(), among = 0.0f;
#pragma unroll 1
        for (int i = lane; i < a.top; i += kWave) top_most = fmaxf(top_most, entry_t[i]);
        bool strange = false;                              // (fmaxf leaves NaN out)
#pragma unroll 1
        for (int i = lane; i < a.top; i += kWave) strange |= entry_t[i] != entry_t[i];
        top_most = wave_max(top_most);
        strange = __any(strange) || wrong;
        const bool empty = !strange && top_most == -__builtin_inff();
#pragma unroll 1
        for (int i = lane; i < a.top; i += kWave) among += __builtin_amdgcn_exp2f((entry_t[i] - top_most) * c);
        among = wave_sum(among);
        if (strange) among = __builtin_nanf("");
        const auto p_of = [&](int i) { return __builtin_amdgcn_exp2f((entry_t[i] - top_most) * c) / among; };
        const float scale = weight * a.temperature;
        if (a.dlogits.p) {
            const float per = empty ? 0.0f : strange ? __builtin_nanf("") : scale / total;
            if (empty) write([&](float) { return 0.0f; });
            else write([&](float v) { return __builtin_amdgcn_exp2f((v - most) * c) * per; });
            // (the stores of all waves have arrived before any of an entry's is made)
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            if (!empty) {
#pragma unroll 1
                for (int i = t; i < a.top; i += THREADS) {
                    const int k = entry_class[i];
                    if (k < 0) continue;
                    float p = 0.0f;
                    bool first = true;
#pragma unroll 2
                    for (int e = 0; e < a.top; ++e) {
                        if (entry_class[e] != k) continue;
                        if (e < i) first = false;
                        p += p_of(e);
                    }
                    if (!first) continue;
                    const float q = __builtin_amdgcn_exp2f((entry_z[i] - most) * c) / total;
                    *as_global<Value>((Value*)a.dlogits.p + row * a.dlogits.ld + k) = (Value)(scale * (q - p));
                }
            }
        }
        // (last, when the row's logits need no registers any more)
        if (a.loss && wave == 0) {
            double sum = 0.0;
            if (!empty) {
                const double apart = log((double)total) - log((double)among), per = 1.0 / (double)a.temperature;
#pragma unroll 1
                for (int i = lane; i < a.top; i += kWave) {
                    const float p = p_of(i);
                    // (an entry of p = 0 adds nothing, whatever the student's logit)
                    if (!(p == 0.0f))
                        sum += (double)p * ((((double)entry_t[i] - (double)top_most) - ((double)entry_z[i] - (double)most)) * per + apart);
                }
            }
            sum = wave_sum_double(sum);
            if (lane == 0) a.loss[row] = empty ? 0.0f : (float)((double)weight * (double)a.temperature * (double)a.temperature * sum);
        }
        __syncthreads();                                   // the entries are the next row's
    }
}

template <int T, int THREADS, int NCH, bool AGAIN, bool NARROW, int BLOCKS>
hipError_t start(const Distil& a, hipStream_t s) {
    k_distil<T, THREADS, NCH, AGAIN, NARROW, BLOCKS><<<dim3((unsigned)std::min(a.rows, kMostRowsAGrid)), THREADS, 0, s>>>(a);
    return hipGetLastError();
}

// BLOCKS: workgroups that a compute unit's registers are to hold: one reads a row while another is worked on.
template <int T>
hipError_t by_width(const Distil& a, hipStream_t s) {
    constexpr int kTwo = T == BF16 ? 2 : 1;
    if (a.classes < kChunk) return start<T, 64, 1, false, true, 8>(a, s);
    if (a.classes <= 512) return start<T, 64, 1, false, false, 8>(a, s);
    if (a.classes <= 2048) return start<T, 256, 1, false, false, 4>(a, s);
    if (a.classes <= 4096) return start<T, 256, 2, false, false, 4>(a, s);
    if (a.classes <= 8192) return start<T, 512, 2, false, false, 2>(a, s);
    if (a.classes <= 16384) return start<T, 512, 4, false, false, 2>(a, s);
    if (a.classes <= 32768) return start<T, 1024, 4, false, false, kTwo>(a, s);
    if (a.classes <= 65536) return start<T, 1024, 8, false, false, kTwo>(a, s);
    if (T == BF16 && a.classes <= 131072) return start<T, 1024, T == BF16 ? 16 : 8, false, false, 1>(a, s);
    return start<T, 1024, 4, true, false, kTwo>(a, s);
}

}  // namespace

hipError_t launch_distil(const Distil& a, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    return a.logits.kind == F32 ? by_width<F32>(a, s) : by_width<BF16>(a, s);
}

}  // namespace ops
}  // namespace lf
