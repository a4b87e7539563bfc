// The distillation loss from a teacher's top logits, and its gradient: softmax of a row of logits against a softmax of a few.  Bound by
// memory: a row is read once, held in registers, and its gradient written once.  4096 x 64000 bf16 219 us, 4.8 TB/s: a workgroup loads, finds
// the maximum, the sum, and stores, and two or three of them overlap on a compute unit.  Small ones are those steps' latencies: 32 x 1000 fp32 4.6 us.
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

// Largest of the values seen so far, of a thread.  Of bf16 two at a time: read as integers of 16 bits with a sign, numbers above zero are in
// order and numbers below it in reverse, so the largest integer is the largest number if that is not below zero, and the smallest is otherwise.
// (A NaN may be missed: the sum has it.)
template <int T> struct Largest;
template <> struct Largest<F32> {
    float most = -__builtin_inff();
    __device__ __forceinline__ void see(const Chunk<F32>& c) {
#pragma unroll
        for (int i = 0; i < 8; ++i) most = larger(most, c.a[i / 4][i % 4]);
    }
    __device__ __forceinline__ float get() const { return most; }
};
template <> struct Largest<BF16> {
    typedef short pair __attribute__((ext_vector_type(2)));
    pair high = {-32768, -32768}, low = {32767, 32767};
    __device__ __forceinline__ void see(const Chunk<BF16>& c) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const unsigned word = c.a[w];              // (of an element of a vector the cast takes the first)
            const pair v = __builtin_bit_cast(pair, word);
            high = __builtin_elementwise_max(high, v);
            low = __builtin_elementwise_min(low, v);
        }
    }
    __device__ __forceinline__ float get() const {
        const int h = max((int)high[0], (int)high[1]), l = min((int)low[0], (int)low[1]);
        return __uint_as_float((unsigned)(h >= 0 ? h : l) << 16);
    }
};

// The values less x, in their type.
__device__ __forceinline__ void subtract(Chunk<BF16>& c, float x) {
    v8bf b = __builtin_bit_cast(v8bf, c.a);
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = (__bf16)((float)b[i] - x);
    c.a = __builtin_bit_cast(v4u, b);
}
__device__ __forceinline__ void subtract(Chunk<F32>& c, float x) {
#pragma unroll
    for (int i = 0; i < 8; ++i) c.a[i / 4][i % 4] -= x;
}

typedef int v4i __attribute__((ext_vector_type(4)));
__host__ __device__ constexpr int whole_fours(int n) { return (n + 3) / 4 * 4; }

// A workgroup of THREADS walks rows; a thread holds NCH chunks of eight logits of one as they lie in memory (all of the row, whose chunks but
// each thread's last NCH - WHOLE are whole; AGAIN: rows that are longer are read again for every pass).  With c = log2(e) / T and b = most c, rounded,
// e^((z - most) / T) is 2^(z c - b) but for a factor that all share: one fused operation before the exponential, off by 3 |z c - b| 2^-24
// of itself, which no sum feels, for where that is large the term is small.  (Where b is so large that its rounding is, numbers that differ
// differ by thousands of it: the largest is subtracted from all of them first, and whatever their type makes of the differences,
// they are as good.)  What the loss subtracts is subtracted in 64 bits: the difference of two logarithms that nearly agree is what a
// student near its teacher has.
//
// Entries: each of the teacher's is read once into LDS with the student's logit of its class, before anything is written (dlogits
// may be the logits).  The gradient q T weight is written from the registers by whoever holds it; after a barrier the
// entries' classes are written again, less p: by the first of the entries that name a class, for all of them, so that nothing
// depends on an order.
template <int T, int THREADS, int NCH, int WHOLE, bool AGAIN, bool NARROW, int WAVES>
__global__ __launch_bounds__(THREADS) __attribute__((amdgpu_waves_per_eu(WAVES))) void k_distil(const Distil a) {
    constexpr int kWaves = THREADS / kWave, kWhole = WHOLE;
    __shared__ float wave_most[kWaves], wave_total[kWaves];
    __shared__ int wave_wrong[kWaves];
    extern __shared__ __attribute__((aligned(16))) float entries[];        // [4][top in whole fours]: the teacher's logit, the student's, p, the class (-1: none)
    float* const entry_t = entries;
    const int fours = whole_fours(a.top);
    float* const entry_z = entries + fours;
    float* const entry_p = entries + 2 * fours;
    int* const entry_class = (int*)(entries + 3 * fours);
    const int t = threadIdx.x, lane = t % kWave, wave = __builtin_amdgcn_readfirstlane(t / kWave);
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
                    const unsigned at = (unsigned)(j < kWhole ? col_of(turn, j) : min(col_of(turn, j), a.classes - kChunk)) * (unsigned)sizeof(Value);
                    const Value* from = (const Value*)((const uint8_t*)a.logits.p + row * a.logits.ld * (int)sizeof(Value) + at);
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
            for (int j = kWhole; j < NCH; ++j) settle<NARROW>(raw[j], a.classes - col_of(turn, j));
        };
        const auto write = [&](auto&& before, auto&& value) {
            for (int turn = 0; turn < turns; ++turn) {
                if constexpr (AGAIN) {
                    load(turn);
                    settle_all(turn);
                    before();
                }
#pragma unroll
                for (int j = 0; j < NCH; ++j) {
                    const int n = a.classes - col_of(turn, j);
                    float v[8];
                    values(raw[j], v);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = value(v[i]);
                    Value* to = (Value*)((uint8_t*)a.dlogits.p + row * a.dlogits.ld * (int)sizeof(Value)
                                         + (unsigned)col_of(turn, j) * (unsigned)sizeof(Value));
                    if (j < kWhole) store_values(to, kChunk, v);
                    else if (n > 0) store_values(to, n, v);
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
        // The entries are asked for ahead of the logits, and the student's logits of their classes behind them: what one waits for the other
        // has waited for.
        const auto entry = [&](int i, int& k, float& v) {
            i = min(i, a.top - 1);
            k = a.top_classes[row * a.top_classes_ld + i];
            const long long at = row * a.top_logits.ld + i;
            v = a.top_logits.kind == F32 ? ((const float*)a.top_logits.p)[at] : (float)((const __bf16*)a.top_logits.p)[at];
        };
        const auto student = [&](int k) { return (float)((const Value*)a.logits.p)[row * a.logits.ld + (k >= 0 && k < a.classes ? k : 0)]; };
        bool wrong = false;                                // a class that is none
        const auto keep = [&](int i, int k, float v, float z) {
            const bool there = k >= 0 && k < a.classes;
            wrong |= k >= a.classes;
            entry_class[i] = there ? k : -1;
            entry_t[i] = there ? v : -__builtin_inff();
            entry_z[i] = z;
        };
        int first_k;
        float first_v;
        entry(t, first_k, first_v);
        if constexpr (!AGAIN) load(0);
        const float first_z = student(first_k);
        if (t < a.top) keep(t, first_k, first_v, first_z);
        if (t < fours - a.top) {                           // (entries of none)
            entry_class[a.top + t] = -1;
            entry_p[a.top + t] = 0.0f;
        }
#pragma unroll 1
        for (int i = t + THREADS; i < a.top; i += THREADS) {
            int k;
            float v;
            entry(i, k, v);
            keep(i, k, v, student(k));
        }
        Largest<T> largest;
        for (int turn = 0; turn < turns; ++turn) {
            if constexpr (AGAIN) load(turn);
            settle_all(turn);
#pragma unroll
            for (int j = 0; j < NCH; ++j) largest.see(raw[j]);
        }
        float most = wave_max(largest.get());
        wrong = __any(wrong);
        if (lane == 0) {
            wave_most[wave] = most;
            wave_wrong[wave] = wrong;
        }
        __syncthreads();
        int any_wrong = wave_wrong[0];
        most = wave_most[0];
#pragma unroll
        for (int i = 1; i < kWaves; ++i) {
            most = larger(most, wave_most[i]);
            any_wrong |= wave_wrong[i];
        }
        // the teacher's softmax: every wave takes its sums for itself, and p of its entries for all
        float top_most = -__builtin_inff(), among = 0.0f;
        bool strange = any_wrong != 0;                     // (the largest leaves NaN out)
#pragma unroll 1
        for (int i = lane; i < a.top; i += kWave) {
            const float v = entry_t[i];
            top_most = larger(top_most, v);
            strange |= v != v;
        }
        top_most = wave_max(top_most);
        strange = __any(strange);
        const bool empty = !strange && top_most == -__builtin_inff();
#pragma unroll 1
        for (int i = lane; i < a.top; i += kWave) among += __builtin_amdgcn_exp2f((entry_t[i] - top_most) * c);
        among = wave_sum(among);
        if (strange) among = __builtin_nanf("");
#pragma unroll 1
        for (int i = t; i < a.top; i += THREADS) entry_p[i] = __builtin_amdgcn_exp2f((entry_t[i] - top_most) * c) / among;
        const bool far = fabsf(most * c) >= 0x1p20f;       // (the whole workgroup's)
        const auto come_near = [&]() {
            if (far) {
#pragma unroll
                for (int j = 0; j < NCH; ++j) subtract(raw[j], most);
            }
        };
        if constexpr (!AGAIN) come_near();
        const float shift = far ? 0.0f : most * c;
        float total = 0.0f;
        for (int turn = 0; turn < turns; ++turn) {
            if constexpr (AGAIN) {
                load(turn);
                settle_all(turn);
                come_near();
            }
#pragma unroll
            for (int j = 0; j < NCH; ++j) {
                float v[8];
                values(raw[j], v);
#pragma unroll
                for (int i = 0; i < 8; ++i) total += __builtin_amdgcn_exp2f(fmaf(v[i], c, -shift));
            }
        }
        total = wave_sum(total);
        if (lane == 0) wave_total[wave] = total;
        __syncthreads();
        total = wave_total[0];
#pragma unroll
        for (int i = 1; i < kWaves; ++i) total += wave_total[i];

        const float scale = weight * a.temperature;
        if (a.dlogits.p) {
            const float per = empty ? 0.0f : strange ? __builtin_nanf("") : scale / total;
            if (empty) write(come_near, [&](float) { return 0.0f; });
            else write(come_near, [&](float v) { return __builtin_amdgcn_exp2f(fmaf(v, c, -shift)) * per; });
        }
        // (total is of 2^(z c - shift), and shift is most c but for its rounding, if it is not 0 with the largest subtracted)
        const double rounding = far ? 0.0 : (double)shift - (double)most * (double)c;
        if (a.loss && wave == kWaves - 1) {
            double sum = 0.0;
            if (!empty) {
                const double apart = log((double)total) - log((double)among) + rounding * 0.69314718055994531, per = 1.0 / (double)a.temperature;
#pragma unroll 1
                for (int i = lane; i < a.top; i += kWave) {
                    const float p = entry_p[i];
                    // (an entry of p = 0 adds nothing, whatever the student's logit)
                    if (!(p == 0.0f))
                        sum += (double)p * ((((double)entry_t[i] - (double)top_most) - ((double)entry_z[i] - (double)most)) * per + apart);
                }
            }
            sum = wave_sum_double(sum);
            if (lane == 0) a.loss[row] = empty ? 0.0f : (float)((double)weight * (double)a.temperature * (double)a.temperature * sum);
        }
        if (a.dlogits.p) {
            // entry i of the thread's, until the stores of all waves have arrived
            const auto corrected = [&](int i, float& value) {
                const int k = entry_class[i];
                if (k < 0) return -1;
                float p = 0.0f;
                bool first = true;
#pragma unroll 2
                for (int e = 0; e < fours; e += 4) {
                    const v4i classes = *reinterpret_cast<const v4i*>(entry_class + e);
                    const v4f ps = *reinterpret_cast<const v4f*>(entry_p + e);
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const bool same = classes[u] == k;
                        p += same ? ps[u] : 0.0f;
                        first &= !(same && e + u < i);
                    }
                }
                const float x = far ? (entry_z[i] - most) * c : fmaf(entry_z[i], c, -shift);
                value = scale * (__builtin_amdgcn_exp2f(x) / total - p);
                return first ? k : -1;
            };
            float mine_value = 0.0f;
            const int mine_class = !empty && t < a.top ? corrected(t, mine_value) : -1;
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            Value* const to = (Value*)a.dlogits.p + row * a.dlogits.ld;
            if (mine_class >= 0) *as_global<Value>(to + mine_class) = (Value)mine_value;
            if (!empty) {
#pragma unroll 1
                for (int i = t + THREADS; i < a.top; i += THREADS) {
                    float value = 0.0f;
                    const int k = corrected(i, value);
                    if (k >= 0) *as_global<Value>(to + k) = (Value)value;
                }
            }
        }
        if (row + gridDim.x < a.rows) __syncthreads();     // the entries are the next row's
    }
}

// REST: how many of a thread's chunks the row's end may cut or leave out.  More than (NCH - REST) * 8 * THREADS classes, and at most NCH of that.
template <int T, int THREADS, int NCH, int REST = 1, bool AGAIN = false, bool NARROW = false>
hipError_t start(const Distil& a, hipStream_t s) {
    constexpr int kRegisters = NCH * (T == BF16 ? 4 : 8) + 60;          // what a thread needs, about: the compiler is held to it
    constexpr int kStep = THREADS > 256 ? THREADS / 256 : 1, kWavesWanted = std::max(1, std::min(8, 512 / kRegisters) / kStep) * kStep;
    k_distil<T, THREADS, NCH, NCH - REST, AGAIN, NARROW, kWavesWanted>
        <<<dim3((unsigned)std::min(a.rows, kMostRowsAGrid)), THREADS, 4 * whole_fours(a.top) * sizeof(float), s>>>(a);
    return hipGetLastError();
}

// A row by as few threads as hold it: what a thread needs beside its logits, some 50 registers, is the same for one chunk and for sixteen,
// so more rows are under way at once (us, this way | by four times the threads: 16384 x 8000 bf16 98 | 150, 512 x 12000 10 | 13, 1024 x 20000 fp32 35
// | 44; of 32 rows either is the call's time, 8).
template <int T>
hipError_t by_width(const Distil& a, hipStream_t s) {
    const int n = a.classes;
    if (n < kChunk) return start<T, 64, 1, 1, false, true>(a, s);
    if (n <= 512) return start<T, 64, 1>(a, s);
    if (n <= 1024) return start<T, 64, 2>(a, s);
    if (n <= 2048) return start<T, 64, 4, 2>(a, s);
    if (n <= 4096) return start<T, 128, 4, 2>(a, s);
    if (n <= 6144) return start<T, 256, 3>(a, s);
    if (n <= 8192) return start<T, 256, 4>(a, s);
    if (n <= 12288) return start<T, 256, 6, 2>(a, s);
    if (n <= 16384) return start<T, 256, 8, 2>(a, s);
    if (n <= 24576) return start<T, 512, 6, 2>(a, s);
    if (n <= 32768) return start<T, 512, 8, 2>(a, s);
    if constexpr (T == BF16) {
        if (n <= 40960) return start<T, 512, 10, 2>(a, s);
        if (n <= 49152) return start<T, 512, 12, 2>(a, s);
        if (n <= 57344) return start<T, 512, 14, 2>(a, s);
        if (n <= 65536) return start<T, 512, 16, 2>(a, s);
    } else {
        if (n <= 49152) return start<T, 1024, 6, 2>(a, s);
        if (n <= 65536) return start<T, 1024, 8, 2>(a, s);
    }
    return start<T, 1024, 4, 4, true>(a, s);
}

}  // namespace

hipError_t launch_distil(const Distil& a, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    return a.logits.kind == F32 ? by_width<F32>(a, s) : by_width<BF16>(a, s);
}

}  // namespace ops
}  // namespace lf
