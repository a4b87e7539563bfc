// Matrices into 8 bits with blocks of 128, as they lie and transposed, and back; with the gradient before an activation, which a
// backward pass makes on the way, and its sums over rows.  All of it is bound by memory: every value is read once.
#include "activation.h"
#include "chunks.h"

#include <algorithm>

namespace lf {
namespace ops {
namespace {

constexpr int kThreads = 256;
constexpr int NONE_KIND = -1;                             // no z
constexpr int kHigh = 8;                                   // rows of a thread, below each other
constexpr int kAcross = kBlock / kChunk;                   // threads along a row
static_assert(kAcross * kBlock / kHigh == kThreads, "the threads hold 128 x 128 values");

__host__ __device__ constexpr int ceil_div(int a, int b) { return a / b + (a % b != 0); }

template <int ACT>
__device__ __forceinline__ void times_slope(float (&d)[8], const float (&z)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) d[i] *= slope(ACT, z[i]);
}
__device__ __forceinline__ void times_slope(int act, float (&d)[8], const float (&z)[8]) {
    switch (act) {
        case SIGMOID: times_slope<SIGMOID>(d, z); break;
        case RELU: times_slope<RELU>(d, z); break;
        case SILU: times_slope<SILU>(d, z); break;
        case GELU: times_slope<GELU>(d, z); break;
        default: break;
    }
}

__device__ __forceinline__ unsigned finite_bits(float v) { return __float_as_uint(finite_magnitude(v)); }
// v / 2^(byte - 127) as the conversion takes it where a group holds what is not finite, which becomes NaN, or has the largest scale, of
// which it holds at most 240 (256 would be no finite number).
__device__ __forceinline__ float scaled(float v, int byte) {
    const float a = v * scale_power(254 - byte), most = byte == kLargestScale ? 240.0f : 448.0f;
    return fabsf(v) < __builtin_inff() ? fminf(fmaxf(a, -most), most) : __builtin_nanf("");
}

// A workgroup keeps a block of 128 x 128 values in registers, thread t eight rows (8 (t / 16) and on) of eight columns (8 (t % 16) and
// on).  A row's group is 16 lanes' chunks, so its scale is a maximum over a row of lanes; a column's is one over the thread's
// eight rows, then over the 16 threads below each other, through LDS, which also turns the transposed codes: 128 bytes of a
// column, whose 8-byte pieces lie at place p ^ (column / 8 % 16), so that the 16 threads of a row write to different banks.
// TILES: one scale for all.  Bound by memory.
template <int T, int Z, bool TILES>
__global__ __launch_bounds__(kThreads) void k_block_save(const BlockSave a, int blocks_x) {
    __shared__ unsigned tops[kThreads / kAcross][kBlock];
    __shared__ float sums[kThreads / kAcross][kBlock];
    __shared__ uint8_t column_byte[kBlock];
    __shared__ __attribute__((aligned(16))) uint8_t turned[kBlock * kBlock];
    const int t = threadIdx.x, across = t % kAcross, down = t / kAcross;
    const int bx = (int)(blockIdx.x % (unsigned)blocks_x), by = (int)(blockIdx.x / (unsigned)blocks_x);
    const int c0 = bx * kBlock, r0 = by * kBlock;
    const int col = c0 + across * kChunk, n = min(max(a.cols - col, 0), kChunk), row = r0 + down * kHigh;

    float v[kHigh][8];
#pragma unroll
    for (int i = 0; i < kHigh; ++i) load_chunk<T>(a.x, row + i, col, row + i < a.rows ? n : 0, v[i]);
    if (Z != NONE_KIND) {
#pragma unroll
        for (int i = 0; i < kHigh; ++i) {
            float z[8];
            load_chunk<Z == NONE_KIND ? T : Z>(a.z, row + i, col, row + i < a.rows ? n : 0, z);
            times_slope(a.act, v[i], z);
        }
    }
    // largest magnitudes: of a row's group in `own`, of the thread's rows in each column; a value that is not finite shows in them
    unsigned own[kHigh], down_top[8] = {};
#pragma unroll
    for (int i = 0; i < kHigh; ++i) {
        unsigned m = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const unsigned b = __float_as_uint(v[i][j]) & 0x7FFFFFFFu;
            m = max(m, b);
            down_top[j] = max(down_top[j], b);
        }
        own[i] = m;
    }
    bool odd = false;
#pragma unroll
    for (int i = 0; i < kHigh; ++i) odd |= own[i] >= 0x7F800000u;
    if (odd) {                                             // what is not finite sets no scale
#pragma unroll
        for (int j = 0; j < 8; ++j) down_top[j] = 0;
#pragma unroll
        for (int i = 0; i < kHigh; ++i) {
            own[i] = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const unsigned b = finite_bits(v[i][j]);
                own[i] = max(own[i], b);
                down_top[j] = max(down_top[j], b);
            }
        }
    }
    if (a.partial) {
        float s[8] = {};
#pragma unroll
        for (int i = 0; i < kHigh; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j] += v[i][j];
#pragma unroll
        for (int j = 0; j < 8; ++j) sums[down][across * kChunk + j] = s[j];
    }
    if (TILES || a.out_t.p) {
#pragma unroll
        for (int j = 0; j < 8; ++j) tops[down][across * kChunk + j] = down_top[j];
    }
    // (every value finite and no group of the largest scale: nothing to look at value by value)
    unsigned most = 0;
#pragma unroll
    for (int i = 0; i < kHigh; ++i) most = max(most, own[i]);
    const bool rare = __syncthreads_or(odd || scale_byte(__uint_as_float(most)) >= kLargestScale);
    int tile_byte = 0;
    if constexpr (TILES) {
        unsigned m = 0;
        for (int i = 0; i < kThreads / kAcross; ++i) m = max(m, tops[i][t % kBlock]);
        m = sixteen_max(m);
        __syncthreads();
        if (t % 16 == 0 && t < kBlock) tops[0][t / 16] = m;
        __syncthreads();
        for (int i = 0; i < kBlock / 16; ++i) m = max(m, tops[0][i]);
        tile_byte = scale_byte(__uint_as_float(m));
        if (t == 0) {
            if (a.out.p) *as_global<uint8_t>(a.out.scales + (long long)by * a.out.scale_ld + bx) = (uint8_t)tile_byte;
            if (a.out_t.p) *as_global<uint8_t>(a.out_t.scales + (long long)bx * a.out_t.scale_ld + by) = (uint8_t)tile_byte;
        }
    } else if (a.out_t.p) {
        if (t < kBlock) {
            unsigned m = 0;
#pragma unroll
            for (int i = 0; i < kThreads / kAcross; ++i) m = max(m, tops[i][t]);
            const int byte = scale_byte(__uint_as_float(m));
            column_byte[t] = (uint8_t)byte;
            if (c0 + t < a.cols) *as_global<uint8_t>(a.out_t.scales + (long long)(c0 + t) * a.out_t.scale_ld + by) = (uint8_t)byte;
        }
    }
    if (a.partial && t >= kThreads - kBlock) {
        const int c = t - (kThreads - kBlock);
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < kThreads / kAcross; ++i) s += sums[i][c];
        if (c0 + c < a.cols) a.partial[(size_t)by * a.cols + c0 + c] = s;
    }
    if (a.out.p) {
#pragma unroll
        for (int i = 0; i < kHigh; ++i) {
            const int byte = TILES ? tile_byte : scale_byte(__uint_as_float(sixteen_max(own[i])));
            const float inverse = scale_power(254 - byte);
            float s[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j] = v[i][j] * inverse;
            if (rare) {
#pragma unroll
                for (int j = 0; j < 8; ++j) s[j] = scaled(v[i][j], byte);
            }
            if (row + i < a.rows) {
                *as_global<v2u>((uint8_t*)a.out.p + (long long)(row + i) * a.out.ld + col) = convert_eight(s);
                if (!TILES && across == 0) *as_global<uint8_t>(a.out.scales + (long long)(row + i) * a.out.scale_ld + bx) = (uint8_t)byte;
            }
        }
    }
    if (!a.out_t.p) return;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int c = across * kChunk + j, byte = TILES ? tile_byte : column_byte[c];
        const float inverse = scale_power(254 - byte);
        float s[8];
#pragma unroll
        for (int i = 0; i < kHigh; ++i) s[i] = v[i][j] * inverse;
        if (rare) {
#pragma unroll
            for (int i = 0; i < kHigh; ++i) s[i] = scaled(v[i][j], byte);
        }
        *reinterpret_cast<v2u*>(turned + c * kBlock + ((down ^ across) * 8)) = convert_eight(s);
    }
    __syncthreads();
    for (int id = t; id < kBlock * kBlock / 16; id += kThreads) {
        const int c = id / 8, p = id % 8, turn = c / kChunk;
        if (c0 + c >= a.cols) break;
        const v2u lo = *reinterpret_cast<const v2u*>(turned + c * kBlock + ((2 * p) ^ turn) * 8);
        const v2u hi = *reinterpret_cast<const v2u*>(turned + c * kBlock + ((2 * p + 1) ^ turn) * 8);
        *as_global<v4u>((uint8_t*)a.out_t.p + (long long)(c0 + c) * a.out_t.ld + r0 + p * 16) = v4u{lo[0], lo[1], hi[0], hi[1]};
    }
}

// A thread takes a chunk of eight.
template <int FROM, int TO>
__global__ __launch_bounds__(kThreads) void k_block_load(int rows, int cols, const Mat from, const Mat to) {
    const long long id = (long long)blockIdx.x * kThreads + threadIdx.x;
    const int chunks = ceil_div(cols, kChunk), col = (int)(id % chunks) * kChunk, n = min(cols - col, kChunk);
    const long long row = id / chunks;
    if (row >= rows) return;
    float v[8];
    load_chunk<FROM>(from, row, col, n, v);
    store_chunk<TO>(to, row, col, n, v, true);
}

template <int T, int Z>
void save(const BlockSave& a, hipStream_t s) {
    const int blocks_x = ceil_div(a.cols, kBlock);
    const dim3 grid((unsigned)((long long)blocks_x * ceil_div(a.rows, kBlock)));
    const int type = a.out.p ? a.out.kind : a.out_t.kind;
    if (type == E4M3_TILES) k_block_save<T, Z, true><<<grid, kThreads, 0, s>>>(a, blocks_x);
    else k_block_save<T, Z, false><<<grid, kThreads, 0, s>>>(a, blocks_x);
}
template <int FROM, int TO>
hipError_t load(int rows, int cols, const Mat& in, const Mat& out, hipStream_t s) {
    const long long blocks = ((long long)rows * ceil_div(cols, kChunk) + kThreads - 1) / kThreads;
    // (a grid has fewer than 2^32 threads: rows are taken in parts)
    const long long most = (1ll << 32) / kThreads - 1;
    if (blocks <= most) {
        k_block_load<FROM, TO><<<dim3((unsigned)blocks), kThreads, 0, s>>>(rows, cols, in, out);
        return hipGetLastError();
    }
    const int part = rows / 2 / kBlock * kBlock;
    const auto rest = [&](const Mat& m, int scale_rows) {
        Mat r = m;
        const int bytes = m.kind == F32 ? 4 : m.kind == BF16 ? 2 : 1;
        r.p = (uint8_t*)m.p + (long long)part * m.ld * bytes;
        if (m.scales) r.scales = m.scales + (long long)scale_rows * m.scale_ld;
        return r;
    };
    const hipError_t e = load<FROM, TO>(part, cols, in, out, s);
    return e != hipSuccess ? e : load<FROM, TO>(rows - part, cols, rest(in, in.kind == E4M3_TILES ? part / kBlock : part), rest(out, 0), s);
}

}  // namespace

int block_partials(int rows) { return ceil_div(rows, kBlock); }

hipError_t launch_block_save(const BlockSave& a, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    if (a.x.kind == F32) {
        if (a.act == NONE) save<F32, NONE_KIND>(a, s);
        else if (a.z.kind == E4M3_128) save<F32, E4M3_128>(a, s);
        else save<F32, F32>(a, s);
    } else {
        if (a.act == NONE) save<BF16, NONE_KIND>(a, s);
        else if (a.z.kind == E4M3_128) save<BF16, E4M3_128>(a, s);
        else save<BF16, BF16>(a, s);
    }
    return hipGetLastError();
}

hipError_t launch_block_load(int rows, int cols, const Mat& in, const Mat& out, hipStream_t s) {
    if (rows == 0) return hipSuccess;
    if (in.kind == E4M3_TILES) return out.kind == F32 ? load<E4M3_TILES, F32>(rows, cols, in, out, s) : load<E4M3_TILES, BF16>(rows, cols, in, out, s);
    return out.kind == F32 ? load<E4M3_128, F32>(rows, cols, in, out, s) : load<E4M3_128, BF16>(rows, cols, in, out, s);
}

}  // namespace ops
}  // namespace lf
