// Matrices into 8 bits with blocks of 128, as they lie and transposed, and back; with the gradient before an activation, which a
// backward pass makes on the way, and its sums over rows.  All of it is bound by memory: every value is read once.  4096 x 8192 bf16 both ways 31 us
// (4.4 TB/s; 34 next to other kernels), with gelu's slope and the sums 53 (half of it arithmetic); with a branch around each load 36 and 60.  Weights
// of 8192 x 8192 bf16 both ways, tiles, 56 us (4.8 TB/s).  Back: 4096 x 8192 to bf16 20.5 us (4.9 TB/s), of tiles 8192 x 8192 37.6 (5.4).
#include "activation.h"
#include "chunks.h"

#include <algorithm>
#include <type_traits>

namespace lf {
namespace ops {
namespace {

constexpr int NONE_KIND = -1;                              // no z
constexpr int kAcross = kBlock / kChunk;                   // threads along a row
constexpr int kLoadThreads = 256;

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

// v / 2^(byte - 127) as the conversion takes it where a group holds what is not finite, which becomes NaN, or has the largest scale, of
// which it holds at most 240 (256 would be no finite number).
__device__ __forceinline__ float scaled(float v, int byte) {
    const float a = v * scale_power(254 - byte), most = byte == kLargestScale ? 240.0f : 448.0f;
    return fabsf(v) < __builtin_inff() ? fminf(fmaxf(a, -most), most) : __builtin_nanf("");
}

// m or the larger of |a| and |b|; a NaN stays one.
__device__ __forceinline__ float largest_of(float m, float a, float b) {
    float r;
    asm("v_maximum3_f32 %0, %1, |%2|, |%3|" : "=v"(r) : "v"(m), "v"(a), "v"(b));
    return r;
}

// A workgroup keeps a block of 128 x 128 values in registers, thread t HIGH rows (HIGH (t / 16) and on) of eight columns (8 (t % 16) and on).  A
// row's group is 16 lanes' chunks, so its scale is a maximum over a row of lanes; a column's is one over the thread's rows, then over
// the threads below each other, through LDS, which also turns the transposed codes: 128 bytes of a column in pieces of HIGH, which
// lie where the threads of a row write to different banks.  TILES: one scale for all.
// HIGH = 8, 256 threads, where there are blocks enough: every value costs some thirty instructions, half of them the slope's, so the
// time is memory's where four blocks a compute unit overlap what they load and what they compute.  HIGH = 4, 512 threads, for a few blocks.
// NARROW: of fewer than eight columns.
template <int T, int Z, bool TILES, int HIGH, bool NARROW = false>
__global__ __launch_bounds__(kAcross * kBlock / HIGH) __attribute__((amdgpu_waves_per_eu(4))) void k_block_save(const BlockSave a, int blocks_x) {
    constexpr int kDown = kBlock / HIGH, kThreads = kAcross * kDown;
    typedef typename std::conditional<HIGH == 8, v2u, unsigned>::type Piece;
    __shared__ float tops[kDown][kBlock];
    __shared__ float sums[kDown][kBlock];
    __shared__ uint8_t column_byte[kBlock];
    __shared__ __attribute__((aligned(16))) uint8_t turned[kBlock * kBlock];
    const int t = threadIdx.x, across = t % kAcross, down = t / kAcross;
    const int bx = (int)(blockIdx.x % (unsigned)blocks_x), by = (int)(blockIdx.x / (unsigned)blocks_x);
    const int c0 = bx * kBlock, r0 = by * kBlock;
    const int col = c0 + across * kChunk, n = min(max(a.cols - col, 0), kChunk), row = r0 + down * HIGH;

    float v[HIGH][8];
    const auto there = [&](int i) { return row + i < a.rows ? n : 0; };
    if (row < a.rows && n > 0) {       // (all loads are under way at once: past the last row it is loaded again)
        Chunk<T> raw[HIGH];
#pragma unroll
        for (int i = 0; i < HIGH; ++i) fetch_chunk<T, NARROW>(raw[i], a.x, min(row + i, a.rows - 1), col, a.cols);
        if constexpr (Z != NONE_KIND) {
            constexpr int kSome = T == F32 && HIGH == 8 ? 4 : HIGH;          // (what registers hold)
#pragma unroll
            for (int from = 0; from < HIGH; from += kSome) {
                Chunk<Z> z_raw[kSome];
#pragma unroll
                for (int i = 0; i < kSome; ++i) fetch_chunk<Z, NARROW>(z_raw[i], a.z, min(row + from + i, a.rows - 1), col, a.cols);
#pragma unroll
                for (int i = 0; i < kSome; ++i) {
                    float z[8];
                    take_chunk<T, NARROW>(raw[from + i], there(from + i), v[from + i]);
                    take_chunk<Z, NARROW>(z_raw[i], there(from + i), z);
                    times_slope(a.act, v[from + i], z);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < HIGH; ++i) take_chunk<T, NARROW>(raw[i], there(i), v[i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < HIGH; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = 0.0f;
    }
    // largest magnitudes: of a row's group in `own`, of the thread's rows in each column; a value that is not finite shows in them
    float own[HIGH], down_top[8];
#pragma unroll
    for (int i = 0; i < HIGH; ++i) {
        own[i] = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; j += 2) own[i] = largest_of(own[i], v[i][j], v[i][j + 1]);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        down_top[j] = 0.0f;
#pragma unroll
        for (int i = 0; i < HIGH; i += 2) down_top[j] = largest_of(down_top[j], v[i][j], v[i + 1][j]);
    }
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < HIGH; i += 2) most = largest_of(most, own[i], own[i + 1]);
    const bool odd = !(most < __builtin_inff());
    if (odd) {                                             // what is not finite sets no scale
        most = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) down_top[j] = 0.0f;
#pragma unroll
        for (int i = 0; i < HIGH; ++i) {
            own[i] = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float b = finite_magnitude(v[i][j]);
                own[i] = fmaxf(own[i], b);
                down_top[j] = fmaxf(down_top[j], b);
            }
            most = fmaxf(most, own[i]);
        }
    }
    if (a.partial) {
        float s[8] = {};
#pragma unroll
        for (int i = 0; i < HIGH; ++i)
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
    const bool rare = __syncthreads_or(odd || scale_byte(most) >= kLargestScale);
    int tile_byte = 0;
    if constexpr (TILES) {
        float m = 0.0f;
        for (int i = 0; i < kDown; ++i) m = fmaxf(m, tops[i][t % kBlock]);
        m = __uint_as_float(sixteen_max(__float_as_uint(m)));
        __syncthreads();
        if (t % 16 == 0 && t < kBlock) tops[0][t / 16] = m;
        __syncthreads();
        for (int i = 0; i < kBlock / 16; ++i) m = fmaxf(m, tops[0][i]);
        tile_byte = scale_byte(m);
        if (t == 0) {
            if (a.out.p) *as_global<uint8_t>(a.out.scales + (long long)by * a.out.scale_ld + bx) = (uint8_t)tile_byte;
            if (a.out_t.p) *as_global<uint8_t>(a.out_t.scales + (long long)bx * a.out_t.scale_ld + by) = (uint8_t)tile_byte;
        }
    } else if (a.out_t.p) {
        if (t < kBlock) {
            float m = 0.0f;
#pragma unroll
            for (int i = 0; i < kDown; ++i) m = fmaxf(m, tops[i][t]);
            const int byte = scale_byte(m);
            column_byte[t] = (uint8_t)byte;
            if (c0 + t < a.cols) *as_global<uint8_t>(a.out_t.scales + (long long)(c0 + t) * a.out_t.scale_ld + by) = (uint8_t)byte;
        }
    }
    if (a.partial && t >= kThreads - kBlock) {
        const int c = t - (kThreads - kBlock);
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < kDown; ++i) s += sums[i][c];
        if (c0 + c < a.cols) a.partial[(size_t)by * a.cols + c0 + c] = s;
    }
    if (a.out.p) {
#pragma unroll
        for (int i = 0; i < HIGH; ++i) {
            const int byte = TILES ? tile_byte : scale_byte(__uint_as_float(sixteen_max(__float_as_uint(own[i]))));
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
    // piece `down` of column c is at place down ^ across of 16, or of 32 at down ^ (4 across % 32): 16 bytes that belong together stay so
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int c = across * kChunk + j, byte = TILES ? tile_byte : column_byte[c];
        const float inverse = scale_power(254 - byte);
        float s[8] = {};
#pragma unroll
        for (int i = 0; i < HIGH; ++i) s[i] = v[i][j] * inverse;
        if (rare) {
#pragma unroll
            for (int i = 0; i < HIGH; ++i) s[i] = scaled(v[i][j], byte);
        }
        const v2u codes = convert_eight(s);
        Piece* const at = reinterpret_cast<Piece*>(turned + c * kBlock) + (HIGH == 8 ? down ^ across : down ^ (4 * across & 31));
        if constexpr (HIGH == 8) *at = codes;
        else *at = codes[0];
    }
    __syncthreads();
    for (int id = t; id < kBlock * kBlock / 16; id += kThreads) {
        const int c = id / 8, p = id % 8, turn = c / kChunk;
        if (c0 + c >= a.cols) break;
        v4u out;
        if constexpr (HIGH == 8) {
            const v2u lo = *reinterpret_cast<const v2u*>(turned + c * kBlock + ((2 * p) ^ turn) * 8);
            const v2u hi = *reinterpret_cast<const v2u*>(turned + c * kBlock + ((2 * p + 1) ^ turn) * 8);
            out = v4u{lo[0], lo[1], hi[0], hi[1]};
        } else {
            out = *reinterpret_cast<const v4u*>(turned + c * kBlock + (p ^ (turn & 7)) * 16);
        }
        *as_global<v4u>((uint8_t*)a.out_t.p + (long long)(c0 + c) * a.out_t.ld + r0 + p * 16) = out;
    }
}

// A thread takes a chunk of eight.
template <int FROM, int TO>
__global__ __launch_bounds__(kLoadThreads) void k_block_load(int rows, int cols, const Mat from, const Mat to) {
    const long long id = (long long)blockIdx.x * kLoadThreads + threadIdx.x;
    const int chunks = ceil_div(cols, kChunk), col = (int)(id % chunks) * kChunk, n = min(cols - col, kChunk);
    const long long row = id / chunks;
    if (row >= rows) return;
    float v[8];
    load_chunk<FROM>(from, row, col, n, v);
    store_chunk<TO>(to, row, col, n, v, true);
}

constexpr long long kFewBlocks = 512;
template <int T, int Z>
void save(const BlockSave& a, hipStream_t s) {
    const int blocks_x = ceil_div(a.cols, kBlock);
    const long long blocks = (long long)blocks_x * ceil_div(a.rows, kBlock);
    const dim3 grid((unsigned)blocks);
    const int type = a.out.p ? a.out.kind : a.out_t.kind;
    constexpr int kMany = kAcross * kBlock / 8, kFew = kAcross * kBlock / 4;
    // (tiles are weights': nothing is multiplied by a slope on the way to them)
    const auto start = [&](auto tiles) {
        if (a.cols < kChunk) k_block_save<T, Z, tiles(), 4, true><<<grid, kFew, 0, s>>>(a, blocks_x);
        else if (blocks <= kFewBlocks) k_block_save<T, Z, tiles(), 4><<<grid, kFew, 0, s>>>(a, blocks_x);
        else k_block_save<T, Z, tiles(), 8><<<grid, kMany, 0, s>>>(a, blocks_x);
    };
    if constexpr (Z == NONE_KIND) {
        if (type == E4M3_TILES) return start(std::true_type());
    }
    start(std::false_type());
}
template <int FROM, int TO>
hipError_t load(int rows, int cols, const Mat& in, const Mat& out, hipStream_t s) {
    const long long blocks = ((long long)rows * ceil_div(cols, kChunk) + kLoadThreads - 1) / kLoadThreads;
    // (a grid has fewer than 2^32 threads: rows are taken in parts)
    const long long most = (1ll << 32) / kLoadThreads - 1;
    if (blocks <= most) {
        k_block_load<FROM, TO><<<dim3((unsigned)blocks), kLoadThreads, 0, s>>>(rows, cols, in, out);
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
