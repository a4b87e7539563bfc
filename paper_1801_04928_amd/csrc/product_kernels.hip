// The matrix product of residual blocks,  C[m][n] = sum_q P(m,q) Q(n,q)  with fp32 sums, in its three uses:
//   forward   P = x  (contiguous along q)          Q = w (contiguous along q)          C = z -> bias, activation, residual
//   dx        P = dz (contiguous along q)          Q = w (contiguous along its own n)
//   dw        P = dz (contiguous along its own m)  Q = x (contiguous along its own n)
// Operands are fp32 or bf16; x may be in 8 bits, whose values are bf16 numbers: they are made when a tile is laid into LDS,
// and the matrix instructions see no difference.
#include "activation.h"
#include "chunks.h"

#include <algorithm>

namespace lf {
namespace ops {
namespace {

constexpr int kRowBytes = 128;            // of a tile, along q: 64 bf16 or 32 fp32
constexpr int kPiece = 8;                 // elements a thread moves at a time

__host__ __device__ constexpr int ceil_div(int a, int b) { return a / b + (a % b != 0); }
__host__ __device__ constexpr int whole_groups(int cols) { return ceil_div(cols, kGroup) * kGroup; }

struct Args {
    Mat P, Q;
    int M, N, K;
    int tiles_m, tiles_n;
    int splits, k_tiles_per_split;
    float* raw;                           // [splits][M][N] if splits > 1
    Finish f;
};

// Elements of a piece on their way from memory to LDS.
template <int KIND> struct Raw;
template <> struct Raw<F32> { v4f a, b; };
template <> struct Raw<BF16> { v8bf a; };
template <> struct Raw<E4M3> { v2u a; int byte; };

// One operand's tile of I rows by BK: loaded into registers, laid into LDS as numbers of the products' type C.
// LDS of a tile contiguous along q: [i][q], rows of eight 16-byte pieces, piece p of row i at place p ^ (i & 7): the rows that a
// matrix operand takes its pieces from then lie in different banks.  Contiguous along i: [q][i]; bf16 is read there by
// transposing loads, eight rows of 64 bytes at a time (q, q+1, q+2, q+3 and eight further), whose 64-byte segments
// change places the same way.
template <class C, int KIND, bool ALONG, int I, int THREADS>
struct Tile {
    static constexpr int BK = kRowBytes / (int)sizeof(C);
    static constexpr int kElems = I * BK;
    static constexpr int kPieces = I * BK / kPiece / THREADS;
    static constexpr int kElemBytes = KIND == F32 ? 4 : KIND == BF16 ? 2 : 1;
    static_assert(kPieces * THREADS * kPiece == I * BK, "whole pieces for every thread");

    Raw<KIND> r[kPieces];

    // Place of this thread's piece u in the tile: i and q.
    static __device__ __forceinline__ void place(int u, int& i, int& q) {
        const int id = threadIdx.x + u * THREADS;
        if constexpr (ALONG) { i = id % (I / kPiece) * kPiece; q = id / (I / kPiece); }
        else { q = id % (BK / kPiece) * kPiece; i = id / (BK / kPiece); }
    }

    // I_all x q_all: the operand.  Rows (or pieces) past i's end are read from the last ones: they only reach results that are
    // not there.  Past the contraction's end everything is zero.
    __device__ __forceinline__ void load(const Mat& m, int i0, int I_all, int q0, int q_all) {
        const bool whole = q0 + BK <= q_all;
        const bool inside = !ALONG || KIND == E4M3 || i0 + I <= I_all || I_all % kPiece == 0;
        if (whole && inside) fast(m, i0, I_all, q0);
        else edge(m, i0, I_all, q0, q_all);
    }
    __device__ __forceinline__ void fast(const Mat& m, int i0, int I_all, int q0) {
        const uint8_t* base = (const uint8_t*)m.p + (ALONG ? (long long)q0 * m.ld + i0 : (long long)i0 * m.ld + q0) * kElemBytes;
#pragma unroll
        for (int u = 0; u < kPieces; ++u) {
            int i, q;
            place(u, i, q);
            const int last = KIND == E4M3 && ALONG ? whole_groups(I_all) : I_all;
            i = ALONG ? min(i, (last - 1) / kPiece * kPiece - i0) : min(i, I_all - 1 - i0);
            const unsigned off = (unsigned)((ALONG ? (long long)q * m.ld + i : (long long)i * m.ld + q) * kElemBytes);
            fetch(u, base + off);
            if constexpr (KIND == E4M3) fetch_scale(u, m, i0, i, q0, q);
        }
    }
    __device__ __forceinline__ void fetch(int u, const uint8_t* p) {
        if constexpr (KIND == F32) {
            r[u].a = *as_global<const any_v4f>(p);
            r[u].b = *as_global<const any_v4f>(p + 16);
        } else if constexpr (KIND == BF16) {
            r[u].a = *as_global<const any_v8bf>(p);
        } else {
            r[u].a = *as_global<const v2u>(p);
        }
    }
    __device__ __forceinline__ void fetch_scale(int u, const Mat& m, int i0, int i, int q0, int q) {
        const long long row = ALONG ? q0 + q : i0 + i;
        const int col = ALONG ? i0 + i : q0 + q;
        if constexpr (KIND == E4M3) r[u].byte = *as_global<const uint8_t>(m.scales + row * m.scale_ld + col / kGroup);
    }
    __device__ __forceinline__ void edge(const Mat& m, int i0, int I_all, int q0, int q_all) {
#pragma unroll
        for (int u = 0; u < kPieces; ++u) {
            int i, q;
            place(u, i, q);
            // n values of the piece are there
            const int n = min(kPiece, ALONG ? (q0 + q < q_all ? I_all - i0 - i : 0) : (i0 + i < I_all ? q_all - q0 - q : 0));
            const long long at = ALONG ? (long long)(q0 + q) * m.ld + i0 + i : (long long)(i0 + i) * m.ld + q0 + q;
            float v[8];
            if constexpr (KIND == E4M3) {
                v2u w = v2u{0u, 0u};
                int byte = 127;
                if (n > 0) {
                    w = *as_global<const v2u>((const uint8_t*)m.p + at);
                    byte = *as_global<const uint8_t>(m.scales + (ALONG ? (long long)(q0 + q) : (long long)(i0 + i)) * m.scale_ld +
                                                     (ALONG ? i0 + i : q0 + q) / kGroup);
                    const unsigned long long keep = n >= 8 ? ~0ull : (1ull << (8 * n)) - 1;
                    w[0] &= (unsigned)keep;
                    w[1] &= (unsigned)(keep >> 32);
                }
                r[u].a = w;
                r[u].byte = byte;
            } else if constexpr (KIND == BF16) {
                load_values((const __bf16*)m.p + at, n, v);
#pragma unroll
                for (int e = 0; e < 8; ++e) r[u].a[e] = (__bf16)v[e];
            } else {
                load_values((const float*)m.p + at, n, v);
                r[u].a = v4f{v[0], v[1], v[2], v[3]};
                r[u].b = v4f{v[4], v[5], v[6], v[7]};
            }
        }
    }

    // Where 16-byte pieces go.
    static __device__ __forceinline__ int at_along_q(int i, int piece) {
        return i * BK + ((piece ^ (i & 7)) * (16 / (int)sizeof(C)));
    }
    static __device__ __forceinline__ int at_along_i(int q, int i) {
        if constexpr (sizeof(C) == 2) {
            constexpr int kSegments = I / 32;
            const int turn = ((q & 3) | ((q >> 1) & 4)) & (kSegments < 8 ? kSegments - 1 : 7);
            return q * I + (((i >> 5) ^ turn) << 5) + (i & 31);
        } else {
            return q * I + i;
        }
    }
    __device__ __forceinline__ void store(C* s) const {
#pragma unroll
        for (int u = 0; u < kPieces; ++u) {
            int i, q;
            place(u, i, q);
            if constexpr (sizeof(C) == 2) {
                v8bf v;
                if constexpr (KIND == BF16) {
                    v = r[u].a;
                } else {
                    const float scale = scale_value(r[u].byte);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const v2bf a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)r[u].a[h], scale, false);
                        const v2bf b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)r[u].a[h], scale, true);
                        v[4 * h] = a[0]; v[4 * h + 1] = a[1]; v[4 * h + 2] = b[0]; v[4 * h + 3] = b[1];
                    }
                }
                *reinterpret_cast<v8bf*>(s + (ALONG ? at_along_i(q, i) : at_along_q(i, q / 8))) = v;
            } else {
                v4f a, b;
                if constexpr (KIND == F32) {
                    a = r[u].a;
                    b = r[u].b;
                } else {
                    float v[8];
                    eight_values(r[u].a, scale_value(r[u].byte), v);
                    a = v4f{v[0], v[1], v[2], v[3]};
                    b = v4f{v[4], v[5], v[6], v[7]};
                }
                if constexpr (ALONG) {
                    *reinterpret_cast<v4f*>(s + at_along_i(q, i)) = a;
                    *reinterpret_cast<v4f*>(s + at_along_i(q, i + 4)) = b;
                } else {
                    *reinterpret_cast<v4f*>(s + at_along_q(i, q / 4)) = a;
                    *reinterpret_cast<v4f*>(s + at_along_q(i, q / 4 + 1)) = b;
                }
            }
        }
    }

    // Operand of one 32-row tile for step `step` of BK: bf16, 16 q a step: lane holds q = 16 step + 8 (lane / 32) .. +7 of row
    // lane % 32.  fp32, 8 q a step: q = 8 step + 4 (lane / 32) .. +3, one matrix instruction for each.
    typedef typename std::conditional<sizeof(C) == 2, v8bf, v4f>::type Operand;
    static constexpr int kSteps = BK / (sizeof(C) == 2 ? 16 : 8);
    static __device__ __forceinline__ Operand operand(const C* s, int i_base, int step) {
        const int lane = threadIdx.x & 63, r32 = lane & 31, half = lane >> 5;
        if constexpr (sizeof(C) == 2) {
            if constexpr (ALONG) {
                // transposing loads: of 16 lanes, lane s supplies the address of four consecutive i of row s / 4 and receives the
                // four rows' values of one i
                typedef short v4s __attribute__((ext_vector_type(4)));
                typedef short v8s __attribute__((ext_vector_type(8)));
                typedef __attribute__((address_space(3))) v4s* lds_v4s_ptr;
                const int s16 = lane & 15;
                const int q = 16 * step + 8 * half + (s16 >> 2), i = i_base + 16 * ((lane >> 4) & 1) + 4 * (s16 & 3);
                const C* at = s + at_along_i(q, i);
                const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_ptr)(at));
                const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_ptr)(at + 4 * I));
                return __builtin_bit_cast(v8bf, (v8s){lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
            } else {
                return *reinterpret_cast<const v8bf*>(s + at_along_q(i_base + r32, 2 * step + half));
            }
        } else {
            if constexpr (ALONG) {
                v4f v;
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = s[at_along_i(8 * step + 4 * half + j, i_base + r32)];
                return v;
            } else {
                return *reinterpret_cast<const v4f*>(s + at_along_q(i_base + r32, 2 * step + half));
            }
        }
    }
};

// ---- what happens to finished sums -------------------------------------------------------------------------------------
__device__ __forceinline__ void load_any(const Mat& m, long long row, int col, int n, float (&v)[8]) {
    if (m.kind == F32) load_chunk<F32>(m, row, col, n, v);
    else load_chunk<BF16>(m, row, col, n, v);
}
__device__ __forceinline__ void store_any(const Mat& m, long long row, int col, int n, const float (&v)[8], bool live) {
    if (m.kind == E4M3) store_chunk<E4M3>(m, row, col, n, v, live);
    else if (m.kind == F32) store_chunk<F32>(m, row, col, n, v, live);
    else store_chunk<BF16>(m, row, col, n, v, live);
}
// Eight columns of row m from n on (n a multiple of 8; the four lanes of a quad hold the four chunks of a group of 32).
__device__ __forceinline__ void finish_chunk(const Finish& f, int M, int N, int m, int n, float (&v)[8]) {
    const int there = m < M ? min(N - n, kChunk) : 0;
    const bool live = m < M && n < whole_groups(N);
    if (f.bias && there > 0) {
        float b[8];
        load_values(f.bias + n, there, b);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += b[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < there ? v[i] : 0.0f;
    if (f.z.p) store_any(f.z, m, n, there, v, live);
    if (f.act != NONE) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = activate(f.act, v[i]);
    }
    if (f.residual.p) {
        float r[8];
        load_any(f.residual, m, n, there, r);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += r[i];
    }
    if (f.y.kind == E4M3) {      // sigmoid(0) is not 0
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < there ? v[i] : 0.0f;
    }
    store_any(f.y, m, n, there, v, live);
}

// ================================================================================================
// tiles of BM x BN, WM x WN waves
// ================================================================================================
template <class C, int PK, int QK, bool P_ALONG, bool Q_ALONG, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void k_product(const Args g) {
    constexpr int kThreads = 64 * WM * WN;
    typedef Tile<C, PK, P_ALONG, BM, kThreads> TP;
    typedef Tile<C, QK, Q_ALONG, BN, kThreads> TQ;
    constexpr int BK = TP::BK, MT = BM / WM / 32, NT = BN / WN / 32;
    constexpr int kStageLd = NT * 32 + 4;
    constexpr int kLds = 2 * (TP::kElems + TQ::kElems) * (int)sizeof(C);
    static_assert(WM * WN * 16 * kStageLd * 4 <= kLds, "the epilogue's staging fits");
    __shared__ __attribute__((aligned(16))) uint8_t lds[kLds];

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int tile = blockIdx.x % (unsigned)(g.tiles_m * g.tiles_n), split = blockIdx.x / (unsigned)(g.tiles_m * g.tiles_n);
    const int m0 = tile % g.tiles_m * BM, n0 = tile / g.tiles_m * BN;
    const int wm = wave / WN * (MT * 32), wn = wave % WN * (NT * 32);
    const int k_tiles = ceil_div(g.K, BK);
    const int kt0 = split * g.k_tiles_per_split, kt1 = min(k_tiles, kt0 + g.k_tiles_per_split);

    v16f acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;

    TP tp;
    TQ tq;
    auto request = [&](int kt) {
        tp.load(g.P, m0, g.M, kt * BK, g.K);
        tq.load(g.Q, n0, g.N, kt * BK, g.K);
    };
    if (kt0 < kt1) {
        request(kt0);
        for (int kt = kt0; kt < kt1; ++kt) {
            C* const sp = reinterpret_cast<C*>(lds) + ((kt - kt0) & 1) * (TP::kElems + TQ::kElems);
            C* const sq = sp + TP::kElems;
            tp.store(sp);
            tq.store(sq);
            __syncthreads();         // and: everybody has read what the next store overwrites
            if (kt + 1 < kt1) request(kt + 1);
#pragma unroll
            for (int step = 0; step < TP::kSteps; ++step) {
                typename TP::Operand a[MT], q[NT];
#pragma unroll
                for (int i = 0; i < MT; ++i) a[i] = TP::operand(sp, wm + 32 * i, step);
#pragma unroll
                for (int j = 0; j < NT; ++j) q[j] = TQ::operand(sq, wn + 32 * j, step);
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < NT; ++j) {
                        if constexpr (sizeof(C) == 2) {
                            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i], q[j], acc[i][j], 0, 0, 0);
                        } else {
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i][e], q[j][e], acc[i][j], 0, 0, 0);
                        }
                    }
            }
        }
    }
    __syncthreads();

    // Accumulator element e of lane (r32, half) of tile (i, j) is C[.. 32 i + 8 (e / 4) + 4 half + e % 4][.. 32 j + r32].  16 rows at
    // a time turn through LDS of the wave's own, so that a lane holds eight consecutive columns.
    float* stage = reinterpret_cast<float*>(lds) + wave * 16 * kStageLd;
    const int r32 = lane & 31, half = lane >> 5;
    constexpr int kAcross = NT * 4, kDown = 64 / kAcross;      // lanes along a row, rows at once
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    stage[(8 * (e >> 2) + 4 * half + (e & 3)) * kStageLd + 32 * j + r32] = acc[i][j][8 * h + e];
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int turn = 0; turn < 16 / kDown; ++turn) {
                const int row = turn * kDown + lane / kAcross, col = lane % kAcross * kChunk;
                const v4f lo = *reinterpret_cast<const v4f*>(stage + row * kStageLd + col);
                const v4f hi = *reinterpret_cast<const v4f*>(stage + row * kStageLd + col + 4);
                float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
                const int m = m0 + wm + 32 * i + 16 * h + row, n = n0 + wn + col;
                if (g.splits > 1) {
                    if (m < g.M && n < g.N)
                        store_values(g.raw + ((size_t)split * g.M + m) * g.N + n, g.N - n, v);
                } else {
                    finish_chunk(g.f, g.M, g.N, m, n, v);
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
}

// Sums of the splits' partial sums, in their order, and what follows.
constexpr int kJoinThreads = 256;
__global__ __launch_bounds__(kJoinThreads) void k_join(const float* raw, int splits, int M, int N, int chunks, const Finish f) {
    const long long id = (long long)blockIdx.x * kJoinThreads + threadIdx.x;
    const long long row = id / chunks;
    const int n = (int)(id % chunks) * kChunk;
    const int m = row < M ? (int)row : M;                     // lanes past the end stay with their quads
    float v[8] = {};
    if (m < M && n < N) {
        for (int p = 0; p < splits; ++p) {
            float u[8];
            load_values(raw + ((size_t)p * M + m) * N + n, N - n, u);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += u[i];
        }
    }
    finish_chunk(f, M, N, m, n, v);
}

// ---- which tiles ---------------------------------------------------------------------------------------------------------
struct Plan { int bm, bn, splits, k_tiles_per_split; };
constexpr int kGroups = 256;             // workgroups that fill the chip
constexpr int kLeastTiles = 4;           // of the contraction a split has

Plan plan_of(int M, int N, int K, bool bf16) {
    const int k_tiles = ceil_div(K, bf16 ? 64 : 32);
    Plan p{64, 64, 1, k_tiles};
    const long long big = (long long)ceil_div(M, 128) * ceil_div(N, 128);
    if (M > 64 && N > 64 && big >= 128) p.bm = p.bn = 128;
    const long long tiles = (long long)ceil_div(M, p.bm) * ceil_div(N, p.bn);
    if (tiles < kGroups) {
        const int want = (int)std::min<long long>(kGroups / tiles, k_tiles / kLeastTiles);
        if (want > 1) {
            p.k_tiles_per_split = ceil_div(k_tiles, want);
            p.splits = ceil_div(k_tiles, p.k_tiles_per_split);
        }
    }
    return p;
}

template <class C, int PK, int QK, bool PA, bool QA, int BM, int BN, int WM, int WN>
void start(const Args& a, hipStream_t s) {
    k_product<C, PK, QK, PA, QA, BM, BN, WM, WN>
        <<<dim3((unsigned)a.tiles_m * a.tiles_n * a.splits), 64 * WM * WN, 0, s>>>(a);
}

template <class C, int PK, int QK, bool PA, bool QA>
hipError_t run(const Product& g, hipStream_t s) {
    const Plan p = plan_of(g.M, g.N, g.K, sizeof(C) == 2);
    const Args a{g.P, g.Q, g.M, g.N, g.K, ceil_div(g.M, p.bm), ceil_div(g.N, p.bn), p.splits, p.k_tiles_per_split, g.raw, g.f};
    if (p.bm == 128) start<C, PK, QK, PA, QA, 128, 128, 2, 2>(a, s);
    else start<C, PK, QK, PA, QA, 64, 64, 2, 2>(a, s);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && p.splits > 1) {
        const int chunks = whole_groups(g.N) / kChunk;
        const long long threads = (long long)g.M * chunks;
        k_join<<<dim3((unsigned)((threads + kJoinThreads - 1) / kJoinThreads)), kJoinThreads, 0, s>>>(g.raw, p.splits, g.M, g.N,
                                                                                                     chunks, g.f);
        e = hipGetLastError();
    }
    return e;
}

template <class C, int T>
hipError_t by_use(const Product& g, hipStream_t s) {
    if (!g.P_along_own && !g.Q_along_own)
        return g.P.kind == E4M3 ? run<C, E4M3, T, false, false>(g, s) : run<C, T, T, false, false>(g, s);
    if (!g.P_along_own) return run<C, T, T, false, true>(g, s);
    return g.Q.kind == E4M3 ? run<C, T, E4M3, true, true>(g, s) : run<C, T, T, true, true>(g, s);
}

}  // namespace

// Of any plan of this product and of smaller ones: splits <= k_tiles / kLeastTiles, and splits * tiles <= kGroups.
size_t product_scratch_bytes(int M, int N, int K, bool bf16) {
    const int splits = ceil_div(K, bf16 ? 64 : 32) / kLeastTiles;
    if (splits < 2) return 0;
    return std::min((size_t)kGroups * 128 * 128, (size_t)splits * M * N) * sizeof(float);
}

hipError_t launch_product(const Product& g, hipStream_t s) {
    return g.P.kind == F32 || g.Q.kind == F32 ? by_use<float, F32>(g, s) : by_use<__bf16, BF16>(g, s);
}

}  // namespace ops
}  // namespace lf
