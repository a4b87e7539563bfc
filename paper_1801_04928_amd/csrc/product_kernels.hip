// The matrix product of residual blocks,  C[m][n] = sum_q P(m,q) Q(n,q)  with fp32 sums, in its three uses:
//   forward   P = x  (contiguous along q)          Q = w (contiguous along q)          C = z -> bias, activation, residual
//   dx        P = dz (contiguous along q)          Q = w (contiguous along its own n)
//   dw        P = dz (contiguous along its own m)  Q = x (contiguous along its own n)
// Operands are fp32 or bf16; x may be in 8 bits, whose values are bf16 numbers: they are made when a tile is laid into LDS,
// and the matrix instructions see no difference.
#include "activation.h"
#include "chunks.h"
#include "column_sums.h"

#include <algorithm>
#include <type_traits>

namespace lf {
namespace ops {
namespace {

constexpr int kRowBytes = 128;            // of a tile, along q: 64 bf16 or 32 fp32

__host__ __device__ constexpr int ceil_div(int a, int b) { return a / b + (a % b != 0); }
__host__ __device__ constexpr int whole_groups(int cols) { return ceil_div(cols, kGroup) * kGroup; }

struct Args {
    Mat P, Q;
    int M, N, K;
    int tiles_m, tiles_n, k_tiles;
    int splits, k_tiles_per_split;
    float* raw;                           // [splits][M][N] if splits > 1
    Finish f;
};

// Elements of a piece on their way from memory to LDS.
template <int KIND, int N> struct Raw;
template <> struct Raw<F32, 4> { v4f a; };
template <> struct Raw<BF16, 8> { v4u a; };
template <> struct Raw<E4M3, 8> { v2u a; int byte; };
template <> struct Raw<E4M3, 16> { v4u a; int byte; };

// One operand's tile of I rows by BK: loaded into registers, laid into LDS as numbers of the products' type C.
//
// Loads are one instruction a piece with no branch around it, whatever the sizes: what is not there is not loaded but something
// that is, and put right on the way to LDS (only in tiles at an end).  A piece that the row's end cuts is loaded from
// as far ahead as makes it whole and its elements moved down.  That needs rows of at least eight elements; narrower
// operands are loaded element by element (NARROW).
//
// LDS of a tile contiguous along q: [i][q], rows of eight 16-byte pieces, piece p of row i at place p ^ (i / 2 % 8): the pieces of
// 16 rows, which LDS serves at once, then lie in different ones of its 64 banks (of rows 128 bytes long two share them).
// Contiguous along i: [q][i]; bf16 is read there by transposing loads, eight rows of 64 bytes at a time (q, q+1, q+2, q+3 and
// eight further), whose 64-byte segments change places the same way; of fp32 the two halves of a wave read rows four
// apart, whose 128-byte segments change places.
template <class C, int KIND, bool ALONG, int I, int THREADS, bool NARROW>
struct Tile {
    static constexpr int BK = kRowBytes / (int)sizeof(C);
    static constexpr int kElems = I * BK;
    static constexpr int kPiece = KIND == E4M3 ? (sizeof(C) == 2 ? 16 : 8) : 16 / (int)sizeof(C);
    static constexpr int kPieces = I * BK / kPiece / THREADS;
    static constexpr int kElemBytes = KIND == F32 ? 4 : KIND == BF16 ? 2 : 1;
    static_assert(kPieces * THREADS * kPiece == I * BK, "whole pieces for every thread");

    Raw<KIND, kPiece> r[kPieces];

    // Place of piece u of thread t in the tile: i and q.
    static __device__ __forceinline__ void place(int t, int u, int& i, int& q) {
        const int id = t + u * THREADS;
        if constexpr (ALONG) { i = id % (I / kPiece) * kPiece; q = id / (I / kPiece); }
        else { q = id % (BK / kPiece) * kPiece; i = id / (BK / kPiece); }
    }
    // Elements of a row that exist in memory: 8 bits come in whole groups.
    static __device__ __forceinline__ int in_memory(int n) { return KIND == E4M3 ? whole_groups(n) : n; }

    // What stays the same from k-tile to k-tile: the offset of every piece in its tile, and of its scale; contiguous along i also
    // that of its column alone, for rows past the contraction's end.
    unsigned at[kPieces], scale_at[KIND == E4M3 ? kPieces : 1];
    __device__ __forceinline__ void begin(const Mat& m, int t, int i0, int I_all) {
        const unsigned ld = (unsigned)m.ld * kElemBytes, scale_ld = (unsigned)m.scale_ld;
#pragma unroll
        for (int u = 0; u < kPieces; ++u) {
            int i, q;
            place(t, u, i, q);
            const unsigned row = min(i, I_all - 1 - i0);
            at[u] = ALONG ? column(i0, i, I_all) * kElemBytes + (unsigned)q * ld : row * ld;
            if constexpr (KIND == E4M3) scale_at[u] = ALONG ? column(i0, i, I_all) / kGroup + (unsigned)q * scale_ld : row * scale_ld;
        }
    }
    static __device__ __forceinline__ unsigned column(int i0, int i, int I_all) { return min(i0 + i, in_memory(I_all) - kPiece); }
    // I_all: rows of the operand; q_end: where this workgroup's part of the contraction ends.
    __device__ __forceinline__ void load(const Mat& m, int t, int i0, int I_all, int q0, int q_end) {
        if constexpr (NARROW) {
            load_elements(m, t, i0, I_all, q0, q_end);
            return;
        }
        const int q_first = min(q0, q_end - 1);
        const unsigned ld = (unsigned)m.ld * kElemBytes, scale_ld = (unsigned)m.scale_ld;
        const uint8_t* base = (const uint8_t*)m.p + (ALONG ? (long long)q_first * ld : (long long)i0 * ld);
        const uint8_t* scales = KIND == E4M3 ? m.scales + (ALONG ? (long long)q_first * scale_ld : (long long)i0 * scale_ld) : nullptr;
#pragma unroll
        for (int u = 0; u < kPieces; ++u) {
            int i, q;
            place(t, u, i, q);
            // past the contraction's end: the tile's first row, or the row's last piece
            const bool there = q_first + q < q_end;
            const unsigned col = ALONG ? column(i0, i, I_all) : min(q0 + q, in_memory(q_end) - kPiece);
            const unsigned off = !ALONG ? at[u] + col * kElemBytes : there ? at[u] : col * kElemBytes;
            if constexpr (KIND == F32) {
                r[u].a = load_vector((const float*)(base + off));
            } else if constexpr (KIND == BF16) {
                r[u].a = __builtin_bit_cast(v4u, load_vector((const __bf16*)(base + off)));
            } else {
                if constexpr (kPiece == 16) r[u].a = *as_global<const v4u>(base + off);
                else r[u].a = *as_global<const v2u>(base + off);
                r[u].byte = *as_global<const uint8_t>(
                    scales + (!ALONG ? scale_at[u] + col / kGroup : there ? scale_at[u] : col / kGroup));
            }
        }
    }
    __device__ __forceinline__ void load_elements(const Mat& m, int t, int i0, int I_all, int q0, int q_end) {
#pragma unroll
        for (int u = 0; u < kPieces; ++u) {
            int i, q;
            place(t, u, i, q);
            const int n = ALONG ? (q0 + q < q_end ? I_all - i0 - i : 0) : (i0 + i < I_all ? q_end - q0 - q : 0);
            const long long row = ALONG ? q0 + q : i0 + i;
            const int col = ALONG ? i0 + i : q0 + q;
            if constexpr (KIND == E4M3) {
                r[u].a = decltype(r[u].a){};
                r[u].byte = 127;
                if (n > 0) {
                    r[u].a = *as_global<const decltype(r[u].a)>((const uint8_t*)m.p + row * m.ld + col);
                    r[u].byte = *as_global<const uint8_t>(m.scales + row * m.scale_ld + col / kGroup);
                }
            } else {
                typedef typename Stored<KIND>::type T;
                const T* p = (const T*)m.p + row * m.ld + col;
                T v[kPiece];
#pragma unroll
                for (int e = 0; e < kPiece; ++e) v[e] = e < n ? *as_global<const T>(p + e) : (T)0.0f;
                __builtin_memcpy(&r[u].a, v, 16);
            }
        }
    }
    // Puts pieces of a tile at an end right: past the contraction's end zeros, cut pieces whole.
    __device__ __forceinline__ void mend(int t, int i0, int I_all, int q0, int q_end) {
#pragma unroll
        for (int u = 0; u < kPieces; ++u) {
            int i, q;
            place(t, u, i, q);
            const bool dead = q0 + q >= q_end;
            if constexpr (KIND == E4M3) {
                keep_codes(r[u].a, ALONG ? (dead ? 0 : kPiece) : q_end - q0 - q);
            } else if constexpr (!NARROW) {
                const int s = ALONG ? max(0, i0 + i - (I_all - kPiece)) : max(0, q0 + q - (q_end - kPiece));
                shift_down(r[u].a, dead ? kPiece : s);
            }
        }
    }
    static __device__ __forceinline__ bool at_end(int i0, int I_all, int q0, int q_end) {
        return q0 + BK > q_end || (ALONG && i0 + I > I_all);
    }

    // Where 16-byte pieces go.
    static __device__ __forceinline__ int at_along_q(int i, int piece) {
        return i * BK + ((piece ^ ((i >> 1) & 7)) * (16 / (int)sizeof(C)));
    }
    static __device__ __forceinline__ int at_along_i(int q, int i) {
        if constexpr (sizeof(C) == 2) {
            constexpr int kSegments = I / 32;
            const int turn = ((q & 3) | ((q >> 1) & 4)) & (kSegments < 8 ? kSegments - 1 : 7);
            return q * I + (((i >> 5) ^ turn) << 5) + (i & 31);
        } else {
            return q * I + (i ^ ((q & 4) << 3));
        }
    }
    __device__ __forceinline__ void store(C* s, int t) const {
#pragma unroll
        for (int u = 0; u < kPieces; ++u) {
            int i, q;
            place(t, u, i, q);
            if constexpr (KIND != E4M3) {
                *reinterpret_cast<decltype(r[u].a)*>(s + (ALONG ? at_along_i(q, i) : at_along_q(i, q / kPiece))) = r[u].a;
            } else if constexpr (sizeof(C) == 2) {
                const float scale = scale_power(r[u].byte);          // (the instruction looks at the exponent alone)
#pragma unroll
                for (int h = 0; h < kPiece / 8; ++h) {
                    v8bf v;
#pragma unroll
                    for (int w = 0; w < 2; ++w) {
                        const v2bf a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)r[u].a[2 * h + w], scale, false);
                        const v2bf b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)r[u].a[2 * h + w], scale, true);
                        v[4 * w] = a[0]; v[4 * w + 1] = a[1]; v[4 * w + 2] = b[0]; v[4 * w + 3] = b[1];
                    }
                    *reinterpret_cast<v8bf*>(s + (ALONG ? at_along_i(q, i + 8 * h) : at_along_q(i, q / 8 + h))) = v;
                }
            } else {
                v4f a, b;
                float v[8];
                eight_values(r[u].a, scale_value(r[u].byte), v);
                a = v4f{v[0], v[1], v[2], v[3]};
                b = v4f{v[4], v[5], v[6], v[7]};
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
    // instructions that a tile takes: requests, stores to LDS, and loads of one operand from there
    static constexpr int kRequests = kPieces * (KIND == E4M3 ? 2 : 1);
    static constexpr int kStores = kElems * (int)sizeof(C) / 16 / THREADS, kReads = ALONG ? 2 : 1;
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
__device__ __forceinline__ void store_any(const Mat& m, long long row, int col, int n, const float (&v)[8], bool live) {
    if (m.kind == E4M3) store_chunk<E4M3>(m, row, col, n, v, live);
    else if (m.kind == F32) store_chunk<F32>(m, row, col, n, v, live);
    else store_chunk<BF16>(m, row, col, n, v, live);
}
template <int ACT>
__device__ __forceinline__ void activate_all(float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = activate(ACT, v[i]);
}
// The residual has the storage type, which is C's.  Zeros if there is none, or no such row.
template <class C>
__device__ __forceinline__ void load_residual(const Finish& f, int M, int m, int n, int there, float (&r)[8]) {
    if (f.residual.p && m < M) {
        load_values((const C*)f.residual.p + m * f.residual.ld + n, there, r);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] = 0.0f;
    }
}
// Eight columns of row m from n on (n a multiple of 8; the four lanes of a quad hold the four chunks of a group of 32).
__device__ __forceinline__ void finish_chunk(const Finish& f, int M, int N, int m, int n, float (&v)[8], const float (&bias)[8],
                                             const float (&residual)[8]) {
    const int there = m < M ? min(N - n, kChunk) : 0;
    const bool live = m < M && n < whole_groups(N);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < there ? v[i] + bias[i] : 0.0f;
    if (f.z.p) store_any(f.z, m, n, there, v, live);
    switch (f.act) {                        // (the branch is outside the loop over the eight values)
        case SIGMOID: activate_all<SIGMOID>(v); break;
        case RELU: activate_all<RELU>(v); break;
        case SILU: activate_all<SILU>(v); break;
        case GELU: activate_all<GELU>(v); break;
        default: break;
    }
    // (past the row's end zeros: sigmoid(0) is not 0, and a group's scale looks at all of its values)
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < there ? v[i] + residual[i] : 0.0f;
    store_any(f.y, m, n, there, v, live);
}

// The order in which a step's instructions are issued, as scheduling groups (0x008 matrix instruction, 0x020 request, 0x100
// LDS read, 0x200 LDS write): after every matrix instruction its share of the next step's reads, all of them in the step's
// first half, of the writes to LDS and of the requests into the registers these have left.  The compiler by itself puts all
// writes and requests before the first matrix instruction, and those stand still meanwhile.
template <int MASK, int N> __device__ __forceinline__ void issue() {
    if constexpr (N > 0) __builtin_amdgcn_sched_group_barrier(MASK, N, 0);
}
template <int M, int READS, int WRITES, int REQUESTS, int I = 0>
__device__ __forceinline__ void interleave() {
    if constexpr (I < M) {
        constexpr int window = M >= 8 ? M : M > 1 ? M / 2 : 1, a = I < window ? I : window, b = I < window ? I + 1 : window;
        issue<0x008, 1>();
        issue<0x100, READS * b / window - READS * a / window>();
        issue<0x200, WRITES * (I + 1) / M - WRITES * I / M>();
        issue<0x020, REQUESTS * (I + 1) / M - REQUESTS * I / M>();
        interleave<M, READS, WRITES, REQUESTS, I + 1>();
    }
}

// ================================================================================================
// tiles of BM x BN by WM x WN waves
// ================================================================================================
// Of KS groups of WM x WN waves each walks every KS-th k-tile of its workgroup's part.  D k-tiles are under way in registers,
// one lies in LDS for the multiplications, and one is laid beside it meanwhile.  The two buffers are arrays of their own, so
// that the compiler knows the writes to one and the reads of the other apart.
// A wave's 64 x 128 of a 256 x 256 tile reads 6 KB of LDS for eight matrix instructions of 32 cycles, with which LDS keeps pace; 64 x
// 64 of a 128 x 128 tile reads 4 KB for four, which takes all of LDS's time, but four times as many tiles fill the chip
// where the matrices are smaller; 64 x 64 tiles do so for the smallest.  Measured: 4096 x 8192 x 8192 bf16 428 us = 1.28 PFLOP/s
// (matrix cores busy 59 %), 512 x 8192 x 8192 in 8 bits 96 us = 0.71 PFLOP/s, weights from memory (34 %), 256 x 4096 x 4096 fp32 68 us
// = 127 TFLOP/s in a long run (72 %).  Registers hold 256 x 256's sums and one k-tile under way, just so: the instance for x in 8 bits
// spills one, that of dx two, and the early barrier's operands do not fit.
template <class C, int BM, int BN, int KS>
constexpr int kLdsElems = KS * (BM + BN) * (kRowBytes / (int)sizeof(C));

template <class C, int PK, int QK, bool P_ALONG, bool Q_ALONG, int BM, int BN, int WM, int WN, int KS, int D, bool NARROW>
__device__ __forceinline__ void product_tile(const Args& g, unsigned block, C* lds0, C* lds1) {
    constexpr int kThreads = 64 * WM * WN;
    typedef Tile<C, PK, P_ALONG, BM, kThreads, NARROW> TP;
    typedef Tile<C, QK, Q_ALONG, BN, kThreads, NARROW> TQ;
    constexpr int BK = TP::BK, MT = BM / WM / 32, NT = BN / WN / 32;
    static_assert(D == 1 || D == 2, "a k-tile's registers and buffer are known when it is compiled");
    // the epilogue's staging, half of the waves in either buffer: as many rows of a wave's own as fit, with groups half of what
    // is divided between them
    constexpr int kStageLd = NT * 32 + 4, kHalf = KS == 1 ? WM * WN / 2 : WM * WN * KS;
    constexpr int kFit = kLdsElems<C, BM, BN, KS> * (int)sizeof(C) / (kHalf * kStageLd * 4), kUnitRows = KS == 1 && kFit >= 32 ? 32 : 16;
    static_assert(kFit >= 16, "the staging fits");

    const int t = threadIdx.x % kThreads, group = KS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / kThreads);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    // Workgroups are dealt to the 8 XCDs in turn: an XCD takes neighbouring tiles (and, of a split product, one split's).
    const int tiles = g.tiles_m * g.tiles_n, total = tiles * g.splits;
    const int per = total / 8, rest = total % 8, xcd = block % 8;
    const int id = xcd * per + min(xcd, rest) + block / 8;
    const int split = id / tiles, tile = id % tiles;
    // ... in bands of eight rows of tiles
    const int band = tile / (8 * g.tiles_n), high = min(8, g.tiles_m - 8 * band), in_band = tile - 8 * band * g.tiles_n;
    const int m0 = (8 * band + in_band % high) * BM, n0 = in_band / high * BN;
    const int wm = wave / WN * (MT * 32), wn = wave % WN * (NT * 32);
    const int kt0 = split * g.k_tiles_per_split, kt1 = min(g.k_tiles, kt0 + g.k_tiles_per_split);
    const int q_end = min(g.K, kt1 * BK);
    const int turns = ceil_div(kt1 - kt0, KS);

    // (two sums of a wave's only 32 x 32 square, taken in turn: a matrix instruction would wait for the one before it)
    constexpr int kChains = MT * NT == 1 ? 2 : 1;
    v16f acc[MT][NT][kChains];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int c = 0; c < kChains; ++c)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][c][e] = 0.0f;

    TP tp[D];
    TQ tq[D];
    auto q_of = [&](int turn) { return (kt0 + turn * KS + group) * BK; };
#pragma unroll
    for (int d = 0; d < D; ++d) {
        tp[d].begin(g.P, t, m0, g.M);
        tq[d].begin(g.Q, t, n0, g.N);
    }
    // (past the last k-tile the last one again, which nothing looks at: no branch around the loads)
    auto request = [&](int d, int turn) {
        const int q0 = q_of(min(turn, turns - 1));
        tp[d].load(g.P, t, m0, g.M, q0, q_end);
        tq[d].load(g.Q, t, n0, g.N, q0, q_end);
    };
    auto mend = [&](int d, int turn) {
        const int q0 = q_of(turn);
        if (TP::at_end(m0, g.M, q0, q_end)) tp[d].mend(t, m0, g.M, q0, q_end);
        if (TQ::at_end(n0, g.N, q0, q_end)) tq[d].mend(t, n0, g.N, q0, q_end);
    };
    auto lay = [&](int d, C* buffer) {
        tp[d].store(buffer, t);
        tq[d].store(buffer + TP::kElems, t);
    };
    typename TP::Operand a[2][MT], q[2][NT];
    auto read = [&](const C* sp, auto step) {
#pragma unroll
        for (int i = 0; i < MT; ++i) a[step() % 2][i] = TP::operand(sp, wm + 32 * i, step());
#pragma unroll
        for (int j = 0; j < NT; ++j) q[step() % 2][j] = TQ::operand(sp + TP::kElems, wn + 32 * j, step());
    };
    auto multiply = [&](auto step) {
        constexpr int set = step() % 2;
        if constexpr (sizeof(C) == 2) {
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    v16f& sum = acc[i][j][step() % kChains];
                    sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[set][i], q[set][j], sum, 0, 0, 0);
                }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < NT; ++j) {
                        v16f& sum = acc[i][j][e % kChains];
                        sum = __builtin_amdgcn_mfma_f32_32x32x2f32(a[set][i][e], q[set][j][e], sum, 0, 0, 0);
                    }
        }
    };
    C* const buffers[2] = {lds0 + group * (TP::kElems + TQ::kElems), lds1 + group * (TP::kElems + TQ::kElems)};
    constexpr std::integral_constant<int, 0> s0;
    constexpr std::integral_constant<int, 1> s1;
    constexpr std::integral_constant<int, 2> s2;
    constexpr std::integral_constant<int, 3> s3;
    static_assert(TP::kSteps == 4, "the steps below");
    constexpr int kMfmas = MT * NT * (sizeof(C) == 2 ? 1 : 4), kStepReads = MT * TP::kReads + NT * TQ::kReads;
    constexpr int kWrites = TP::kStores + TQ::kStores, kRequests = TP::kRequests + TQ::kRequests;
    // Multiplies a k-tile and lays the next one, which goes to the buffer that all waves had read before the last barrier.  EARLY:
    // the barrier stands before the last step, whose operands are in registers by then, and the next tile's first operands are
    // read while it is multiplied.  (Of 256 x 256 tiles these registers are not there: they would be spilled.)
    constexpr bool EARLY = MT * NT <= 4;
    const auto k_tile = [&](int turn, auto at) {
        constexpr int d = at(), next = (d + 1) % D;
        mend(next, turn + 1);
        lay(next, buffers[(d + 1) & 1]);
        request(next, turn + 1 + D);
        if constexpr (!EARLY) {
            read(buffers[d & 1], s0);
            issue<0x100, kStepReads>();
        }
        read(buffers[d & 1], s1);
        multiply(s0);
        read(buffers[d & 1], s2);
        multiply(s1);
        read(buffers[d & 1], s3);
        multiply(s2);
        if constexpr (!NARROW) {
            interleave<kMfmas, kStepReads, kWrites / 3, kRequests / 3>();
            interleave<kMfmas, kStepReads, kWrites * 2 / 3 - kWrites / 3, kRequests * 2 / 3 - kRequests / 3>();
            interleave<kMfmas, kStepReads, kWrites - kWrites * 2 / 3, kRequests - kRequests * 2 / 3>();
        }
        if constexpr (EARLY) {
            __syncthreads();
            read(buffers[(d + 1) & 1], s0);
            multiply(s3);
            if constexpr (!NARROW) interleave<kMfmas, kStepReads, 0, 0>();
        } else {
            multiply(s3);
            interleave<kMfmas, 0, 0, 0>();
            __syncthreads();
        }
    };
    if (turns > 0) {
#pragma unroll
        for (int d = 0; d < D; ++d) request(d, d);
        mend(0, 0);
        lay(0, buffers[0]);
        request(0, D);
        __syncthreads();
        if constexpr (EARLY) read(buffers[0], s0);
        int turn = 0;
        // (a way out between the two would cost the sums a second set of registers)
        for (; turn + 1 < turns; turn += 2) {
            k_tile(turn, s0);
            k_tile(turn + 1, s1);
        }
        if (turn < turns) {
            if constexpr (!EARLY) read(buffers[0], s0);
            read(buffers[0], s1);
            multiply(s0);
            read(buffers[0], s2);
            multiply(s1);
            read(buffers[0], s3);
            multiply(s2);
            multiply(s3);
        }
        __syncthreads();          // the buffers become the epilogue's
    }
    if constexpr (kChains == 2) acc[0][0][0] += acc[0][0][1];
    // Accumulator element e of lane (r32, half) of square (i, j) is C[.. 32 i + 8 (e / 4) + 4 half + e % 4][.. 32 j + r32]: of a wave's
    // rows, unit u, rows kUnitRows u and on, is kElems elements of every square in a row of them.
    constexpr int kUnits = MT * 32 / kUnitRows / KS, kElems = kUnitRows / 2;
    float own[kUnits][NT][kElems];
    const auto element = [&](int u, int j, int e) {
        return acc[u * kUnitRows / 32][j][0][u * kUnitRows % 32 / 2 + e];
    };
    if constexpr (KS == 1) {
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int e = 0; e < kElems; ++e) own[u][j][e] = element(u, j, e);
    } else {
        // of two groups' sums each finishes half: it gives the other half away and adds what it gets
        static_assert(KS == 2 && 2 * kUnits * NT * kElems * kThreads * 4 <= kLdsElems<C, BM, BN, KS> * (int)sizeof(C), "the sums fit");
        v4f* sums = reinterpret_cast<v4f*>(lds0);
        constexpr int kVecs = kElems / 4, kAll = kUnits * NT * kVecs * kThreads;
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int v = 0; v < kVecs; ++v) {
                    v4f give;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float low = element(u, j, 4 * v + e), high = element(u + kUnits, j, 4 * v + e);
                        own[u][j][4 * v + e] = group == 0 ? low : high;
                        give[e] = group == 0 ? high : low;
                    }
                    sums[group * kAll + ((u * NT + j) * kVecs + v) * kThreads + t] = give;
                }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int v = 0; v < kVecs; ++v) {
                    const v4f got = sums[(1 - group) * kAll + ((u * NT + j) * kVecs + v) * kThreads + t];
#pragma unroll
                    for (int e = 0; e < 4; ++e) own[u][j][4 * v + e] += got[e];
                }
    }

    // Rows turn through LDS, the wave's own, so that a lane holds eight consecutive columns; nobody waits.  (With groups all of it
    // in the second buffer: the first still holds sums.)
    const int r32 = lane & 31, half = lane >> 5, of_all = group * WM * WN + wave;
    float* stage = reinterpret_cast<float*>(KS == 1 && of_all < kHalf ? lds0 : lds1) + (KS == 1 ? of_all % kHalf : of_all) * (kUnitRows * kStageLd);
    constexpr int kAcross = NT * 4, kDown = 64 / kAcross;      // lanes along a row, rows at once
    const int n = n0 + wn + lane % kAcross * kChunk, n_there = min(max(g.N - n, 0), kChunk);
    // the column stays the same: its bias is loaded once; a residual is under way while the rows before it are finished
    float bias[8];
    if (g.f.bias && g.splits == 1) {
        load_values(g.f.bias + n, n_there, bias);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) bias[i] = 0.0f;
    }
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < kElems; ++e)
                stage[(8 * (e >> 2) + 4 * half + (e & 3)) * kStageLd + 32 * j + r32] = own[u][j][e];
        __builtin_amdgcn_wave_barrier();
        // (one copy of what follows in the code: an epilogue unrolled is larger than the instruction cache)
        const int first = m0 + wm + kUnitRows * (group * kUnits + u);
        float residual[8];
        load_residual<C>(g.f, g.M, first + lane / kAcross, n, n_there, residual);
#pragma unroll 1
        for (int row = lane / kAcross; row < kUnitRows; row += kDown) {
            const int col = lane % kAcross * kChunk, m = first + row;
            const v4f lo = *reinterpret_cast<const v4f*>(stage + row * kStageLd + col);
            const v4f hi = *reinterpret_cast<const v4f*>(stage + row * kStageLd + col + 4);
            float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]}, r[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) r[i] = residual[i];
            load_residual<C>(g.f, g.M, row + kDown < kUnitRows ? m + kDown : g.M, n, n_there, residual);
            if (g.splits > 1) {
                if (m < g.M && n_there > 0) store_values(g.raw + ((size_t)split * g.M + m) * g.N + n, n_there, v);
            } else {
                finish_chunk(g.f, g.M, g.N, m, n, v, bias, r);
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

template <class C, int PK, int QK, bool P_ALONG, bool Q_ALONG, int BM, int BN, int WM, int WN, int KS, int D, bool NARROW>
__global__ __launch_bounds__(64 * WM * WN * KS) void k_product(const Args g) {
    __shared__ __attribute__((aligned(16))) C lds0[kLdsElems<C, BM, BN, KS>];
    __shared__ __attribute__((aligned(16))) C lds1[kLdsElems<C, BM, BN, KS>];
    product_tile<C, PK, QK, P_ALONG, Q_ALONG, BM, BN, WM, WN, KS, D, NARROW>(g, blockIdx.x, lds0, lds1);
}

// Both products of a backward pass in one launch: the first `first` workgroups take dx, the others dw.
template <class C, int T, int XK, int B, int KS>
__global__ __launch_bounds__(256 * KS) void k_both(const Args dx, const Args dw, unsigned first) {
    __shared__ __attribute__((aligned(16))) C lds0[kLdsElems<C, B, B, KS>];
    __shared__ __attribute__((aligned(16))) C lds1[kLdsElems<C, B, B, KS>];
    if (blockIdx.x < first) product_tile<C, T, T, false, true, B, B, 2, 2, KS, 2, false>(dx, blockIdx.x, lds0, lds1);
    else product_tile<C, T, XK, true, true, B, B, 2, 2, KS, 2, false>(dw, blockIdx.x - first, lds0, lds1);
}

// Sums of the splits' partial sums, in their order, and what follows.
struct Join {
    const float* raw;
    int splits, M, N, chunks;
    Finish f;
};
Join join_of(const Args& a) { return Join{a.raw, a.splits, a.M, a.N, whole_groups(a.N) / kChunk, a.f}; }
unsigned join_blocks(const Join& a, int threads) {
    return a.splits > 1 ? (unsigned)(((long long)a.M * a.chunks + threads - 1) / threads) : 0;
}
template <class C, int THREADS>
__device__ __forceinline__ void join(const Join& a, unsigned block) {
    const long long id = (long long)block * THREADS + threadIdx.x;
    const long long row = id / a.chunks;
    const int n = (int)(id % a.chunks) * kChunk;
    const int m = row < a.M ? (int)row : a.M;                 // lanes past the end stay with their quads
    const int there = m < a.M ? min(max(a.N - n, 0), kChunk) : 0;
    float v[8] = {}, bias[8] = {}, residual[8];
    if (a.f.bias) load_values(a.f.bias + n, there, bias);
    load_residual<C>(a.f, a.M, m, n, there, residual);
    const float* at = a.raw + (size_t)m * a.N + n;
    const size_t step = (size_t)a.M * a.N;
    const auto add = [&](int p, int some) {
        float u[8];
        load_values(at + p * step, some, u);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += u[i];
    };
    if (there == kChunk) {                // whole chunks: eight loads under way
#pragma unroll 8
        for (int p = 0; p < a.splits; ++p) add(p, kChunk);
    } else if (there > 0) {
        for (int p = 0; p < a.splits; ++p) add(p, there);
    }
    finish_chunk(a.f, a.M, a.N, m, n, v, bias, residual);
}
constexpr int kJoinThreads = 256;
template <class C>
__global__ __launch_bounds__(kJoinThreads) void k_join(const Join a) { join<C, kJoinThreads>(a, blockIdx.x); }

// What a backward pass of split products ends with, in one launch: both products' sums and those of db.
template <class C>
__global__ __launch_bounds__(kFinishThreads) void k_join_all(const Join dx, unsigned x_blocks, const Join dw, unsigned w_blocks,
                                                             const ColumnSums db) {
    if (blockIdx.x < x_blocks) join<C, kFinishThreads>(dx, blockIdx.x);
    else if (blockIdx.x < x_blocks + w_blocks) join<C, kFinishThreads>(dw, blockIdx.x - x_blocks);
    else finish_columns(db, blockIdx.x - x_blocks - w_blocks);
}

// ================================================================================================
// a few rows
// ================================================================================================
// One sample, or up to four: the product is the reading of w.  A wave takes two outputs and walks their rows of w, 512 q a
// step, with the same q of x; a workgroup's outputs are whole chunks, or whole groups of 32 (WAVES = 16) where the results
// are kept in 8 bits.  Bound by memory: all of a wave's requests for some thousand q are under way at once.  1, 2, 4 rows x 4096 x
// 4096 bf16, with the launch: 7.9, 9.5, 10.9 us (one row in a long run 7.4 = 4.5 TB/s), against 12.8, 12.9, 12.9 with 64 x 64 tiles,
// split and joined.  Beyond four rows the multiplications, 8 a row and value of w, would take longer than the reading.
constexpr int kFewRows = 4, kFewOutputs = 2;
template <class C, int XK, int ROWS, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_few(const Args g) {
    constexpr int kStep = 64 * kChunk, kUnroll = ROWS == 1 ? 4 : ROWS == 4 && XK == E4M3 ? 1 : 2, kOutputs = WAVES * kFewOutputs;
    __shared__ float sums[ROWS][kOutputs];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n0 = blockIdx.x * kOutputs, n = n0 + wave * kFewOutputs;
    float sum[ROWS][kFewOutputs] = {};
    const auto step = [&](int q0, auto unroll, bool whole) {
        constexpr int U = unroll();
        float x[U][ROWS][8], w[U][kFewOutputs][8];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int q = q0 + u * kStep + lane * kChunk, there = whole ? kChunk : min(g.K - q, kChunk);
#pragma unroll
            for (int o = 0; o < kFewOutputs; ++o)
                load_values((const C*)g.Q.p + min(n + o, g.N - 1) * g.Q.ld + q, there, w[u][o]);
#pragma unroll
            for (int m = 0; m < ROWS; ++m) load_chunk<XK>(g.P, min(m, g.M - 1), q, there, x[u][m]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int m = 0; m < ROWS; ++m)
#pragma unroll
                for (int o = 0; o < kFewOutputs; ++o)
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum[m][o] = fmaf(x[u][m][e], w[u][o][e], sum[m][o]);
    };
    int q0 = 0;
    for (; q0 + kUnroll * kStep <= g.K; q0 += kUnroll * kStep) step(q0, std::integral_constant<int, kUnroll>(), true);
    for (; q0 < g.K; q0 += kStep) step(q0, std::integral_constant<int, 1>(), false);
#pragma unroll
    for (int m = 0; m < ROWS; ++m)
#pragma unroll
        for (int o = 0; o < kFewOutputs; ++o) {
            const float all = wave_sum(sum[m][o]);
            if (lane == 0) sums[m][wave * kFewOutputs + o] = all;
        }
    __syncthreads();
    constexpr int kChunks = kOutputs / kChunk;
    if (threadIdx.x >= ROWS * kChunks) return;
    const int m = threadIdx.x / kChunks, col = threadIdx.x % kChunks * kChunk, there = min(max(g.N - n0 - col, 0), kChunk);
    float v[8], bias[8] = {}, residual[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = sums[m][col + i];
    if (g.f.bias) load_values(g.f.bias + n0 + col, there, bias);
    load_residual<C>(g.f, g.M, m, n0 + col, there, residual);
    finish_chunk(g.f, g.M, g.N, m, n0 + col, v, bias, residual);
}

// ---- which tiles ---------------------------------------------------------------------------------------------------------
struct Plan {
    int bm, bn, splits, k_tiles_per_split;
    double us;                           // what it takes, by the measurements
};
constexpr int kGroups = 256;             // workgroups that fill the chip
constexpr int kLeastTiles = 4;           // of the contraction a split has

// The split of a product in tiles of one size that takes the least time: a turn of kGroups workgroups takes so many us for 1024 of the
// contraction and so many for its start and end; splits store their sums and read them again at 5 TB/s, in a launch more.
// Measured forward, us, 64 | 128 | 256, bf16 4096 x 4096 x 64: 19 | 20 | 17, x 512: 41 | 34 | 28, x 4096: 211 | 139 | 117; 2048 x 2048 x
// 64: 7.2 | 8.4 | 14, x 1024: 19 | 17 | 31; 1024 x 2048 x 2048 18 | 20 | 29; 512 x 8192 x 8192 127 | 81 | 88, 4096 x 8192 x 8192 830 | 523 | 429.
// The prices are these products'.  A backward pass of middle size takes more than they say, for its operands are read from LDS
// transposed and its two products' turns are counted one by one: 2314 x 2020 x 632 bf16, both, 48 us where this says 29.
Plan plan_with(int tile, int M, int N, int K, bool bf16) {
    const double start = tile == 64 ? 0.85 : tile == 128 ? 3.3 : 10.5;
    const double per_1024 = tile == 64 ? (bf16 ? 3.0 : 16.0) : tile == 128 ? 8.0 : 26.0;
    const int k_tiles = ceil_div(K, bf16 ? 64 : 32);
    const long long tiles = (long long)ceil_div(M, tile) * ceil_div(N, tile);
    const int most = (int)std::max<long long>(1, std::min<long long>(kGroups / tiles, k_tiles / kLeastTiles));
    Plan best{tile, tile, 1, k_tiles, 1e300};
    for (int want = 1; want <= most; want = want < most && 2 * want > most ? most : 2 * want) {
        const int per = std::max(1, ceil_div(k_tiles, want)), splits = std::max(1, ceil_div(k_tiles, per));
        double us = (double)((tiles * splits + kGroups - 1) / kGroups) * (start + per_1024 * per * (bf16 ? 64 : 32) / 1024);
        if (splits > 1) us += 3.0 + (double)splits * M * N * 8 / 5e6;
        if (us < best.us) best = Plan{tile, tile, splits, per, us};
    }
    return best;
}
// 128 x 128 and 256 x 256 tiles are for bf16 (fp32 is 5 % faster with 128 from 500 of them on, and slower below).
Plan plan_of(int M, int N, int K, bool bf16) {
    Plan best = plan_with(64, M, N, K, bf16);
    for (int tile = 128; bf16 && tile <= 256; tile *= 2) {
        const Plan p = plan_with(tile, M, N, K, bf16);
        if (p.us < best.us) best = p;
    }
    return best;
}

template <class C, int PK, int QK, bool PA, bool QA, int BM, int BN, int WM, int WN, int KS, int D, bool NARROW>
void start(const Args& a, hipStream_t s) {
    k_product<C, PK, QK, PA, QA, BM, BN, WM, WN, KS, D, NARROW>
        <<<dim3((unsigned)a.tiles_m * a.tiles_n * a.splits), 64 * WM * WN * KS, 0, s>>>(a);
}

// Whether a row of the operand is too short for whole pieces.
bool narrow(const Mat& m, bool along_own, int own, int K) { return m.kind != E4M3 && (along_own ? own : K) < 8; }

template <class C>
Args args_of(const Product& g, const Plan& p) {
    return Args{g.P, g.Q, g.M, g.N, g.K, ceil_div(g.M, p.bm), ceil_div(g.N, p.bn), ceil_div(g.K, kRowBytes / (int)sizeof(C)),
                p.splits, p.k_tiles_per_split, g.raw, g.f};
}
bool is_narrow(const Product& g) {
    return g.K == 0 || narrow(g.P, g.P_along_own, g.M, g.K) || narrow(g.Q, g.Q_along_own, g.N, g.K);
}

template <class C, int XK, int ROWS>
void few(const Args& a, hipStream_t s) {
    if (a.f.y.kind == E4M3 || (a.f.z.p && a.f.z.kind == E4M3)) {
        k_few<C, XK, ROWS, 16><<<dim3((unsigned)ceil_div(a.N, 16 * kFewOutputs)), 64 * 16, 0, s>>>(a);
    } else {
        k_few<C, XK, ROWS, 4><<<dim3((unsigned)ceil_div(a.N, 4 * kFewOutputs)), 64 * 4, 0, s>>>(a);
    }
}

template <class C, int PK, int QK, bool PA, bool QA>
hipError_t run(const Product& g, hipStream_t s) {
    if constexpr (!PA && !QA) {
        if (g.M <= kFewRows) {
            const Args a = args_of<C>(g, Plan{64, 64, 1, 1, 0});
            if (g.M == 1) few<C, PK, 1>(a, s);
            else if (g.M == 2) few<C, PK, 2>(a, s);
            else few<C, PK, 4>(a, s);
            return hipGetLastError();
        }
    }
    const Plan p = plan_of(g.M, g.N, g.K, sizeof(C) == 2);
    const Args a = args_of<C>(g, p);
    if (is_narrow(g)) {
        const Args n = args_of<C>(g, Plan{64, 64, 1, ceil_div(g.K, kRowBytes / (int)sizeof(C)), 0});
        start<C, PK, QK, PA, QA, 64, 64, 2, 2, 1, 1, true>(n, s);
        return hipGetLastError();
    }
    // Where a compute unit has one workgroup, two groups of waves share its contraction, so that a matrix core's other wave
    // multiplies while one waits, and divide the epilogue.  One group -> two, us, 60 passes at a time: fp32 256 x 4096 x 4096
    // 80 -> 76; bf16 256 x 4096 x 4096 21.1 -> 19.9, 768 x 4096 x 4096 37.1 -> 35.9, 512 x 8192 x 8192 in 8 bits 103 -> 100.  With
    // more workgroups than that there is another wave anyway.
    const bool alone = (long long)a.tiles_m * a.tiles_n * a.splits <= kGroups;
    if (p.bm == 256) {
        if constexpr (sizeof(C) == 2) start<C, PK, QK, PA, QA, 256, 256, 4, 2, 1, 1, false>(a, s);
    } else if (p.bm == 128) {
        if constexpr (sizeof(C) == 2) {
            if (alone) start<C, PK, QK, PA, QA, 128, 128, 2, 2, 2, 1, false>(a, s);
            else start<C, PK, QK, PA, QA, 128, 128, 2, 2, 1, 2, false>(a, s);
        }
    } else {
        if (alone) start<C, PK, QK, PA, QA, 64, 64, 2, 2, 2, 2, false>(a, s);
        else start<C, PK, QK, PA, QA, 64, 64, 2, 2, 1, 2, false>(a, s);
    }
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && p.splits > 1) {
        const Join j = join_of(a);
        k_join<C><<<dim3(join_blocks(j, kJoinThreads)), kJoinThreads, 0, s>>>(j);
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

// Both products of a backward pass side by side, then what their splits and db still need: three launches with the one
// before, not five or six, which is most of a small pass's time.  Tiles of one size, 64 or 128, for both.
template <class C, int T, int XK>
hipError_t both(const Product& dx, const Plan& px, const Product& dw, const Plan& pw, const ColumnSums& db, hipStream_t s) {
    const Args x = args_of<C>(dx, px), w = args_of<C>(dw, pw);
    const unsigned first = (unsigned)x.tiles_m * x.tiles_n * x.splits, all = first + (unsigned)w.tiles_m * w.tiles_n * w.splits;
    if (px.bm == 128) {
        if constexpr (sizeof(C) == 2) k_both<C, T, XK, 128, 1><<<dim3(all), 256, 0, s>>>(x, w, first);
    } else if (all <= kGroups) {
        k_both<C, T, XK, 64, 2><<<dim3(all), 512, 0, s>>>(x, w, first);
    } else {
        k_both<C, T, XK, 64, 1><<<dim3(all), 256, 0, s>>>(x, w, first);
    }
    const hipError_t e = hipGetLastError();
    const Join jx = join_of(x), jw = join_of(w);
    const unsigned bx = join_blocks(jx, kFinishThreads), bw = join_blocks(jw, kFinishThreads), bb = finish_blocks(db);
    if (e != hipSuccess || bx + bw + bb == 0) return e;
    k_join_all<C><<<dim3(bx + bw + bb), kFinishThreads, 0, s>>>(jx, bx, jw, bw, db);
    return hipGetLastError();
}
template <class C, int T>
hipError_t both_of(const Product& dx, const Plan& px, const Product& dw, const Plan& pw, const ColumnSums& db, hipStream_t s) {
    return dw.Q.kind == E4M3 ? both<C, T, E4M3>(dx, px, dw, pw, db, s) : both<C, T, T>(dx, px, dw, pw, db, s);
}

}  // namespace

// Of any plan of this product and of smaller ones: splits <= k_tiles / kLeastTiles, and splits * tiles <= kGroups.
size_t product_scratch_bytes(int M, int N, int K, bool bf16) {
    const int splits = ceil_div(K, bf16 ? 64 : 32) / kLeastTiles;
    if (splits < 2) return 0;
    return std::min((size_t)kGroups * 256 * 256, (size_t)splits * M * N) * sizeof(float);
}

hipError_t launch_product(const Product& g, hipStream_t s) {
    return g.P.kind == F32 || g.Q.kind == F32 ? by_use<float, F32>(g, s) : by_use<__bf16, BF16>(g, s);
}

hipError_t launch_backward(const Product& dx, const Product& dw, const ColumnSums& db, hipStream_t s) {
    const bool bf16 = dx.P.kind == BF16;
    if (!is_narrow(dx) && !is_narrow(dw)) {
        // one tile for both saves two launches, 4 us
        const double apart = plan_of(dx.M, dx.N, dx.K, bf16).us + plan_of(dw.M, dw.N, dw.K, bf16).us + 4.0;
        Plan x = plan_with(64, dx.M, dx.N, dx.K, bf16), w = plan_with(64, dw.M, dw.N, dw.K, bf16);
        if (bf16) {
            const Plan x2 = plan_with(128, dx.M, dx.N, dx.K, true), w2 = plan_with(128, dw.M, dw.N, dw.K, true);
            if (x2.us + w2.us < x.us + w.us) {
                x = x2;
                w = w2;
            }
        }
        if (x.us + w.us < apart)
            return bf16 ? both_of<__bf16, BF16>(dx, x, dw, w, db, s) : both_of<float, F32>(dx, x, dw, w, db, s);
    }
    hipError_t e = launch_column_finish(db, s);
    if (e == hipSuccess) e = launch_product(dx, s);
    return e == hipSuccess ? launch_product(dw, s) : e;
}

}  // namespace ops
}  // namespace lf
