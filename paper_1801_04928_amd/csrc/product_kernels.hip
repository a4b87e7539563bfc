// The matrix product of residual blocks,  C[m][n] = sum_q P(m,q) Q(n,q)  with fp32 sums, in its three uses:
//   forward   P = x  (contiguous along q)          Q = w (contiguous along q)          C = z -> bias, activation, residual
//   dx        P = dz (contiguous along q)          Q = w (contiguous along its own n)
//   dw        P = dz (contiguous along its own m)  Q = x (contiguous along its own n)
// Operands are fp32 or bf16; x may be in 8 bits, whose values are bf16 numbers: they are made when a tile is laid into LDS,
// and the matrix instructions see no difference.
#include "activation.h"
#include "chunks.h"

#include <algorithm>
#include <cstdlib>
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
template <> struct Raw<F32, 8> { v4f a[2]; };
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
// LDS of a tile contiguous along q: [i][q], rows of eight 16-byte pieces, piece p of row i at place p ^ (i & 7): the rows that a
// matrix operand takes its pieces from then lie in different banks.  Contiguous along i: [q][i]; bf16 is read there by
// transposing loads, eight rows of 64 bytes at a time (q, q+1, q+2, q+3 and eight further), whose 64-byte segments
// change places the same way.
template <class C, int KIND, bool ALONG, int I, int THREADS, bool NARROW>
struct Tile {
    static constexpr int BK = kRowBytes / (int)sizeof(C);
    static constexpr int kElems = I * BK;
    static constexpr int kPiece = KIND == E4M3 && sizeof(C) == 2 ? 16 : 8;
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

    // What stays the same from k-tile to k-tile: of every piece, its row's offset in the tile (contiguous along q) or its column's
    // (along i), and the same for its scale.
    unsigned at[kPieces], scale_at[KIND == E4M3 ? kPieces : 1];
    __device__ __forceinline__ void begin(const Mat& m, int t, int i0, int I_all) {
#pragma unroll
        for (int u = 0; u < kPieces; ++u) {
            int i, q;
            place(t, u, i, q);
            const int row = min(i, I_all - 1 - i0), col = min(i0 + i, in_memory(I_all) - kPiece);
            at[u] = ALONG ? (unsigned)col * kElemBytes : (unsigned)row * (unsigned)m.ld * kElemBytes;
            if constexpr (KIND == E4M3) scale_at[u] = ALONG ? (unsigned)(col / kGroup) : (unsigned)row * (unsigned)m.scale_ld;
        }
    }
    // I_all: rows of the operand; q_end: where this workgroup's part of the contraction ends.  live: all ones, or zero past its last
    // tile (anything may be loaded then, nothing looks at it).
    __device__ __forceinline__ void load(const Mat& m, int t, int i0, int I_all, int q0, int q_end, unsigned live) {
        if constexpr (NARROW) {
            if (live) load_elements(m, t, i0, I_all, q0, q_end);
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
            const unsigned row = ALONG ? min(q, q_end - 1 - q_first) : 0;
            const unsigned col = ALONG ? 0 : min(q0 + q, in_memory(q_end) - kPiece);
            const unsigned off = (at[u] + (ALONG ? row * ld : col * kElemBytes)) & live;
            if constexpr (KIND == F32) {
                r[u].a[0] = *as_global<const any_v4f>(base + off);
                r[u].a[1] = *as_global<const any_v4f>(base + off + 16);
            } else if constexpr (KIND == BF16) {
                r[u].a = __builtin_bit_cast(v4u, *as_global<const any_v8bf>(base + off));
            } else {
                if constexpr (kPiece == 16) r[u].a = *as_global<const v4u>(base + off);
                else r[u].a = *as_global<const v2u>(base + off);
                r[u].byte = *as_global<const uint8_t>(scales + ((scale_at[u] + (ALONG ? row * scale_ld : col / kGroup)) & live));
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
                float v[8];
                typedef typename Stored<KIND>::type T;
                load_values((const T*)m.p + row * m.ld + col, n, v);
                if constexpr (KIND == F32) {
                    r[u].a[0] = v4f{v[0], v[1], v[2], v[3]};
                    r[u].a[1] = v4f{v[4], v[5], v[6], v[7]};
                } else {
                    v8bf b;
#pragma unroll
                    for (int e = 0; e < 8; ++e) b[e] = (__bf16)v[e];
                    r[u].a = __builtin_bit_cast(v4u, b);
                }
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
                shift_down(r[u].a, dead ? 8 : s);
            }
        }
    }
    static __device__ __forceinline__ bool at_end(int i0, int I_all, int q0, int q_end) {
        return q0 + BK > q_end || (ALONG && i0 + I > I_all);
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
    __device__ __forceinline__ void store(C* s, int t) const {
#pragma unroll
        for (int u = 0; u < kPieces; ++u) {
            int i, q;
            place(t, u, i, q);
            if constexpr (KIND == BF16) {
                *reinterpret_cast<v4u*>(s + (ALONG ? at_along_i(q, i) : at_along_q(i, q / 8))) = r[u].a;
            } else if constexpr (sizeof(C) == 2) {
                const float scale = scale_value(r[u].byte);
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
                if constexpr (KIND == F32) {
                    a = r[u].a[0];
                    b = r[u].a[1];
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
template <int ACT>
__device__ __forceinline__ void activate_all(float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = activate(ACT, v[i]);
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
    switch (f.act) {                        // (the branch is outside the loop over the eight values)
        case SIGMOID: activate_all<SIGMOID>(v); break;
        case RELU: activate_all<RELU>(v); break;
        case SILU: activate_all<SILU>(v); break;
        case GELU: activate_all<GELU>(v); break;
        default: break;
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
// tiles of BM x BN; KS groups of WM x WN waves share a tile's contraction
// ================================================================================================
// A group walks every KS-th k-tile of its workgroup's part.  D k-tiles of it are under way in registers, one lies in LDS for the
// multiplications, and one is laid beside it meanwhile: one barrier a k-tile.
template <class C, int BM, int BN, int KS>
constexpr int kLdsElems = KS * 2 * (BM + BN) * (kRowBytes / (int)sizeof(C));

template <class C, int PK, int QK, bool P_ALONG, bool Q_ALONG, int BM, int BN, int WM, int WN, int KS, int D, bool NARROW>
__device__ __forceinline__ void product_tile(const Args& g, unsigned block, C* lds) {
    constexpr int kThreads = 64 * WM * WN;
    typedef Tile<C, PK, P_ALONG, BM, kThreads, NARROW> TP;
    typedef Tile<C, QK, Q_ALONG, BN, kThreads, NARROW> TQ;
    constexpr int BK = TP::BK, MT = BM / WM / 32, NT = BN / WN / 32;
    constexpr int kBuffer = TP::kElems + TQ::kElems;
    // rows of the epilogue's staging: with groups all of the tile's, else as many of a wave's own as fit
    constexpr int kStageLd = KS > 1 ? BN + 4 : NT * 32 + 4;
    constexpr int kStageRows = KS > 1 ? BM : WM * WN * 32 * kStageLd * 4 <= 2 * kBuffer * (int)sizeof(C) ? 32 : 16;
    static_assert((KS > 1 ? 1 : WM * WN) * kStageRows * kStageLd * 4 <= 2 * kBuffer * (int)sizeof(C), "the staging fits");

    const int t = threadIdx.x % kThreads, group = __builtin_amdgcn_readfirstlane(threadIdx.x / kThreads);
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

    v16f acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;

    TP tp[D];
    TQ tq[D];
    auto q_of = [&](int turn) { return (kt0 + turn * KS + group) * BK; };
#pragma unroll
    for (int d = 0; d < D; ++d) {
        tp[d].begin(g.P, t, m0, g.M);
        tq[d].begin(g.Q, t, n0, g.N);
    }
    auto request = [&](int d, int turn) {
        // (an operand of the address, not a branch around the load)
        const unsigned live = __builtin_amdgcn_readfirstlane(turn < turns ? ~0u : 0u);
        tp[d].load(g.P, t, m0, g.M, q_of(turn), q_end, live);
        tq[d].load(g.Q, t, n0, g.N, q_of(turn), q_end, live);
    };
    C* const mine = lds + group * 2 * kBuffer;
    auto lay = [&](int d, int turn) {
        const int q0 = q_of(turn);
        if (TP::at_end(m0, g.M, q0, q_end)) tp[d].mend(t, m0, g.M, q0, q_end);
        if (TQ::at_end(n0, g.N, q0, q_end)) tq[d].mend(t, n0, g.N, q0, q_end);
        C* const buffer = mine + (turn & 1) * kBuffer;
        tp[d].store(buffer, t);
        tq[d].store(buffer + TP::kElems, t);
    };
    auto multiply = [&](int turn) {
        const C* const sp = mine + (turn & 1) * kBuffer;
        const C* const sq = sp + TP::kElems;
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
    };
    if (turns > 0) {
#pragma unroll
        for (int d = 0; d < D; ++d) request(d, d);
        lay(0, 0);
        request(0, D);
        __syncthreads();
        for (int turn = 0;; turn += D) {
#pragma unroll
            for (int d = 0; d < D; ++d) {
                // k-tile turn + d + 1 goes to the buffer that was read before the last barrier
                lay((d + 1) % D, turn + d + 1);
                request((d + 1) % D, turn + d + 1 + D);
                multiply(turn + d);
                __syncthreads();
                if (turn + d + 1 == turns) goto multiplied;
            }
        }
    }
multiplied:

    // Accumulator element e of lane (r32, half) of tile (i, j) is C[.. 32 i + 8 (e / 4) + 4 half + e % 4][.. 32 j + r32].  Rows turn
    // through LDS, so that a lane holds eight consecutive columns.
    const int r32 = lane & 31, half = lane >> 5;
    auto finish = [&](int m, int n, float (&v)[8]) {
        if (g.splits > 1) {
            if (m < g.M && n < g.N) store_values(g.raw + ((size_t)split * g.M + m) * g.N + n, g.N - n, v);
        } else {
            finish_chunk(g.f, g.M, g.N, m, n, v);
        }
    };
    if constexpr (KS > 1) {
        // every group lays its sums down, all threads add them up
        float* stage = reinterpret_cast<float*>(mine);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    stage[(wm + 32 * i + 8 * (e >> 2) + 4 * half + (e & 3)) * kStageLd + wn + 32 * j + r32] = acc[i][j][e];
        __syncthreads();
        constexpr int kChunks = BM * BN / kChunk;
        // (one copy of what follows in the code, here and below: an epilogue unrolled is larger than the instruction cache)
#pragma unroll 1
        for (int chunk = threadIdx.x; chunk < kChunks; chunk += kThreads * KS) {
            const int row = chunk / (BN / kChunk), col = chunk % (BN / kChunk) * kChunk;
            float v[8] = {};
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const float* from = reinterpret_cast<const float*>(lds + k * 2 * kBuffer) + row * kStageLd + col;
                const v4f lo = *reinterpret_cast<const v4f*>(from), hi = *reinterpret_cast<const v4f*>(from + 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) { v[i] += lo[i]; v[4 + i] += hi[i]; }
            }
            finish(m0 + row, n0 + col, v);
        }
    } else {
        // in LDS of the wave's own: nobody waits
        float* stage = reinterpret_cast<float*>(lds) + wave * kStageRows * kStageLd;
        constexpr int kAcross = NT * 4, kDown = 64 / kAcross;      // lanes along a row, rows at once
        constexpr int kElems = kStageRows / 2;                     // accumulator elements that hold these rows
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int h = 0; h < 16 / kElems; ++h) {
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int e = 0; e < kElems; ++e)
                        stage[(8 * (e >> 2) + 4 * half + (e & 3)) * kStageLd + 32 * j + r32] = acc[i][j][kElems * h + e];
                __builtin_amdgcn_wave_barrier();
#pragma unroll 1
                for (int row = lane / kAcross; row < kStageRows; row += kDown) {
                    const int col = lane % kAcross * kChunk;
                    const v4f lo = *reinterpret_cast<const v4f*>(stage + row * kStageLd + col);
                    const v4f hi = *reinterpret_cast<const v4f*>(stage + row * kStageLd + col + 4);
                    float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
                    finish(m0 + wm + 32 * i + kStageRows * h + row, n0 + wn + col, v);
                }
                __builtin_amdgcn_wave_barrier();
            }
    }
}

template <class C, int PK, int QK, bool P_ALONG, bool Q_ALONG, int BM, int BN, int WM, int WN, int KS, int D, bool NARROW>
__global__ __launch_bounds__(64 * WM * WN * KS) void k_product(const Args g) {
    __shared__ __attribute__((aligned(16))) C lds[kLdsElems<C, BM, BN, KS>];
    product_tile<C, PK, QK, P_ALONG, Q_ALONG, BM, BN, WM, WN, KS, D, NARROW>(g, blockIdx.x, lds);
}

// Both products of a backward pass in one launch: the first `first` workgroups take dx, the others dw.
template <class C, int T, int XK, int BM, int BN, int WM, int WN, int KS, int D>
__global__ __launch_bounds__(64 * WM * WN * KS) void k_both(const Args dx, const Args dw, unsigned first) {
    __shared__ __attribute__((aligned(16))) C lds[kLdsElems<C, BM, BN, KS>];
    if (blockIdx.x < first) product_tile<C, T, T, false, true, BM, BN, WM, WN, KS, D, false>(dx, blockIdx.x, lds);
    else product_tile<C, T, XK, true, true, BM, BN, WM, WN, KS, D, false>(dw, blockIdx.x - first, lds);
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
struct Plan { int bm, bn, groups, splits, k_tiles_per_split; };
constexpr int kGroups = 256;             // workgroups that fill the chip
constexpr int kLeastTiles = 4;           // of the contraction a split has

Plan plan_of(int M, int N, int K, bool bf16) {
    const int k_tiles = ceil_div(K, bf16 ? 64 : 32);
    Plan p{64, 64, 1, 1, k_tiles};
    const auto tiles_of = [&](int b) { return (long long)ceil_div(M, b) * ceil_div(N, b); };
    if (const char* e = getenv("PLAN")) { p.bm = p.bn = atoi(e); if (p.bm > 256) { p.bm = p.bn = 64; p.groups = 4; } }
    else if (bf16 && tiles_of(256) >= 200) p.bm = p.bn = 256;
    else if (tiles_of(128) >= 128) p.bm = p.bn = 128;
    const long long tiles = tiles_of(p.bm);
    int want = (int)std::max<long long>(1, std::min<long long>(kGroups / tiles, k_tiles / kLeastTiles));
    if (const char* e = getenv("SPLIT")) want = std::max(1, std::min(atoi(e), want));
    if (want > 1) {
        p.k_tiles_per_split = ceil_div(k_tiles, want);
        p.splits = ceil_div(k_tiles, p.k_tiles_per_split);
    }
    return p;
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

template <class C, int PK, int QK, bool PA, bool QA>
hipError_t run(const Product& g, hipStream_t s) {
    const Plan p = plan_of(g.M, g.N, g.K, sizeof(C) == 2);
    const Args a = args_of<C>(g, p);
    if (is_narrow(g)) {
        const Args n = args_of<C>(g, Plan{64, 64, 1, 1, ceil_div(g.K, kRowBytes / (int)sizeof(C))});
        start<C, PK, QK, PA, QA, 64, 64, 2, 2, 1, 1, true>(n, s);
        return hipGetLastError();
    }
    if (p.bm == 256) {
        if constexpr (sizeof(C) == 2) start<C, PK, QK, PA, QA, 256, 256, 4, 2, 1, 1, false>(a, s);
    } else if (p.bm == 128) {
        start<C, PK, QK, PA, QA, 128, 128, 2, 2, 1, 2, false>(a, s);
    } else if (p.groups == 4) {
        start<C, PK, QK, PA, QA, 64, 64, 2, 2, 4, 2, false>(a, s);
    } else {
        start<C, PK, QK, PA, QA, 64, 64, 2, 2, 1, 4, false>(a, s);
    }
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

template <class C, int T, int XK>
hipError_t both(const Product& dx, const Product& dw, int groups, hipStream_t s) {
    const Args x = args_of<C>(dx, plan_of(dx.M, dx.N, dx.K, sizeof(C) == 2));
    const Args w = args_of<C>(dw, plan_of(dw.M, dw.N, dw.K, sizeof(C) == 2));
    const unsigned first = (unsigned)x.tiles_m * x.tiles_n, all = first + (unsigned)w.tiles_m * w.tiles_n;
    if (groups == 4) k_both<C, T, XK, 64, 64, 2, 2, 4, 2><<<dim3(all), 1024, 0, s>>>(x, w, first);
    else k_both<C, T, XK, 64, 64, 2, 2, 1, 4><<<dim3(all), 256, 0, s>>>(x, w, first);
    return hipGetLastError();
}
template <class C, int T>
hipError_t both_of(const Product& dx, const Product& dw, int groups, hipStream_t s) {
    return dw.Q.kind == E4M3 ? both<C, T, E4M3>(dx, dw, groups, s) : both<C, T, T>(dx, dw, groups, s);
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

hipError_t launch_both(const Product& dx, const Product& dw, hipStream_t s) {
    const bool bf16 = dx.P.kind == BF16;
    const Plan x = plan_of(dx.M, dx.N, dx.K, bf16), w = plan_of(dw.M, dw.N, dw.K, bf16);
    if (x.bm == 64 && w.bm == 64 && x.groups == w.groups && x.splits == 1 && w.splits == 1 && !is_narrow(dx) && !is_narrow(dw))
        return bf16 ? both_of<__bf16, BF16>(dx, dw, x.groups, s) : both_of<float, F32>(dx, dw, x.groups, s);
    const hipError_t e = launch_product(dx, s);
    return e == hipSuccess ? launch_product(dw, s) : e;
}

}  // namespace ops
}  // namespace lf
