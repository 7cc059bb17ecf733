// Low-rank adapters of many requests beside a shared projection (ss_adapter_add):
//     out[t] = base[t] + s_r B_a (A_a x[t])
// for the rows t of each request r, with its agent's A [rank][n_in] and
// B [n_out][rank] where the pool keeps them.
//
// Two kernels.  k_adapter_in computes A x in tiles of up to 16 or 32 rows of one request,
// the sum over n_in cut into pieces so that few rows still fill the card; the
// pieces go to the workspace in 32 bits and k_adapter_out adds them up, in the same
// order every time, when it loads them.  Both are matrix products of 16 x 16 x 32
// whose operands are rows contiguous along the summed index, so lanes load them
// from memory in the layout the instruction wants.
#include <algorithm>
#include <type_traits>

#include "ss_model.h"

namespace ss {

namespace {

constexpr int kThreads = 256;
constexpr unsigned kOutCols = 512;      // columns of out per round of a workgroup, 128 a wave

struct AdapterArgs {
    Table tab;
    const char* a;
    const char* b;
    u64 a_unit, b_unit;
    unsigned unit, rank, n_in, n_out;
    const char* x;
    const char* base;
    char* out;
    u64 x_row, base_row, out_row;       // bytes
    const float* scales;
    const unsigned* row_off;
    const unsigned* agents;
    unsigned n_rows, n_requests;
    float* low;                         // [pieces][n_rows][rank]: parts of A x
    int* unit_of;                       // [n_requests]: each request's adapter, -1 = away
    unsigned pieces, piece;             // pieces of n_in, and elements of one
    unsigned cols;                      // columns of out per workgroup
};

// Tile i of the batch: request r's tiles begin at row_off[r] / kTile + r, which leaves
// room for every request's last, partly filled tile without a pass over the offsets.
// Returns the tile's rows (0: no such tile).
template <unsigned kTile>
__device__ inline unsigned tile_of(const AdapterArgs& A, unsigned i, unsigned* r, unsigned* row0) {
    *r = wave_search(A.n_requests, i, [&](unsigned j) {
        const u64 s = (u64)A.row_off[j] / kTile + j;
        return (unsigned)(s < 0xffffffffu ? s : 0xffffffffu);
    });
    const unsigned b = A.row_off[*r], rows = request_rows(A.row_off, *r, A.n_rows);
    const u64 first = (u64)b / kTile + *r;
    if (i < first) return 0;
    const u64 at = ((u64)i - first) * kTile;
    if (at >= rows) return 0;
    *row0 = b + (unsigned)at;
    return rows - at < kTile ? rows - (unsigned)at : kTile;
}

__device__ inline int adapter_of(const AdapterArgs& A, unsigned r) {
    u64 first;
    const unsigned n = A.tab.row(A.agents[r], &first);
    return A.unit < n ? A.tab.unit(first + A.unit) : -1;
}

// The unit that k_adapter_in noted.  Offsets that break the rules can show the kernels
// different requests, so what was noted may be anything.
__device__ inline int unit_of(const AdapterArgs& A, unsigned r) {
    const int u = A.unit_of[r];
    return u >= 0 && (u64)u < A.tab.capacity ? u : -1;
}

// A workgroup per tile of up to 16 kSub rows and piece.  kTiles = rank / 16 (rounded up)
// products of 16 ranks x 16 rows for each 16 rows; the four waves take 32 elements of the
// piece in turn, as many of their reads in flight as registers hold.
template <class T, int kTiles, int kSub>
__global__ __launch_bounds__(kThreads) void k_adapter_in(AdapterArgs A) {
    __shared__ __align__(16) f32x4 s_acc[3][kTiles * kSub][64];
    unsigned r, row0;
    const unsigned piece = workgroup() % A.pieces;
    const unsigned rows = tile_of<16 * kSub>(A, workgroup() / A.pieces, &r, &row0);
    if (!rows) return;
    const int unit = adapter_of(A, r);
    if (threadIdx.x == 0) A.unit_of[r] = unit;          // the same from every tile and piece
    if (unit < 0) return;
    const unsigned lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const unsigned col = lane % 16, quad = lane / 16;
    const unsigned k0 = piece * A.piece, k1 = min(A.n_in, k0 + A.piece);
    const char* xr[kSub];
#pragma unroll
    for (int s = 0; s < kSub; ++s)
        xr[s] = A.x + (u64)(row0 + (16 * s + col < rows ? 16 * s + col : 0)) * A.x_row;
    const char* am = A.a + (u64)unit * A.a_unit;
    const char* ar[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
        ar[t] = am + (u64)(t * 16 + col < A.rank ? t * 16 + col : 0) * A.n_in * 2;
    f32x4 acc[kTiles][kSub];
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int s = 0; s < kSub; ++s) acc[t][s] = f32x4{0, 0, 0, 0};
    const u32x4 zero = {0, 0, 0, 0};
    constexpr int kSteps = kTiles == 1 ? 8 : kTiles == 2 ? 4 : kTiles == 4 ? 2 : 1;
#pragma unroll 1
    for (unsigned k = k0 + wave * 32; k < k1; k += 128 * kSteps) {
        u32x4 xf[kSteps][kSub], af[kSteps][kTiles];
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
            const unsigned at = k + 128 * u + quad * 8;
            const u64 off = (u64)(at < k1 ? at : k0) * 2;
#pragma unroll
            for (int s = 0; s < kSub; ++s) xf[u][s] = *reinterpret_cast<const u32x4*>(xr[s] + off);
#pragma unroll
            for (int t = 0; t < kTiles; ++t) af[u][t] = *reinterpret_cast<const u32x4*>(ar[t] + off);
        }
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
            const bool in = k + 128 * u + quad * 8 < k1;
#pragma unroll
            for (int s = 0; s < kSub; ++s)
                if (!in || 16 * s + col >= rows) xf[u][s] = zero;
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                if (!in || t * 16 + col >= A.rank) af[u][t] = zero;
#pragma unroll
                for (int s = 0; s < kSub; ++s) acc[t][s] = T::mma(af[u][t], xf[u][s], acc[t][s]);
            }
        }
    }
    if (wave) {
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int s = 0; s < kSub; ++s) s_acc[wave - 1][t * kSub + s][lane] = acc[t][s];
    }
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int s = 0; s < kSub; ++s) {
        if (16 * s + col >= rows) continue;
        float* to = A.low + ((u64)piece * A.n_rows + row0 + 16 * s + col) * A.rank;
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            const int i = t * kSub + s;
            const f32x4 sum = acc[t][s] + s_acc[0][i][lane] + s_acc[1][i][lane] + s_acc[2][i][lane];
            const unsigned rr = t * 16 + quad * 4;
            if (rr < A.rank) *reinterpret_cast<f32x4*>(to + rr) = sum;
        }
    }
}

// A workgroup per tile of up to 16 kSub rows and A.cols columns; a wave takes 128 of each
// 512 of them.  A x enters as two 16-bit parts, the rounded value and what the rounding left,
// so that its 32 bits count for 16 (bf16) or 22 (fp16) of them; for fp16 each row is
// first multiplied by a power of two that brings its largest value to 2^14 .. 2^15, as sums
// can pass that type's range at both ends: values down to 2^-17 of the row's largest keep 22
// bits, smaller ones are off by 2^-39 of it at most.  Up to rank 16 the summed indices
// behind the last rank are zeros that cost no reads (both parts side by side in one product,
// B read for each: 64 requests of 24 rows x 14,336 columns 48 us, as it is 44 us).
// Column n0 + 8 (lane % 16) + j is that of product j, so a lane ends up with eight
// columns next to each other of four rows and moves them in 16 bytes, with nothing
// exchanged.  HBM bounds it: base and B are asked for before the wait for A x.
template <class T, int kSub>
__global__ __launch_bounds__(kThreads, kSub == 1 ? 3 : 2) void k_adapter_out(AdapterArgs A) {
    constexpr unsigned kRows = 16 * kSub, kPitch = 2 * 128 + 8;
    __shared__ __align__(16) unsigned short s_h[kRows][kPitch];     // ranks up to 128, their rests
    __shared__ float s_scale[kRows];
    unsigned r, row0;
    const unsigned parts = (A.n_out + A.cols - 1) / A.cols;
    const unsigned rows = tile_of<kRows>(A, workgroup() / parts, &r, &row0);
    if (!rows) return;
    const int unit = unit_of(A, r);
    if (unit < 0 && A.base == A.out) return;
    const unsigned lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const unsigned col = lane % 16, quad = lane / 16;
    const unsigned n0 = workgroup() % parts * A.cols + wave * 128;       // the wave's, the same
    const unsigned n1 = min(A.n_out, workgroup() % parts * A.cols + A.cols);     // for all lanes
    const unsigned rank8 = A.rank / 8;
    const char* const bm = A.b + (u64)(unit < 0 ? 0 : unit) * A.b_unit;
    auto load_base = [&](unsigned n, u32x4 (*base)[4]) {
#pragma unroll
        for (int s = 0; s < kSub; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const unsigned t = 16 * s + 4 * quad + i;
                base[s][i] = u32x4{0, 0, 0, 0};
                if (n < n1 && t < rows)
                    base[s][i] = *reinterpret_cast<const u32x4*>(A.base + (u64)(row0 + t) * A.base_row + (u64)n * 2);
            }
    };
    // eight ranks of columns n .. n + 7 in step k
    auto load_b = [&](unsigned n, unsigned k, u32x4* b) {
        const unsigned c = 4 * k + quad;
        const bool there = n < n1 && c < rank8;
        const unsigned at = there ? (n * rank8 + c) * 16 : 0;            // below 2^31
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            b[j] = *reinterpret_cast<const u32x4*>(bm + (there ? at + j * A.rank * 2 : 0u));
            if (!there) b[j] = u32x4{0, 0, 0, 0};
        }
    };
    u32x4 base[kSub][4], bf[8];
    load_base(n0 + 8 * col, base);
    if (unit >= 0) load_b(n0 + 8 * col, 0, bf);
    if (unit >= 0) {
        // 16 lanes a row: eight ranks each
        for (unsigned i0 = 0; i0 < kRows; i0 += 16) {
            const unsigned i = i0 + threadIdx.x / 16, c = threadIdx.x % 16 * 8;
            float h[8], top = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) h[j] = 0.f;
            if (i < rows && c < A.rank)
#pragma unroll 2
                for (unsigned p = 0; p < A.pieces; ++p) {
                    const float* from = A.low + ((u64)p * A.n_rows + row0 + i) * A.rank + c;
                    const f32x4 u = *reinterpret_cast<const f32x4*>(from);
                    const f32x4 v = *reinterpret_cast<const f32x4*>(from + 4);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        h[j] += u[j];
                        h[4 + j] += v[j];
                    }
                }
#pragma unroll
            for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(h[j]));
#pragma unroll
            for (int m = 8; m; m >>= 1) top = fmaxf(top, __shfl_xor(top, m));
            float unscale = 1.f;
            if constexpr (std::is_same<T, F16>::value) {
                if (top > 0.f && top < INFINITY) {
                    const int e = min(max(ilogbf(top), -100), 100) - 14;
                    unscale = ldexpf(1.f, e);
                    const float s = ldexpf(1.f, -e);
#pragma unroll
                    for (int j = 0; j < 8; ++j) h[j] *= s;
                }
            }
            if (c == 0) s_scale[i] = unscale * (A.scales ? A.scales[r] : 1.f);
            unsigned hi[4], lo[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                hi[j] = T::pack(h[2 * j], h[2 * j + 1]);
                const float a = T::lo(hi[j]), b = T::hi(hi[j]);     // no rest of an infinity
                lo[j] = T::pack(fabsf(a) < INFINITY ? h[2 * j] - a : 0.f,
                                fabsf(b) < INFINITY ? h[2 * j + 1] - b : 0.f);
            }
            const u32x4 high = {hi[0], hi[1], hi[2], hi[3]}, rest = {lo[0], lo[1], lo[2], lo[3]};
            *reinterpret_cast<u32x4*>(&s_h[i][c]) = high;               // 0 behind the last rank
            *reinterpret_cast<u32x4*>(&s_h[i][128 + c]) = rest;
        }
        __syncthreads();
    }
#pragma unroll 1
    for (unsigned nw = n0; nw < n1; nw += kOutCols) {
        const unsigned n = nw + 8 * col;                // the lane's first of eight
        f32x4 acc[kSub][8];
#pragma unroll
        for (int t = 0; t < kSub; ++t)
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[t][j] = f32x4{0, 0, 0, 0};
        if (unit >= 0) {
            const unsigned steps = (A.rank + 31) / 32;
#pragma unroll 1
            for (unsigned k = 0; k < steps; ++k) {
#pragma unroll
                for (int t = 0; t < kSub; ++t) {
                    const unsigned short* h = &s_h[16 * t + col][32 * k + 8 * quad];
                    const u32x4 high = *reinterpret_cast<const u32x4*>(h);
#pragma unroll
                    for (int j = 0; j < 8; ++j) acc[t][j] = T::mma(high, bf[j], acc[t][j]);
                    const u32x4 rest = *reinterpret_cast<const u32x4*>(h + 128);
#pragma unroll
                    for (int j = 0; j < 8; ++j) acc[t][j] = T::mma(rest, bf[j], acc[t][j]);
                }
                if (k + 1 < steps) load_b(n, k + 1, bf);
                else load_b(n + kOutCols, 0, bf);
            }
        }
#pragma unroll
        for (int s = 0; s < kSub; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const unsigned t = 16 * s + 4 * quad + i;
                if (n >= n1 || t >= rows) continue;
                u32x4 w = base[s][i];
                if (unit >= 0) {
                    const float f = s_scale[t];
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        w[j] = T::pack(T::lo(w[j]) + f * acc[s][2 * j][i], T::hi(w[j]) + f * acc[s][2 * j + 1][i]);
                }
                store_past(w, A.out + (u64)(row0 + t) * A.out_row + (u64)n * 2);
            }
        load_base(n + kOutCols, base);
    }
}

// Decoding in bf16, and at rank 8: a workgroup per tile of up to four rows and A.cols columns.  With so few rows
// B's bytes bound it, so they are read as they lie, 16 bytes a lane, and multiplied in
// 32 bits: a column's ranks are in kSplit = rank / 8 lanes next to each other, each of
// which takes eight columns in a row, so that the sums need log2(kSplit) exchanges and
// leave in 16 bytes.  8 KB are in flight per wave while the 8 KB before are used
// (256 adapters of rank 16 by 14,336 columns: 26 us, as matrix products 38 us).
constexpr unsigned kFewRows = 4;
template <class T, int kSplit>
__global__ __launch_bounds__(kThreads, 3) void k_adapter_out_few(AdapterArgs A) {
    constexpr unsigned kCols = 512 / kSplit;            // columns of a wave's round
    unsigned r, row0;
    const unsigned parts = (A.n_out + A.cols - 1) / A.cols;
    const unsigned rows = tile_of<kFewRows>(A, workgroup() / parts, &r, &row0);
    if (!rows) return;
    const int unit = unit_of(A, r);
    if (unit < 0 && A.base == A.out) return;
    const unsigned lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const unsigned c = lane % kSplit, col = lane / kSplit * 8;          // ranks 8 c .., columns col ..
    const unsigned n0 = workgroup() % parts * A.cols + wave * kCols;
    const unsigned n1 = min(A.n_out, workgroup() % parts * A.cols + A.cols);
    if (unit < 0) {
        for (unsigned n = n0 + lane * 8; n < n1; n += 4 * kCols)
            if (lane * 8 < kCols)
                for (unsigned t = 0; t < rows; ++t)
                    *reinterpret_cast<u32x4*>(A.out + (u64)(row0 + t) * A.out_row + (u64)n * 2) =
                        *reinterpret_cast<const u32x4*>(A.base + (u64)(row0 + t) * A.base_row + (u64)n * 2);
        return;
    }
    const char* const bm = A.b + (u64)unit * A.b_unit;
    auto load = [&](unsigned nw, u32x4* b) {
        const unsigned at = nw + col < n1 ? ((nw + col) * kSplit + c) * 16 : c * 16;
#pragma unroll
        for (int j = 0; j < 8; ++j) b[j] = *reinterpret_cast<const u32x4*>(bm + (at + j * kSplit * 16));
    };
    u32x4 b[2][8];
    if (n0 < n1) load(n0, b[0]);
    const float scale = A.scales ? A.scales[r] : 1.f;
    float h[kFewRows][8];
#pragma unroll
    for (unsigned t = 0; t < kFewRows; ++t) {
#pragma unroll
        for (int j = 0; j < 8; ++j) h[t][j] = 0.f;
        if (t < rows)
            for (unsigned p = 0; p < A.pieces; ++p) {
                const float* from = A.low + ((u64)p * A.n_rows + row0 + t) * A.rank + 8 * c;
                const f32x4 u = *reinterpret_cast<const f32x4*>(from);
                const f32x4 v = *reinterpret_cast<const f32x4*>(from + 4);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    h[t][j] += u[j];
                    h[t][4 + j] += v[j];
                }
            }
    }
    auto use = [&](unsigned nw, const u32x4* b) {
        const unsigned n = nw + col;
#pragma unroll
        for (unsigned t = 0; t < kFewRows; ++t) {
            if (t >= rows) break;
            u32x4 base = {0, 0, 0, 0};
            if (c == 0 && n < n1)
                base = *reinterpret_cast<const u32x4*>(A.base + (u64)(row0 + t) * A.base_row + (u64)n * 2);
            float y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                y[j] = 0.f;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    y[j] = fmaf(T::lo(b[j][k]), h[t][2 * k], y[j]);
                    y[j] = fmaf(T::hi(b[j][k]), h[t][2 * k + 1], y[j]);
                }
            }
#pragma unroll
            for (int m = kSplit / 2; m; m >>= 1)
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] += __shfl_xor(y[j], m);
            if (c == 0 && n < n1) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    base[j] = T::pack(T::lo(base[j]) + scale * y[2 * j], T::hi(base[j]) + scale * y[2 * j + 1]);
                *reinterpret_cast<u32x4*>(A.out + (u64)(row0 + t) * A.out_row + (u64)n * 2) = base;
            }
        }
    };
#pragma unroll 1
    for (unsigned nw = n0; nw < n1; nw += 8 * kCols) {
        if (nw + 4 * kCols < n1) load(nw + 4 * kCols, b[1]);
        use(nw, b[0]);
        if (nw + 4 * kCols >= n1) break;
        if (nw + 8 * kCols < n1) load(nw + 8 * kCols, b[0]);
        use(nw + 4 * kCols, b[1]);
    }
}

template <class T, int kSplit>
void out_few_launch(const AdapterArgs& A, hipStream_t st) {
    // two rounds a wave where there are workgroups enough: each reads its way to the
    // adapter before it streams (256 rows x 14,336 columns: one round 44 us, two 38 us,
    // four 40 us; 16 rows x 4,096: one 11.6 us, two 12.2 us)
    AdapterArgs B = A;
    const unsigned tiles = A.n_rows / kFewRows + A.n_requests, round = 4 * 512 / kSplit;
    B.cols = (u64)tiles * ((A.n_out + round - 1) / round) >= 1024 ? 2 * round : round;
    hipLaunchKernelGGL((k_adapter_out_few<T, kSplit>), grid_of((A.n_out + B.cols - 1) / B.cols * tiles),
                       dim3(kThreads), 0, st, B);
}

template <class T, int kSub>
void out_launch(const AdapterArgs& A, hipStream_t st) {
    const unsigned tiles = A.n_rows / (16 * kSub) + A.n_requests;
    // a workgroup reads its way to the adapter before it streams, so it takes several
    // 512 columns where there are more workgroups than run at a time
    const unsigned pieces = (A.n_out + kOutCols - 1) / kOutCols;
    // (all at once: two or three a compute unit), of about the same length each
    const unsigned most = kSub == 1 ? 768 : 512;
    const unsigned rounds = (unsigned)(((u64)pieces * tiles + 4 * most - 1) / (4 * most));
    const unsigned want = std::max(1u, (unsigned)((u64)most * rounds / tiles));      // pieces' groups
    const unsigned each = std::max(1u, (pieces + want - 1) / want);
    AdapterArgs B = A;
    B.cols = kOutCols * each;
    const dim3 grid = grid_of((pieces + each - 1) / each * tiles), block(kThreads);
    hipLaunchKernelGGL((k_adapter_out<T, kSub>), grid, block, 0, st, B);
}

// Whether requests have more rows than a tile of 16 as a rule: tiles of 32 then read A and
// B half as often (4,096 x 14,336: 64 requests of 20 rows at rank 64 70 us, in tiles of 16
// rows 93 us; of 24 rows at rank 16 44 and 58 us; of 16 rows 40 us, in tiles of 16 38 us).
bool long_rows(u64 n_rows, u64 n_requests) { return n_rows > 16 * n_requests; }

template <class T, int kSub>
void in_launch(const AdapterArgs& A, hipStream_t st) {
    const dim3 grid = grid_of(A.pieces * (A.n_rows / (16 * kSub) + A.n_requests)), block(kThreads);
    switch ((A.rank + 15) / 16) {
        case 1: hipLaunchKernelGGL((k_adapter_in<T, 1, kSub>), grid, block, 0, st, A); break;
        case 2: hipLaunchKernelGGL((k_adapter_in<T, 2, kSub>), grid, block, 0, st, A); break;
        case 3:
        case 4: hipLaunchKernelGGL((k_adapter_in<T, 4, kSub>), grid, block, 0, st, A); break;
        default: hipLaunchKernelGGL((k_adapter_in<T, 8, kSub>), grid, block, 0, st, A); break;
    }
}

template <class T>
void adapter_launch(const AdapterArgs& A, hipStream_t st) {
    if (long_rows(A.n_rows, A.n_requests)) {
        in_launch<T, 2>(A, st);
        return out_launch<T, 2>(A, st);
    }
    in_launch<T, 1>(A, st);
    // Up to one row a request as a rule no product of 16 rows is worth its reads: bf16, 256
    // requests, 4,096 x 14,336, an adapter each: rank 8 32 us, as products 39 us; 16 47 and
    // 55 us; 32 79 and 80 us; 64 143 and 170 us; 128 278 and 339 us (64 requests: 16 and 18,
    // 20 and 21, 29 and 25, 50 and 46, 87 and 86 us; eight: 11 us either way, from rank 64 on 14
    // and 14, 18 and 20 us).  fp16 halves take a conversion each, for which registers do not
    // suffice from rank 16 on (256 requests: rank 8 30 and 40 us, 16 76 and 55 us, 32 120 and
    // 80 us, 64 197 and 169 us, 128 396 and 339 us), so they go this way at rank 8 only.
    // With two rows a request it wins less where there are many (bf16, 256 requests: rank 16
    // 50 and 54 us, 32 82 and 75 us, 64 145 and 152 us) than it loses where there are few
    // (eight: 13.1 and 11.3 us, 17.6 and 12.0 us, 19.8 and 14.4 us).
    if (A.n_rows <= A.n_requests) {
        if (A.rank == 8) return out_few_launch<T, 1>(A, st);
        if constexpr (std::is_same<T, Bf16>::value) {
            switch (A.rank) {
                case 16: return out_few_launch<T, 2>(A, st);
                case 32: return out_few_launch<T, 4>(A, st);
                case 64: return out_few_launch<T, 8>(A, st);
                case 128: return out_few_launch<T, 16>(A, st);
            }
        }
    }
    out_launch<T, 1>(A, st);
}

// n_in is cut into pieces of at least 256 elements (two rounds of the four waves)
// until about four workgroups a compute unit run (256 adapters of 4,096 x 14,336: 38 us,
// eight 47 us), two for long rows, whose pieces cost more to add up (8 prompts of 2,048 x
// 8,192, rank 64: 54 us, one 57 us).
void pieces_of(u64 n_rows, u64 n_requests, u64 n_in, unsigned* pieces, unsigned* piece) {
    const bool rows = long_rows(n_rows, n_requests);
    const u64 tiles = n_rows / (rows ? 32 : 16) + n_requests, most = rows ? 512 : 1024;
    const u64 want = std::max<u64>(1, std::min<u64>((most + tiles - 1) / tiles, (n_in + 255) / 256));
    const u64 len = ((n_in + want - 1) / want + 127) / 128 * 128;
    *piece = (unsigned)len;
    *pieces = (unsigned)((n_in + len - 1) / len);
}

// The parts of A x, then the requests' units.
u64 low_bytes(u64 n_rows, u64 n_requests, u64 n_in, u64 rank) {
    unsigned pieces, piece;
    pieces_of(n_rows, n_requests, n_in, &pieces, &piece);
    return pieces * n_rows * rank * 4;
}

ss_status adapter_args(const ss_adapters* a) {
    if (!a) return set_err(SS_ERR_ARG, "adapters is NULL");
    const ss_status s = table_args(a->units, a->agent_off, a->n_agents, a->n_entries, a->capacity_units);
    if (s != SS_OK) return s;
    if (!a->a || !a->b || ((reinterpret_cast<uintptr_t>(a->a) | reinterpret_cast<uintptr_t>(a->b)) & 15))
        return set_err(SS_ERR_ARG, "adapters a and b must be 16-byte aligned pointers");
    if (a->rank < 8 || a->rank > 128 || a->rank % 8)
        return set_err(SS_ERR_ARG, "rank must be a multiple of 8 in [8, 128]");
    for (u64 n : {a->n_in, a->n_out})
        if (n < 8 || n % 8 || n >= (1u << 24))
            return set_err(SS_ERR_ARG, "n_in and n_out must be multiples of 8 in [8, 2^24)");
    if (a->type != SS_BF16 && a->type != SS_F16)
        return set_err(SS_ERR_ARG, "adapters must be SS_BF16 or SS_F16, not type %u", a->type);
    if (a->a_unit_bytes % 16 || a->b_unit_bytes % 16 || a->a_unit_bytes >= (1ull << 31) ||
        a->b_unit_bytes >= (1ull << 31))
        return set_err(SS_ERR_ARG, "adapter byte distances must be multiples of 16 below 2^31");
    if (2ull * a->rank * std::max(a->n_in, a->n_out) >= (1ull << 31))
        return set_err(SS_ERR_ARG, "a matrix is too large (2^31 bytes)");
    if (a->capacity_units > 1 && (a->a_unit_bytes < 2ull * a->rank * a->n_in ||
                                  a->b_unit_bytes < 2ull * a->rank * a->n_out))
        return set_err(SS_ERR_ARG, "a matrix does not fit into a unit's chunk");
    return SS_OK;
}

}  // namespace

}  // namespace ss

using namespace ss;

extern "C" {

uint64_t ss_adapter_add_workspace(const ss_adapters* adapters, uint32_t n_rows, uint32_t n_requests) {
    if (adapter_args(adapters) != SS_OK || n_rows == 0 || n_requests == 0 || n_rows >= (1u << 31) ||
        n_requests >= (1u << 20))
        return 0;
    return low_bytes(n_rows, n_requests, adapters->n_in, adapters->rank) + 4ull * n_requests;
}

ss_status ss_adapter_add(const ss_adapters* adapters, const ss_batch* batch, const void* x,
                         const void* base, void* out, uint64_t x_stride, uint64_t base_stride,
                         uint64_t out_stride, const float* scales, void* workspace,
                         uint64_t workspace_bytes, void* stream) {
    ss_status s = adapter_args(adapters);
    if (s == SS_OK) s = batch_args(batch, false, false);
    if (s != SS_OK) return s;
    const u64 rows = batch->n_rows;
    if (rows == 0 || batch->n_requests == 0) return SS_OK;
    const unsigned n_in = adapters->n_in, n_out = adapters->n_out;
    if ((s = rows_args("x", x, rows, 1, n_in, x_stride, n_in, false)) != SS_OK ||
        (s = rows_args("base", base, rows, 1, n_out, base_stride, n_out, false)) != SS_OK ||
        (s = rows_args("out", out, rows, 1, n_out, out_stride, n_out, true)) != SS_OK)
        return s;
    // workgroups of the kernel that has most
    if ((rows / kFewRows + batch->n_requests) * ((n_out + 255) / 256) >= (1ull << 31))
        return set_err(SS_ERR_ARG, "n_rows * n_out is too large");
    const u64 x_bytes = rows_bytes(rows, 1, n_in, x_stride, 0);
    const u64 base_bytes = rows_bytes(rows, 1, n_out, base_stride, 0);
    const u64 out_bytes = rows_bytes(rows, 1, n_out, out_stride, 0);
    const uintptr_t x0 = reinterpret_cast<uintptr_t>(x), b0 = reinterpret_cast<uintptr_t>(base);
    const uintptr_t o0 = reinterpret_cast<uintptr_t>(out);
    if (x0 < o0 + out_bytes && o0 < x0 + x_bytes) return set_err(SS_ERR_ARG, "out overlaps x");
    if (!(b0 == o0 && base_stride == out_stride) && b0 < o0 + out_bytes && o0 < b0 + base_bytes)
        return set_err(SS_ERR_ARG, "out overlaps base without being it");
    const u64 need = ss_adapter_add_workspace(adapters, batch->n_rows, batch->n_requests);
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15))
        return set_err(SS_ERR_ARG, "workspace must be a 16-byte aligned pointer");
    if (workspace_bytes < need)
        return set_err(SS_ERR_ARG, "workspace_bytes %llu < %llu", (unsigned long long)workspace_bytes,
                       (unsigned long long)need);
    DeviceMemory mem;
    if ((s = mem.current()) != SS_OK ||
        (s = table_memory(adapters->units, adapters->agent_off, adapters->n_agents, adapters->n_entries,
                          mem)) != SS_OK ||
        (s = batch_memory(batch, false, false, mem)) != SS_OK)
        return s;
    const u64 last = adapters->capacity_units - 1;
    if (!mem.has(adapters->a, last * adapters->a_unit_bytes + 2ull * adapters->rank * n_in))
        return device_error("adapters a", mem.dev);
    if (!mem.has(adapters->b, last * adapters->b_unit_bytes + 2ull * adapters->rank * n_out))
        return device_error("adapters b", mem.dev);
    if (!mem.has(x, x_bytes)) return device_error("x", mem.dev);
    if (!mem.has(base, base_bytes)) return device_error("base", mem.dev);
    if (!mem.has(out, out_bytes)) return device_error("out", mem.dev);
    if (scales && !mem.has(scales, (u64)batch->n_requests * 4))
        return device_error("scales", mem.dev);
    if (!mem.has(workspace, need)) return device_error("workspace", mem.dev);
    AdapterArgs A{};
    A.tab = table_of(adapters->units, adapters->agent_off, adapters->n_agents, adapters->n_entries,
                     adapters->capacity_units);
    A.a = static_cast<const char*>(adapters->a);
    A.b = static_cast<const char*>(adapters->b);
    A.a_unit = adapters->a_unit_bytes;
    A.b_unit = adapters->b_unit_bytes;
    A.unit = adapters->unit;
    A.rank = adapters->rank;
    A.n_in = n_in;
    A.n_out = n_out;
    A.x = static_cast<const char*>(x);
    A.base = static_cast<const char*>(base);
    A.out = static_cast<char*>(out);
    A.x_row = 2 * x_stride;
    A.base_row = 2 * base_stride;
    A.out_row = 2 * out_stride;
    A.scales = scales;
    A.row_off = batch->row_off;
    A.agents = batch->agents;
    A.n_rows = batch->n_rows;
    A.n_requests = batch->n_requests;
    A.low = static_cast<float*>(workspace);
    A.unit_of = reinterpret_cast<int*>(static_cast<char*>(workspace) +
                                       low_bytes(rows, batch->n_requests, n_in, adapters->rank));
    pieces_of(rows, batch->n_requests, n_in, &A.pieces, &A.piece);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (adapters->type == SS_BF16) adapter_launch<Bf16>(A, st);
    else adapter_launch<F16>(A, st);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return set_err(SS_ERR_HIP, "adapter kernels: %s", hipGetErrorString(e));
    return SS_OK;
}

}  // extern "C"
