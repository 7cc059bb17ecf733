// Attention of a ragged batch over a pool's KV pages, with prefixes that groups
// of requests share (ss_prefix_attention).
//
// Work is cut into items.  A stack is a list of rows that read the same keys: a
// request's rows over its own tokens, or all rows of a group over the group's
// prefix, so that the prefix is read once per tile of rows instead of once per
// request.  Row m of a stack is query row m / G, query head m % G of the G query
// heads of a key/value head.  An item is (stack, tile of rows, range of keys, key/value
// head).  k_attend_plan lists the items, k_attend computes them with a running
// maximum and sum, k_attend_join joins the parts of rows that several items share:
//     m = max_i m_i,  l = sum_i l_i 2^(m_i - m),  out = sum_i o_i 2^(m_i - m) / l.
#include <algorithm>
#include <cmath>

#include "ss_model.h"

namespace ss {

namespace {

constexpr unsigned kNone = 0xffffffffu;
constexpr unsigned kBlock = 64;             // keys of one step of an item
constexpr unsigned kTarget = 1024;          // items that a call is split into at least, if it can
constexpr unsigned kMinBlocks = 4;          // and key blocks that an item has at least
constexpr unsigned kTileRows = 16;

struct Stack {
    u64 first[2];       // table entries of the two segments of keys: prefix, own tokens
    u64 part;           // first partial row, or ~0: one item per tile, written straight out
    unsigned keys[2];   // tokens with a page
    unsigned row0, rows;
    int see;            // row i of the stack sees own tokens 0 .. see + i
    unsigned chunk;     // key blocks of an item
    unsigned splits;    // items per tile and head
    unsigned pool;      // a request's stack: the stack of its group's prefix, or kNone
};
static_assert(sizeof(Stack) == 56, "three words and eight halves");

struct AttendArgs {
    Table tab;
    const char* k;
    const char* v;
    u64 k_unit, v_unit, token_bytes, head_bytes, scale_off;
    const char* q;
    char* out;
    float* lse;
    u64 q_row, q_head, out_row, out_head;       // bytes
    const unsigned* row_off;
    const unsigned* agents;
    const unsigned* lens;
    const unsigned* group_off;
    const unsigned* prefix_agents;
    const unsigned* prefix_lens;
    unsigned n_rows, n_requests, n_groups;
    unsigned n_heads, per;                      // key/value heads, query heads of each
    unsigned dim, shift;
    float scale;                                // times log2(e)
    // workspace
    unsigned* n_items;                          // items per head; 1 where the offsets are valid
    unsigned* item0;                            // [stacks + 1] first item of each stack
    Stack* stacks;                              // [n_requests + n_groups]
    float* part_o;                              // [part_rows][padded dim]
    float2* part_ml;                            // [part_rows] maximum (log2), sum
    u64 part_rows;
};

constexpr int kPlanThreads = 1024;

// A request's group (kNone = none): groups are searched as the requests are.
__device__ unsigned group_of(const AttendArgs& A, unsigned r) {
    unsigned lo = 0, hi = A.n_groups;           // largest g with group_off[g] <= r
    while (hi - lo > 1) {
        const unsigned mid = (lo + hi) / 2;
        if (A.group_off[mid] <= r) lo = mid;
        else hi = mid;
    }
    if (hi <= lo) return kNone;
    return A.group_off[lo] <= r && r < A.group_off[lo + 1] && A.group_off[lo + 1] <= A.n_requests
        ? lo : kNone;
}

__device__ unsigned tokens_with_page(const AttendArgs& A, unsigned agent, unsigned len, u64* first) {
    const u64 most = (u64)A.tab.row(agent, first) << A.shift;
    return (unsigned)(len < most ? len : most);
}

// Whether the prefix of group g is read by a stack of its own: where several
// requests share it and are so short that a tile of rows holds more than one.
// Otherwise each request reads prefix and own tokens in one go, without parts.
__device__ bool pooled(const AttendArgs& A, unsigned g, unsigned* row0, unsigned* rows) {
    const unsigned b = A.group_off[g], e = A.group_off[g + 1];
    *row0 = *rows = 0;
    if (b >= e || e > A.n_requests) return false;
    const unsigned r0 = A.row_off[b], r1 = A.row_off[e];
    if (r0 >= r1 || r1 > A.n_rows) return false;
    *row0 = r0;
    *rows = r1 - r0;
    return e - b > 1 && (u64)*rows * A.per < (u64)(e - b) * 64 && A.prefix_lens[g] > 0;
}

__device__ unsigned blocks_of(const Stack& s) {
    return (s.keys[0] + kBlock - 1) / kBlock + (s.keys[1] + kBlock - 1) / kBlock;
}
__device__ u64 tiles_of(const AttendArgs& A, const Stack& s) {
    return ((u64)s.rows * A.per + kTileRows - 1) / kTileRows;
}

__device__ Stack stack_of(const AttendArgs& A, unsigned s) {
    Stack t{};
    t.part = ~0ull;
    t.pool = kNone;
    if (s < A.n_requests) {
        t.row0 = A.row_off[s];
        t.rows = request_rows(A.row_off, s, A.n_rows);
        if (!t.rows) return t;
        const unsigned len = A.lens[s];
        const long long see = (long long)len - t.rows;
        t.see = (int)(see < -1 - (long long)t.rows ? -1 - (long long)t.rows
                                                   : see > 0x7fffffff ? 0x7fffffff : see);
        t.keys[1] = tokens_with_page(A, A.agents[s], len, &t.first[1]);
        const unsigned g = A.n_groups ? group_of(A, s) : kNone;
        if (g != kNone) {
            unsigned row0, rows;
            if (pooled(A, g, &row0, &rows)) t.pool = A.n_requests + g;
            else t.keys[0] = tokens_with_page(A, A.prefix_agents[g], A.prefix_lens[g], &t.first[0]);
        }
    } else {
        const unsigned g = s - A.n_requests;
        unsigned row0, rows;
        if (!pooled(A, g, &row0, &rows)) return t;
        t.row0 = row0;
        t.rows = rows;
        t.keys[0] = tokens_with_page(A, A.prefix_agents[g], A.prefix_lens[g], &t.first[0]);
    }
    return t;
}

// One workgroup: the stacks, how they are split, and where each one's items and
// parts begin.  Keys are cut into pieces of about 1/kTarget of the call's work.
__global__ __launch_bounds__(kPlanThreads) void k_attend_plan(AttendArgs A) {
    __shared__ u64 s_sum[kPlanThreads / 64][3];
    __shared__ u64 s_base[2];
    const unsigned n = A.n_requests + A.n_groups, tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
    u64 work = 0, own_rows = 0, pool_rows = 0;
    for (unsigned s = tid; s < n; s += kPlanThreads) {
        const Stack t = stack_of(A, s);
        A.stacks[s] = t;
        work += tiles_of(A, t) * blocks_of(t);
        (s < A.n_requests ? own_rows : pool_rows) += t.rows;
    }
#pragma unroll
    for (int m = 32; m; m >>= 1) {
        work += __shfl_xor(work, m);
        own_rows += __shfl_xor(own_rows, m);
        pool_rows += __shfl_xor(pool_rows, m);
    }
    if (lane == 0) {
        s_sum[wave][0] = work;
        s_sum[wave][1] = own_rows;
        s_sum[wave][2] = pool_rows;
    }
    if (tid < 2) s_base[tid] = 0;
    __syncthreads();
    work = own_rows = pool_rows = 0;
    for (int w = 0; w < kPlanThreads / 64; ++w) {
        work += s_sum[w][0];
        own_rows += s_sum[w][1];
        pool_rows += s_sum[w][2];
    }
    // offsets that give a row to two requests: nothing is computed
    const bool valid = own_rows <= A.n_rows && pool_rows <= A.n_rows;
    const u64 even = (work * A.n_heads + kTarget - 1) / kTarget;
    const unsigned chunk = (unsigned)(even > kMinBlocks ? (even < kNone ? even : kNone) : kMinBlocks);
    for (unsigned s0 = 0; s0 < n; s0 += kPlanThreads) {
        const unsigned s = s0 + tid;
        Stack t{};
        u64 items = 0, parts = 0;
        if (s < n && valid) {
            t = A.stacks[s];
            const unsigned blocks = blocks_of(t);
            t.chunk = chunk;
            t.splits = (unsigned)(((u64)blocks + chunk - 1) / chunk);
            if (s < A.n_requests && t.pool == kNone && t.splits == 0) t.splits = 1;  // writes zeros
            if (!t.rows) t.splits = 0;
            items = tiles_of(A, t) * t.splits;
            if (t.splits > 1 || t.pool != kNone || s >= A.n_requests)
                parts = (u64)t.rows * A.per * A.n_heads * t.splits;
        }
        // exclusive sums over the workgroup, carried from one thousand to the next
        u64 a = items, b = parts;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            const u64 x = __shfl_up(a, m), y = __shfl_up(b, m);
            if (lane >= (unsigned)m) {
                a += x;
                b += y;
            }
        }
        __syncthreads();
        if (lane == 63) {
            s_sum[wave][0] = a;
            s_sum[wave][1] = b;
        }
        __syncthreads();
        u64 at = s_base[0] + a - items, part = s_base[1] + b - parts;
        for (unsigned w = 0; w < wave; ++w) {
            at += s_sum[w][0];
            part += s_sum[w][1];
        }
        if (s < n) {
            if (parts) t.part = part + parts <= A.part_rows ? part : 0;
            A.stacks[s] = t;
            A.item0[s] = (unsigned)at;
        }
        __syncthreads();
        if (tid == kPlanThreads - 1) {
            s_base[0] = at + items;
            s_base[1] = part + parts;
        }
        __syncthreads();
    }
    if (tid == 0) {
        // more parts than the workspace holds cannot be for valid offsets
        const bool fits = s_base[1] <= A.part_rows && s_base[0] < kNone;
        A.item0[n] = fits ? (unsigned)s_base[0] : 0;
        A.n_items[0] = fits ? (unsigned)s_base[0] : 0;
        A.n_items[1] = fits && valid;
    }
}

constexpr int kWaves = 4;

// The output (or partial) of `rows` rows of an item whose sums the workgroup
// holds in LDS: o[row][kDim + 4], ml[row] = maximum, sum.
struct Sink {
    const AttendArgs& A;
    const Stack& s;
    unsigned tile_row;          // first stack row of the item
    unsigned split, head;
    __device__ u64 part_row(unsigned m) const {
        const u64 total = (u64)s.rows * A.per;
        return s.part + ((u64)head * s.splits + split) * total + m;
    }
};

// 16 rows and a range of keys.  The four waves take 64-key blocks in turn, each
// with a running maximum and sum of its own, and join at the end: with so few
// rows a key or value is used once, so it goes from memory to registers and
// through the matrix product without a stop in LDS.
//     S^T = K Q^T:  a lane holds the scores of one row (lane % 16) with four keys
//                   of each 16 (quad q = lane / 16: keys 4 q .. 4 q + 3);
//     O^T = V^T P^T: P^T is read in just that layout (key slot 8 q + j of 32 keys is
//                   key 16 (j / 4) + 4 q + j % 4), so weights never leave their lane.
// V^T wants eight keys of one column in a lane: a lane loads kCols = dim / 16
// columns of its eight keys, whole rows per quarter wave, and pairs them up by
// byte permutes (column lane * kCols + i in product i).
template <class T, int kDim, bool kE4m3>
__device__ void few_rows(const AttendArgs& A, const Stack& s, unsigned head, unsigned tile,
                         unsigned split, float* lds_o, float2* lds_ml) {
    typedef typename std::conditional<kE4m3, Bf16, T>::type P;      // weights times scales: range
    constexpr int kCols = kDim / 16, kFrags = kDim / 32;
    constexpr int kSub = kDim > 128 ? 2 : 4;        // 16-key sub-blocks held at a time
    const unsigned lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const unsigned col = lane % 16, quad = lane / 16;
    const unsigned total = s.rows * A.per;
    const unsigned m = tile * kTileRows + col;              // this lane's stack row
    const unsigned row = m / A.per, g = m - row * A.per;
    // own tokens that this lane's row sees
    const int lim = m < total ? (int)min((long long)s.keys[1], max(0ll, (long long)s.see + row + 1)) : 0;
    const unsigned last = min(total - 1, tile * kTileRows + kTileRows - 1) / A.per;
    const unsigned most = (unsigned)min((long long)s.keys[1], max(0ll, (long long)s.see + last + 1));
    const unsigned nb0 = (s.keys[0] + kBlock - 1) / kBlock;
    const unsigned nb = nb0 + (most + kBlock - 1) / kBlock;
    const u64 b0 = (u64)split * s.chunk;
    const u64 b1 = min((u64)nb, b0 + s.chunk);

    // Q: fragment f of 32 dims; slot 8 quad + j is dim 32 f + 8 quad + j, and for
    // e4m3 (16 codes a load) dim 64 (f / 2) + 16 quad + 8 (f % 2) + j
    u32x4 qf[kFrags];
    unsigned kdim[kFrags];
#pragma unroll
    for (int f = 0; f < kFrags; ++f) {
        kdim[f] = kE4m3 ? 64 * (f / 2) + 16 * quad + 8 * (f % 2) : 32 * f + 8 * quad;
        qf[f] = u32x4{0, 0, 0, 0};
        if (m < total && kdim[f] < A.dim)
            qf[f] = *reinterpret_cast<const u32x4*>(A.q + (u64)(s.row0 + row) * A.q_row +
                                                    (u64)(head * A.per + g) * A.q_head + 2 * kdim[f]);
    }
    f32x4 o[kCols];
#pragma unroll
    for (int i = 0; i < kCols; ++i) o[i] = f32x4{0, 0, 0, 0};
    float top = -INFINITY, sum = 0.f;
    const unsigned vdim = col * kCols < A.dim ? col * kCols : 0;    // columns behind dim: unused
    const unsigned page_mask = (1u << A.shift) - 1u;
    const char* kbase = A.k + (u64)head * A.head_bytes;
    const char* vbase = A.v + (u64)head * A.head_bytes;

    for (u64 b = b0 + wave; b < b1; b += kWaves) {
        const bool own = b >= nb0;
        const unsigned key0 = (unsigned)(own ? b - nb0 : b) * kBlock;
        const u64 first = s.first[own];
        const unsigned limit = own ? most : s.keys[0];
        // lane l looks up key l of the block
        const unsigned key = key0 + lane;
        int unit = -1;
        if (key < limit) unit = A.tab.unit(first + (key >> A.shift));
        const u64 there = __ballot(unit >= 0);
        if (!there) continue;
        const int spare = __shfl(unit, __builtin_ctzll(there));      // some unit that can be read
        const int safe = unit >= 0 ? unit : spare;
#pragma unroll
        for (int s0 = 0; s0 < 4; s0 += kSub) {
            float sc[kSub][4], kscale[kSub][4], vscale[kSub][4];
            u64 vo[kSub][4];
            f32x4 st[kSub];
            u32x4 kf[kSub][kFrags];
            unsigned vr[kSub][4][kCols / 2];
#pragma unroll
            for (int t = 0; t < kSub; ++t) {
                const unsigned kk = (s0 + t) * 16 + col;
                const int u = __shfl(safe, kk);
                const char* p = kbase + (u64)u * A.k_unit + (u64)((key0 + kk) & page_mask) * A.token_bytes;
                if constexpr (kE4m3) {
#pragma unroll
                    for (int f = 0; f < kFrags; f += 2) {
                        const u32x4 c = *reinterpret_cast<const u32x4*>(p + (kdim[f] < A.dim ? kdim[f] : 0));
                        kf[t][f] = u32x4{T::template from_e4m3<false>(c[0]), T::template from_e4m3<true>(c[0]),
                                         T::template from_e4m3<false>(c[1]), T::template from_e4m3<true>(c[1])};
                        kf[t][f + 1] = u32x4{T::template from_e4m3<false>(c[2]), T::template from_e4m3<true>(c[2]),
                                             T::template from_e4m3<false>(c[3]), T::template from_e4m3<true>(c[3])};
                    }
                } else {
#pragma unroll
                    for (int f = 0; f < kFrags; ++f)
                        kf[t][f] = *reinterpret_cast<const u32x4*>(p + 2 * (kdim[f] < A.dim ? kdim[f] : 0));
                }
                if (A.dim != kDim) {
#pragma unroll
                    for (int f = 0; f < kFrags; ++f)
                        if (kdim[f] >= A.dim) kf[t][f] = u32x4{0, 0, 0, 0};
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const unsigned vk = (s0 + t) * 16 + 4 * quad + i;
                    const int vu = __shfl(safe, vk);
                    const unsigned slot = (key0 + vk) & page_mask;
                    vo[t][i] = (u64)vu * A.v_unit;
                    const char* vp = vbase + vo[t][i] + (u64)slot * A.token_bytes + vdim * (kE4m3 ? 1 : 2);
                    if constexpr (kE4m3) {
                        const u64 so = A.scale_off + 4 * (((u64)head << A.shift) + slot);
                        kscale[t][i] = *reinterpret_cast<const float*>(A.k + (u64)vu * A.k_unit + so);
                        vscale[t][i] = *reinterpret_cast<const float*>(A.v + vo[t][i] + so);
                        unsigned c[kCols / 4];
#pragma unroll
                        for (int w = 0; w < kCols / 4; ++w) c[w] = reinterpret_cast<const unsigned*>(vp)[w];
#pragma unroll
                        for (int w = 0; w < kCols / 4; ++w) {
                            vr[t][i][2 * w] = P::template from_e4m3<false>(c[w]);
                            vr[t][i][2 * w + 1] = P::template from_e4m3<true>(c[w]);
                        }
                    } else {
                        typedef unsigned wide __attribute__((ext_vector_type(kCols / 2)));
                        const wide c = *reinterpret_cast<const wide*>(vp);
#pragma unroll
                        for (int w = 0; w < kCols / 2; ++w) vr[t][i][w] = c[w];
                    }
                }
            }
#pragma unroll
            for (int t = 0; t < kSub; ++t) {
                st[t] = f32x4{0, 0, 0, 0};
#pragma unroll
                for (int f = 0; f < kFrags; ++f) st[t] = T::mma(kf[t][f], qf[f], st[t]);
            }
            float best = top;
#pragma unroll
            for (int t = 0; t < kSub; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float x = st[t][i] * A.scale;
                    if constexpr (kE4m3) x *= kscale[t][i];
                    const unsigned kk = (s0 + t) * 16 + 4 * quad + i;
                    const bool seen = (there >> kk & 1) && (!own || (int)(key0 + kk) < lim);
                    sc[t][i] = seen ? x : -INFINITY;
                    best = fmaxf(best, sc[t][i]);
                }
            best = fmaxf(best, __shfl_xor(best, 16));
            best = fmaxf(best, __shfl_xor(best, 32));
            const float ref = best == -INFINITY ? 0.f : best;
            const float shrink = exp2f(top - ref);
            top = best;
            sum *= shrink;
#pragma unroll
            for (int i = 0; i < kCols; ++i) o[i] *= shrink;
            unsigned pw[kSub][2];
#pragma unroll
            for (int t = 0; t < kSub; ++t) {
                float w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    w[i] = exp2f(sc[t][i] - ref);
                    sum += w[i];
                    // a token that is away has no scale either
                    if constexpr (kE4m3) w[i] = sc[t][i] == -INFINITY ? 0.f : w[i] * vscale[t][i];
                }
                pw[t][0] = P::pack(w[0], w[1]);
                pw[t][1] = P::pack(w[2], w[3]);
            }
            if (there != ~0ull) {           // what is stored there may be anything
#pragma unroll
                for (int t = 0; t < kSub; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!(there >> ((s0 + t) * 16 + 4 * quad + i) & 1)) {
#pragma unroll
                            for (int w = 0; w < kCols / 2; ++w) vr[t][i][w] = 0;
                        }
            }
#pragma unroll
            for (int t = 0; t < kSub; t += 2) {
                const u32x4 p = {pw[t][0], pw[t][1], pw[t + 1][0], pw[t + 1][1]};
#pragma unroll
                for (int i = 0; i < kCols; ++i) {
                    constexpr unsigned kLow = 0x05040100u, kHigh = 0x07060302u;
                    const unsigned sel = i % 2 ? kHigh : kLow;
                    const u32x4 a = {__builtin_amdgcn_perm(vr[t][1][i / 2], vr[t][0][i / 2], sel),
                                     __builtin_amdgcn_perm(vr[t][3][i / 2], vr[t][2][i / 2], sel),
                                     __builtin_amdgcn_perm(vr[t + 1][1][i / 2], vr[t + 1][0][i / 2], sel),
                                     __builtin_amdgcn_perm(vr[t + 1][3][i / 2], vr[t + 1][2][i / 2], sel)};
                    o[i] = P::mma(a, p, o[i]);
                }
            }
        }
    }
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);

    // join the four waves: lds_o[wave][row][kDim + 4], lds_ml[wave][row]
    constexpr int kPitch = kDim + 4;
    if (quad == 0) lds_ml[wave * 16 + col] = float2{top, sum};
    __syncthreads();
    float all = -INFINITY, l = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) all = fmaxf(all, lds_ml[w * 16 + col].x);
    const float ref = all == -INFINITY ? 0.f : all;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) l += lds_ml[w * 16 + col].y * exp2f(lds_ml[w * 16 + col].x - ref);
    const bool direct = s.part == ~0ull;
    const float mine = exp2f(top - ref) * (direct ? (l > 0.f || l != l ? 1.f / l : 0.f) : 1.f);
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int i = 0; i < kCols; ++i)
            lds_o[(wave * 16 + col) * kPitch + (4 * quad + r) * kCols + i] = o[i][r] * mine;
    __syncthreads();
    const u64 part0 = s.part + ((u64)head * s.splits + split) * total;
    for (unsigned e = threadIdx.x; e < 16 * (kDim / 4); e += kWaves * 64) {
        const unsigned mm = e / (kDim / 4), d = e % (kDim / 4) * 4;
        const unsigned sm = tile * kTileRows + mm;
        if (sm >= total || d >= A.dim) continue;
        f32x4 x = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
            x += *reinterpret_cast<const f32x4*>(&lds_o[(w * 16 + mm) * kPitch + d]);
        if (direct) {
            const unsigned rr = sm / A.per, hh = head * A.per + (sm - rr * A.per);
            char* to = A.out + (u64)(s.row0 + rr) * A.out_row + (u64)hh * A.out_head + 2 * d;
            *reinterpret_cast<u32x2*>(to) = u32x2{T::pack(x[0], x[1]), T::pack(x[2], x[3])};
        } else {
            *reinterpret_cast<f32x4*>(&A.part_o[(part0 + sm) * kDim + d]) = x;
        }
    }
    if (wave == 0 && quad == 0 && m < total) {
        if (direct) {
            if (A.lse)
                A.lse[(u64)(s.row0 + row) * (A.n_heads * A.per) + head * A.per + g] =
                    (all + log2f(l)) * 0.6931471805599453f;
        } else {
            A.part_ml[part0 + m] = float2{all, l};
        }
    }
    __syncthreads();            // the next item's LDS
}

template <class T, int kDim, bool kE4m3>
__global__ __launch_bounds__(kWaves * 64, kDim > 128 ? 1 : 2) void k_attend(AttendArgs A) {
    __shared__ __align__(16) float s_o[kWaves * 16 * (kDim + 4)];
    __shared__ float2 s_ml[kWaves * 16];
    const u64 n = (u64)*A.n_items * A.n_heads;
    const unsigned stacks = A.n_requests + A.n_groups;
    for (u64 it = blockIdx.x; it < n; it += gridDim.x) {
        const unsigned entry = (unsigned)(it / A.n_heads), head = (unsigned)(it % A.n_heads);
        // stacks without items share their first item with the next one, which
        // is the one that the search gives
        const unsigned si = wave_search(stacks, entry, [&](unsigned i) { return A.item0[i]; });
        const Stack s = A.stacks[si];
        const unsigned local = entry - A.item0[si];
        const unsigned tiles = (unsigned)tiles_of(A, s);
        if (s.splits == 0 || local >= tiles * s.splits) continue;
        few_rows<T, kDim, kE4m3>(A, s, head, local % tiles, local / tiles, s_o, s_ml);
    }
}

// Joins the parts of rows that several items share: a wave takes a row, head
// after head, kDim / 64 columns a lane.
template <class T, int kDim>
__global__ __launch_bounds__(256) void k_attend_join(AttendArgs A) {
    constexpr int kCols = kDim / 64;
    const unsigned lane = threadIdx.x % 64;
    const unsigned heads = A.n_heads * A.per;
    const u64 n = (u64)A.n_rows * heads;
    u64 w = (u64)blockIdx.x * 4 + threadIdx.x / 64;
    if (w >= n || !A.n_items[1]) return;
    const unsigned t = (unsigned)(w / heads), qh = (unsigned)(w % heads);
    const unsigned r = wave_search(A.n_requests, t, [&](unsigned i) { return A.row_off[i]; });
    const Stack own = A.stacks[r];
    if (t < own.row0 || t - own.row0 >= own.rows) return;
    if (own.part == ~0ull && own.pool == kNone) return;     // written straight out
    const unsigned head = qh / A.per, g = qh - head * A.per;
    float top = -INFINITY, sum = 0.f, x[kCols];
#pragma unroll
    for (int c = 0; c < kCols; ++c) x[c] = 0.f;
    for (int which = 0; which < 2; ++which) {
        const Stack& s = which ? A.stacks[own.pool == kNone ? r : own.pool] : own;
        // offsets that break the rules can put a request outside its group's rows
        if (which && (own.pool == kNone || t < s.row0 || t - s.row0 >= s.rows)) break;
        const u64 total = (u64)s.rows * A.per;
        const u64 first = s.part + (u64)head * s.splits * total + (u64)(t - s.row0) * A.per + g;
        for (unsigned i = 0; i < s.splits; ++i) {
            const float2 ml = A.part_ml[first + i * total];
            const float best = fmaxf(top, ml.x), ref = best == -INFINITY ? 0.f : best;
            const float a = exp2f(top - ref), b = exp2f(ml.x - ref);
            top = best;
            sum = sum * a + ml.y * b;
            const float* p = &A.part_o[(first + i * total) * kDim + lane * kCols];
#pragma unroll
            for (int c = 0; c < kCols; ++c)
                x[c] = x[c] * a + (lane * kCols + c < A.dim ? p[c] * b : 0.f);
        }
    }
    const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
    char* to = A.out + (u64)t * A.out_row + (u64)qh * A.out_head;
#pragma unroll
    for (int c = 0; c < kCols; ++c)
        if (lane * kCols + c < A.dim)
            reinterpret_cast<unsigned short*>(to)[lane * kCols + c] =
                (unsigned short)T::pack(x[c] * inv, 0.f);
    if (A.lse && lane == 0) A.lse[(u64)t * heads + qh] = (top + log2f(sum)) * 0.6931471805599453f;
}

unsigned padded(unsigned dim) { return dim <= 64 ? 64 : dim <= 128 ? 128 : 256; }
u64 up(u64 x) { return (x + 255) & ~255ull; }

// Partial rows at most: every row once for its own tokens and once for a shared
// prefix, and a tile for each split beyond a stack's first; there are at most
// kTarget of those, as every one but a stack's last has its share of the work.
u64 part_rows(u64 n_rows, u64 n_q_heads) {
    return 2 * n_rows * n_q_heads + (u64)kTarget * kTileRows;
}

struct Layout {
    u64 item0, stacks, ml, o, bytes;
};
Layout layout_of(u64 n_rows, u64 n_requests, u64 n_groups, u64 n_q_heads, unsigned dim) {
    Layout l;
    const u64 n = n_requests + n_groups, rows = part_rows(n_rows, n_q_heads);
    l.item0 = 256;
    l.stacks = up(l.item0 + 4 * (n + 1));
    l.ml = up(l.stacks + sizeof(Stack) * n);
    l.o = up(l.ml + 8 * rows);
    l.bytes = l.o + 4 * rows * padded(dim);
    return l;
}

template <class T, int kDim, bool kE4m3>
void attend_launch(const AttendArgs& A, unsigned cus, hipStream_t st) {
    hipLaunchKernelGGL(k_attend_plan, dim3(1), dim3(kPlanThreads), 0, st, A);
    hipLaunchKernelGGL((k_attend<T, kDim, kE4m3>), dim3(cus * (kDim > 128 ? 1 : 2)), dim3(kWaves * 64),
                       0, st, A);
    const u64 waves = (u64)A.n_rows * A.n_heads * A.per;
    hipLaunchKernelGGL((k_attend_join<T, kDim>), dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, st, A);
}

template <class T, bool kE4m3>
void attend_dim(const AttendArgs& A, unsigned cus, hipStream_t st) {
    switch (padded(A.dim)) {
        case 64: attend_launch<T, 64, kE4m3>(A, cus, st); break;
        case 128: attend_launch<T, 128, kE4m3>(A, cus, st); break;
        default: attend_launch<T, 256, kE4m3>(A, cus, st); break;
    }
}

ss_status attend_args(const ss_kv_cache* c, const ss_batch* b, uint32_t type, uint32_t n_q_heads) {
    ss_status s = cache_args(c, type);
    if (s == SS_OK) s = batch_args(b, true, true);
    if (s != SS_OK) return s;
    if (n_q_heads < 1 || n_q_heads > 65536 || n_q_heads % c->n_heads)
        return set_err(SS_ERR_ARG, "n_q_heads must be a multiple of the cache's n_heads, at most 65536");
    if ((u64)b->n_rows * n_q_heads >= (1ull << 31))
        return set_err(SS_ERR_ARG, "n_rows * n_q_heads must be below 2^31");
    return SS_OK;
}

}  // namespace

}  // namespace ss

using namespace ss;

extern "C" {

uint64_t ss_prefix_attention_workspace(const ss_kv_cache* cache, const ss_batch* batch,
                                       uint32_t n_q_heads) {
    if (!cache || attend_args(cache, batch, cache->type == SS_F16 ? SS_F16 : SS_BF16, n_q_heads) != SS_OK)
        return 0;
    return layout_of(batch->n_rows, batch->n_requests, batch->n_groups, n_q_heads, cache->head_dim).bytes;
}

ss_status ss_prefix_attention(const ss_kv_cache* cache, const ss_batch* batch, const void* q,
                              void* out, float* lse, uint32_t type, uint32_t n_q_heads,
                              uint64_t q_row_stride, uint64_t q_head_stride,
                              uint64_t out_row_stride, uint64_t out_head_stride, float scale,
                              void* workspace, uint64_t workspace_bytes, void* stream) {
    ss_status s = attend_args(cache, batch, type, n_q_heads);
    if (s != SS_OK) return s;
    if (!std::isfinite(scale)) return set_err(SS_ERR_ARG, "scale must be finite");
    if (batch->n_rows == 0 || batch->n_requests == 0) return SS_OK;
    const unsigned dim = cache->head_dim;
    const u64 rows = batch->n_rows;
    if ((s = rows_args("q", q, rows, n_q_heads, dim, q_row_stride, q_head_stride, false)) != SS_OK ||
        (s = rows_args("out", out, rows, n_q_heads, dim, out_row_stride, out_head_stride, true)) != SS_OK)
        return s;
    const Layout l = layout_of(rows, batch->n_requests, batch->n_groups, n_q_heads, dim);
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15))
        return set_err(SS_ERR_ARG, "workspace must be a 16-byte aligned pointer");
    if (workspace_bytes < l.bytes)
        return set_err(SS_ERR_ARG, "workspace_bytes %llu < %llu", (unsigned long long)workspace_bytes,
                       (unsigned long long)l.bytes);
    const u64 q_bytes = rows_bytes(rows, n_q_heads, dim, q_row_stride, q_head_stride);
    const u64 out_bytes = rows_bytes(rows, n_q_heads, dim, out_row_stride, out_head_stride);
    const uintptr_t q0 = reinterpret_cast<uintptr_t>(q), o0 = reinterpret_cast<uintptr_t>(out);
    if (q0 < o0 + out_bytes && o0 < q0 + q_bytes) return set_err(SS_ERR_ARG, "out overlaps q");
    int dev = -1;
    if ((s = current_device(&dev)) != SS_OK || (s = cache_memory(cache, dev)) != SS_OK ||
        (s = batch_memory(batch, true, true, dev)) != SS_OK)
        return s;
    if (!device_range_ok(q, q_bytes, dev)) return device_error("q", dev);
    if (!device_range_ok(out, out_bytes, dev)) return device_error("out", dev);
    if (lse && !device_range_ok(lse, rows * n_q_heads * 4, dev)) return device_error("lse", dev);
    if (!device_range_ok(workspace, l.bytes, dev)) return device_error("workspace", dev);
    int cus = 256;
    if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess) {
        (void)hipGetLastError();
        cus = 256;
    }
    AttendArgs A{};
    A.tab = table_of(cache->units, cache->agent_off, cache->n_agents, cache->n_entries,
                     cache->capacity_units);
    A.k = static_cast<const char*>(cache->k);
    A.v = static_cast<const char*>(cache->v);
    A.k_unit = cache->k_unit_bytes;
    A.v_unit = cache->v_unit_bytes;
    A.token_bytes = cache->token_bytes;
    A.head_bytes = cache->head_bytes;
    A.scale_off = cache->scale_off;
    A.q = static_cast<const char*>(q);
    A.out = static_cast<char*>(out);
    A.lse = lse;
    A.q_row = 2 * q_row_stride;
    A.q_head = 2 * q_head_stride;
    A.out_row = 2 * out_row_stride;
    A.out_head = 2 * out_head_stride;
    A.row_off = batch->row_off;
    A.agents = batch->agents;
    A.lens = batch->lens;
    A.group_off = batch->group_off;
    A.prefix_agents = batch->prefix_agents;
    A.prefix_lens = batch->prefix_lens;
    A.n_rows = batch->n_rows;
    A.n_requests = batch->n_requests;
    A.n_groups = batch->n_groups;
    A.n_heads = cache->n_heads;
    A.per = n_q_heads / cache->n_heads;
    A.dim = dim;
    A.shift = (unsigned)__builtin_ctz(cache->page_tokens);
    A.scale = scale * 1.4426950408889634f;
    char* ws = static_cast<char*>(workspace);
    A.n_items = reinterpret_cast<unsigned*>(ws);
    A.item0 = reinterpret_cast<unsigned*>(ws + l.item0);
    A.stacks = reinterpret_cast<Stack*>(ws + l.stacks);
    A.part_ml = reinterpret_cast<float2*>(ws + l.ml);
    A.part_o = reinterpret_cast<float*>(ws + l.o);
    A.part_rows = part_rows(rows, n_q_heads);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const unsigned n_cus = (unsigned)std::max(cus, 1);
    if (type == SS_BF16) {
        if (cache->type == SS_E4M3) attend_dim<Bf16, true>(A, n_cus, st);
        else attend_dim<Bf16, false>(A, n_cus, st);
    } else {
        if (cache->type == SS_E4M3) attend_dim<F16, true>(A, n_cus, st);
        else attend_dim<F16, false>(A, n_cus, st);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return set_err(SS_ERR_HIP, "prefix attention kernels: %s", hipGetErrorString(e));
    return SS_OK;
}

}  // extern "C"
