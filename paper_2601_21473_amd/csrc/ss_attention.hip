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
#include <type_traits>

#include "ss_model.h"

namespace ss {

namespace {

constexpr unsigned kNone = 0xffffffffu;
constexpr unsigned kBlock = 64;             // keys of one step of an item
// A call's items are about kTarget, twice the workgroups that run at a time, so that they
// even out (64 agents over a prefix of 8,192: 1,024 items 70 us, 512 80 us, 2,048 78 us; one
// of 131,071 tokens 121, 117 and 126 us), of kMinBlocks blocks at least (8: 72 us).
constexpr unsigned kTarget = 1024;
constexpr unsigned kAtOnce = 512;           // workgroups that run at a time: two a compute unit, dim 256 one
constexpr unsigned kMinBlocks = 4;
constexpr unsigned kXcds = 8;               // of the card, each with its own L2
constexpr unsigned kMostRows = 128;         // rows of the largest tile

struct Stack {
    u64 first[2];       // table entries of the two segments of keys: prefix, own tokens
    u64 part;           // first partial row, or ~0: one item per tile, written straight out
    unsigned keys[2];   // tokens with a page
    unsigned row0, rows;
    int see;            // row i of the stack sees own tokens 0 .. see + i
    unsigned splits;    // items per tile and head
    unsigned pool;      // a request's stack: its group, if that has a stack of its own, or kNone
    unsigned pad;
};
static_assert(sizeof(Stack) == 56, "three words and eight halves");

// An item, the same for every head.
struct Item {
    u64 first[2];
    u64 part;
    unsigned keys[2];
    unsigned row0, rows;
    int see;
    unsigned splits;
    unsigned tile_rows, tile, split, chunk;     // key blocks [split chunk, (split + 1) chunk)
};
static_assert(sizeof(Item) == 64, "four 16-byte words");

// A row whose parts are joined: its own tokens' and its prefix's.
struct JoinRow {
    u64 first[2];       // the part of head 0, query head 0, split 0
    unsigned total[2];  // rows of the stack: the distance between splits
    unsigned splits[2];
    unsigned row, pad[3];
};
static_assert(sizeof(JoinRow) == 48, "three 16-byte words");

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
    float scale;                                // |scale| log2(e), 1 for a scale of 0
    unsigned q_keep, q_flip;                    // queries' bits that count, and that turn
    // workspace
    unsigned* counts;                           // items per head, rows to join
    unsigned* taken;                            // [16 kXcds] items taken behind the first
    Item* items;                                // [most_items]
    JoinRow* joins;                             // [n_rows]
    Stack* stacks;                              // [n_groups] of the prefixes
    u64 most_items;
    float* part_o;                              // [part_rows][padded dim]
    float2* part_ml;                            // [part_rows] maximum (log2), sum
    u64 part_rows;
};

constexpr unsigned kPlanThreads = 512;

__device__ unsigned tokens_with_page(const AttendArgs& A, unsigned agent, unsigned len, u64* first) {
    const u64 most = (u64)A.tab.row(agent, first) << A.shift;
    return (unsigned)std::min<u64>(std::min<u64>(len, most), 0x7fffffc0u);
}

__device__ unsigned blocks_of(const Stack& s) {
    return (s.keys[0] + kBlock - 1) / kBlock + (s.keys[1] + kBlock - 1) / kBlock;
}
// Rows of a stack's tiles: 16 while they hold all (nothing to share, so registers
// suffice), else 64 or, where the registers hold the sums of so many, 128 through LDS.
// (64 stacks over 4,000 keys of 8 heads of 128: 4 rows 187 us, in tiles of 64 202 us; 128
// rows 204 us, in two tiles of 64 253 us; 256 rows 344 us, in four 445 us.)
__device__ unsigned tile_rows(const AttendArgs& A, const Stack& s) {
    const u64 rows = (u64)s.rows * A.per;
    return rows <= 16 ? 16 : rows <= 64 || A.dim > 128 ? 64 : 128;
}
__device__ unsigned tiles_of(const AttendArgs& A, const Stack& s) {
    const u64 n = tile_rows(A, s);
    return (unsigned)(((u64)s.rows * A.per + n - 1) / n);
}

// The stack of group g's prefix.  It has rows (a stack of its own) where several
// requests share the prefix and are so short that a tile of rows holds more than
// one; otherwise each request reads prefix and own tokens in one go, without parts.
// (64 requests of 8 heads of 128, 4 query heads each, over a prefix of 8,192: one row each
// 51 us, without pools 226 us; 15 rows 194 and 235 us; 24 rows, so not pooled, 296 us, with
// a pool 301 us, and over a prefix of 1,000 61 and 111 us.)
__device__ Stack prefix_stack(const AttendArgs& A, unsigned g) {
    Stack t{};
    t.part = ~0ull;
    t.pool = kNone;
    const unsigned b = A.group_off[g], e = A.group_off[g + 1];
    u64 first;
    const unsigned len = A.prefix_lens[g];
    const unsigned keys = tokens_with_page(A, A.prefix_agents[g], len, &first);
    if (b >= e || e > A.n_requests) return t;
    const unsigned r0 = A.row_off[b], r1 = A.row_off[e];
    t.keys[0] = keys;
    t.first[0] = first;
    if (r0 < r1 && r1 <= A.n_rows && e - b > 1 && (u64)(r1 - r0) * A.per < (u64)(e - b) * 64 && len) {
        t.row0 = r0;
        t.rows = r1 - r0;
    }
    return t;
}

// The stack of request s's own tokens, without its prefix.
__device__ Stack request_stack(const AttendArgs& A, unsigned s) {
    Stack t{};
    t.part = ~0ull;
    t.pool = kNone;
    t.row0 = A.row_off[s];
    const unsigned len = A.lens[s], agent = A.agents[s];
    t.rows = request_rows(A.row_off, s, A.n_rows);
    const long long see = (long long)len - t.rows;
    t.see = (int)(see < -1 - (long long)t.rows ? -1 - (long long)t.rows
                                               : see > 0x7fffffff ? 0x7fffffff : see);
    u64 first;
    t.keys[1] = tokens_with_page(A, agent, len, &first);
    t.first[1] = first;
    return t;
}

// Adds to request s's stack its group's prefix, as keys of its own or as a pool.  begin
// and end are the groups' offsets, prefix their stacks.
template <class P, class B>
__device__ void add_prefix(unsigned s, unsigned n_groups, B begin, const P& prefix, Stack& t) {
    unsigned lo = 0, hi = n_groups;             // the largest g with begin(g) <= s
    while (hi - lo > 1) {
        const unsigned mid = (lo + hi) / 2;
        if (begin(mid) <= s) lo = mid;
        else hi = mid;
    }
    if (hi <= lo || begin(lo) > s || s >= begin(lo + 1)) return;
    const Stack& p = prefix[lo];
    if (p.rows) {
        t.pool = lo;
    } else {
        t.keys[0] = p.keys[0];
        t.first[0] = p.first[0];
    }
}

// What the planning workgroup carries from kPlanThreads stacks to the next.
struct PlanState {
    Stack stack[kPlanThreads];
    unsigned at[2][kPlanThreads + 1];           // first item, first row to join, of each stack
    unsigned sum[kPlanThreads / 64][3];
    unsigned base[3];                           // items, rows to join, parts per head so far
};

// Lists the items and the rows to join of up to kPlanThreads stacks, thread by thread;
// pools are in `prefix`, where a prefix's own stack (`group`) goes too.
__device__ void plan_stacks(const AttendArgs& A, Stack t, bool own, unsigned group, unsigned chunk,
                            Stack* prefix, bool more, PlanState& S) {
    const unsigned tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
    const unsigned blocks = blocks_of(t);
    t.splits = blocks / chunk + (blocks % chunk != 0);
    if (own && t.pool == kNone && t.splits == 0) t.splits = 1;          // writes zeros
    if (!t.rows) t.splits = 0;
    const bool joined = own && (t.splits > 1 || t.pool != kNone);
    const unsigned v[3] = {tiles_of(A, t) * t.splits, joined ? t.rows : 0,
                           joined || !own ? t.rows * A.per * t.splits : 0};
    // exclusive sums over the workgroup
    unsigned a[3] = {v[0], v[1], v[2]};
#pragma unroll
    for (int m = 1; m < 64; m <<= 1)
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            const unsigned x = __shfl_up(a[k], m);
            if (lane >= (unsigned)m) a[k] += x;
        }
    if (lane == 63) {
#pragma unroll
        for (int k = 0; k < 3; ++k) S.sum[wave][k] = a[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        a[k] -= v[k];
        for (unsigned w = 0; w < wave; ++w) a[k] += S.sum[w][k];
    }
    if (v[2]) t.part = (u64)(S.base[2] + a[2]) * A.n_heads;
    if (group != kNone) prefix[group] = t;
    S.stack[tid] = t;
    S.at[0][tid] = a[0];
    S.at[1][tid] = a[1];
    if (tid == kPlanThreads - 1) {
        S.at[0][kPlanThreads] = a[0] + v[0];
        S.at[1][kPlanThreads] = a[1] + v[1];
    }
    __syncthreads();
    // the stack of an item or row: the last that begins at or before it
    auto find = [&](int k, unsigned i) {
        unsigned lo = 0;
#pragma unroll
        for (unsigned step = kPlanThreads / 2; step; step /= 2)
            if (S.at[k][lo + step] <= i) lo += step;
        return lo;
    };
    const unsigned items = S.at[0][kPlanThreads], joins = S.at[1][kPlanThreads];
    const unsigned base0 = S.base[0], base1 = S.base[1];
    if (!more) __syncthreads();
    if ((u64)base0 + items <= A.most_items)
        for (unsigned i = tid; i < items; i += kPlanThreads) {
            const unsigned f = find(0, i), j = i - S.at[0][f];
            const Stack& s = S.stack[f];
            const unsigned tiles = tiles_of(A, s);
            // tiles next to each other read the same keys
            A.items[base0 + i] = Item{{s.first[0], s.first[1]}, s.part, {s.keys[0], s.keys[1]},
                                          s.row0, s.rows, s.see, s.splits, tile_rows(A, s),
                                          j % tiles, j / tiles, chunk};
        }
    if ((u64)base1 + joins <= A.n_rows)
        for (unsigned i = tid; i < joins; i += kPlanThreads) {
            const unsigned f = find(1, i);
            const Stack& s = S.stack[f];
            JoinRow r{};
            r.row = s.row0 + (i - S.at[1][f]);
            r.first[0] = s.part + (u64)(r.row - s.row0) * A.per;
            r.total[0] = s.rows * A.per;
            r.splits[0] = s.splits;
            if (s.pool != kNone) {
                const Stack& p = prefix[s.pool];
                // offsets that break the rules can put a request outside its group's rows
                if (r.row >= p.row0 && r.row - p.row0 < p.rows) {
                    r.first[1] = p.part + (u64)(r.row - p.row0) * A.per;
                    r.total[1] = p.rows * A.per;
                    r.splits[1] = p.splits;
                }
            }
            A.joins[base1 + i] = r;
        }
    if (more) __syncthreads();          // before base changes
    if (tid == kPlanThreads - 1) {
        S.base[0] += a[0] + v[0];
        S.base[1] += a[1] + v[1];
        S.base[2] += a[2] + v[2];
    }
    if (more) __syncthreads();
}

// One workgroup: the stacks, how they are split, and what there is to do.  Keys are cut
// into pieces of about 1/kTarget of the call's work.  Reads that wait for each other
// bound it, so a request's own ones are out before its group is looked at, and items and
// joins carry all that their kernels need.
__global__ __launch_bounds__(kPlanThreads) void k_attend_plan(AttendArgs A) {
    __shared__ PlanState S;
    __shared__ float s_work[kPlanThreads / 64][3];
    __shared__ unsigned s_rows[kPlanThreads / 64][2];
    const unsigned tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
    // in 32-bit floats, as they only set how fine the pieces are: key blocks of all tiles,
    // tiles, and the most blocks that one has
    float work = 0.f, tiles = 0.f, longest = 0.f;
    auto count = [&](const Stack& t) {
        const float n = (float)tiles_of(A, t), b = (float)blocks_of(t);
        work += n * b;
        tiles += n;
        longest = fmaxf(longest, t.rows ? b : 0.f);
    };
    unsigned own_rows = 0, pool_rows = 0;       // saturating: one of n_rows says enough
    auto add = [](unsigned a, unsigned b) { return a + b < a ? ~0u : a + b; };
    // Batches of up to kPlanThreads requests and groups: groups in the first threads,
    // requests in the last, so that they are in other waves as a rule and read at the
    // same time; all in LDS.  Larger ones: groups in the workspace, requests kPlanThreads
    // at a time, and again for their items.
    const unsigned n_requests = A.n_requests, n_groups = A.n_groups;
    const bool small = n_requests + n_groups <= kPlanThreads;
    const bool is_group = tid < n_groups, is_request = kPlanThreads - 1 - tid < n_requests;
    Stack mine{};
    if (small) {
        if (is_group) {
            mine = prefix_stack(A, tid);
            S.stack[tid] = mine;
            S.at[0][tid] = A.group_off[tid];
            if (tid == n_groups - 1) S.at[0][n_groups] = A.group_off[n_groups];
            pool_rows = mine.rows;
        } else if (is_request) {
            mine = request_stack(A, kPlanThreads - 1 - tid);
            own_rows = mine.rows;
        }
        __syncthreads();
        if (is_request && n_groups)
            add_prefix(kPlanThreads - 1 - tid, n_groups, [&](unsigned g) { return S.at[0][g]; }, S.stack, mine);
        count(mine);
    } else {
        for (unsigned g = tid; g < n_groups; g += kPlanThreads) {
            const Stack t = prefix_stack(A, g);
            A.stacks[g] = t;
            count(t);
            pool_rows = add(pool_rows, t.rows);
        }
        __syncthreads();
        for (unsigned s = tid; s < n_requests; s += kPlanThreads) {
            Stack t = request_stack(A, s);
            add_prefix(s, n_groups, [&](unsigned g) { return A.group_off[g]; }, A.stacks, t);
            count(t);
            own_rows = add(own_rows, t.rows);
        }
    }
#pragma unroll
    for (int m = 32; m; m >>= 1) {
        work += __shfl_xor(work, m);
        tiles += __shfl_xor(tiles, m);
        longest = fmaxf(longest, __shfl_xor(longest, m));
        own_rows = add(own_rows, __shfl_xor(own_rows, m));
        pool_rows = add(pool_rows, __shfl_xor(pool_rows, m));
    }
    if (lane == 0) {
        s_work[wave][0] = work;
        s_work[wave][1] = tiles;
        s_work[wave][2] = longest;
        s_rows[wave][0] = own_rows;
        s_rows[wave][1] = pool_rows;
    }
    if (tid < 3) S.base[tid] = 0;
    __syncthreads();
    work = tiles = 0.f;
    own_rows = pool_rows = 0;
#pragma unroll
    for (unsigned w = 0; w < kPlanThreads / 64; ++w) {
        work += s_work[w][0];
        tiles += s_work[w][1];
        longest = fmaxf(longest, s_work[w][2]);
        own_rows = add(own_rows, s_rows[w][0]);
        pool_rows = add(pool_rows, s_rows[w][1]);
    }
    const float even = ceilf(work * (float)A.n_heads * (1.f / kTarget));
    unsigned chunk = even < (float)kMinBlocks ? kMinBlocks : even < 1e9f ? (unsigned)even : 1000000000u;
    // No piece at all where whole tiles, kAtOnce at a time, end within a tenth of the even
    // share: parts cost what they write and the join reads (64 stacks of 128 rows over 4,000
    // keys 204 us, in two pieces 282 us).
    const float share = (float)A.n_heads * (A.dim > 128 ? 2.f / kAtOnce : 1.f / kAtOnce);
    if (ceilf(tiles * share) * longest <= 1.1f * work * share)
        chunk = std::max(chunk, (unsigned)longest);
    // offsets that give a row to two requests: nothing is computed
    if (own_rows <= A.n_rows && pool_rows <= A.n_rows) {
        // prefixes first: their items are the longest
        if (small) {
            plan_stacks(A, mine, is_request, is_group ? tid : kNone, chunk, S.stack, false, S);
        } else {
            for (unsigned g0 = 0; g0 < n_groups; g0 += kPlanThreads) {
                const unsigned g = g0 + tid;
                plan_stacks(A, g < n_groups ? A.stacks[g] : Stack{}, false, g < n_groups ? g : kNone,
                            chunk, A.stacks, true, S);
            }
            for (unsigned s0 = 0; s0 < n_requests; s0 += kPlanThreads) {
                const unsigned s = s0 + tid;
                Stack t{};
                if (s < n_requests) {
                    t = request_stack(A, s);
                    add_prefix(s, n_groups, [&](unsigned g) { return A.group_off[g]; }, A.stacks, t);
                }
                plan_stacks(A, t, s < n_requests, kNone, chunk, A.stacks, true, S);
            }
        }
    }
    __syncthreads();
    if (tid == 0) {
        // more than the workspace holds cannot be for valid offsets
        const bool fits = (u64)S.base[2] * A.n_heads <= A.part_rows && S.base[0] <= A.most_items &&
            S.base[1] <= A.n_rows;
        A.counts[0] = fits ? S.base[0] : 0;
        A.counts[1] = fits ? S.base[1] : 0;
    }
    if (tid < kXcds) A.taken[16 * tid] = 0;
}

constexpr int kWaves = 4;
// A weight may pass the running reference by 2^kSlack before sums are rescaled:
// the reference then stays for most blocks, and a block's maximum need not be known
// to all lanes of a row.  2^8 is exact in every type and far from their ranges.
constexpr float kSlack = 8.f;

// The kernel's arguments, read again: what one tile size needs of them is not kept in
// scalar registers for the others (up to 70 were spilled, into the inner loops too).
__device__ __forceinline__ AttendArgs again() {
    typedef const __attribute__((address_space(4))) AttendArgs* Constant;
    Constant p = (Constant)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *(const AttendArgs*)p;
}

// The lane, of which the compiler knows nothing: what follows from it is worked out for
// each item anew and not kept in registers beside the other tile sizes' values (they
// spilled up to 60 registers).
__device__ __forceinline__ unsigned own_lane() {
    unsigned lane = threadIdx.x % 64;
    asm volatile("" : "+v"(lane));
    return lane;
}

// A lane's share of 16 keys and values as they come from memory, and where it lies.
// Products want S^T = K Q^T and O^T = V^T P^T with 16 x 16 x 32 products:
//   K: a lane holds key lane % 16, dims 8 q .. 8 q + 7 of each 32 (q = lane / 16); for
//      e4m3 it loads 16 codes at once, so its dims are 16 q .. + 15 of each 64, which
//      the queries follow (slot_dim);
//   S^T leaves it with the scores of row lane % 16 for keys 4 q .. 4 q + 3;
//   V: it loads dim / 16 columns of those four keys, so a quarter wave reads whole
//      rows, and pairs keys up by byte permutes: product i yields the columns
//      lane * (dim / 16) + i.  Key slot 8 q + j of 32 is key 16 (j / 4) + 4 q + j % 4,
//      which is how the weights lie in S^T: they never leave their lane.
template <class T, int kDim, bool kE4m3>
struct Keys {
    static constexpr int kCols = kDim / 16, kFrags = kDim / 32;
    static constexpr int kLoads = kE4m3 ? kFrags / 2 : kFrags;
    static constexpr int kWords = kE4m3 ? kCols / 4 : kCols / 2;
    // Weights are rounded to 16 bits, which is what the products take: half a step each, as the
    // output's own rounding (bf16 outputs are off by 2.3e-3 in the mean square where 32-bit
    // weights leave 1.7e-3, fp16 by 2.7e-4 and 2.1e-4).  A second part for what that leaves
    // doubles the products with the values, which bound prompts.
    // Weights times the values' scales need bf16's range; for fp16 rows, whose outputs
    // keep three more bits, what their rounding leaves is multiplied too (in bf16 alone
    // the outputs were off by 1.5e-3 where plain 32-bit sums are by 2.1e-4).
    typedef typename std::conditional<kE4m3, Bf16, T>::type P;
    static constexpr int kParts = kE4m3 && std::is_same<T, F16>::value ? 2 : 1;
    // fp16 weights are held against 2^-kLift of the reference, 2^(kLift + kSlack) at most:
    // held against the reference itself those below 2^-14 of it lost bits, and those below
    // 2^-25 became nothing, which many of them together show (8,000 weights of 2^-25: the
    // output was off by 3%).
    static constexpr float kLift = std::is_same<P, F16>::value ? 6.f : 0.f;
    static constexpr float kUnlift = kLift == 6.f ? 1.f / 64 : 1.f;
    // The parts of four weights.
    static __device__ __forceinline__ void weights(f32x4 e, unsigned (*w)[2]) {
        w[0][0] = P::pack(e[0], e[1]);
        w[0][1] = P::pack(e[2], e[3]);
        if constexpr (kParts == 2) {
            w[1][0] = P::pack(e[0] - P::lo(w[0][0]), e[1] - P::hi(w[0][0]));
            w[1][1] = P::pack(e[2] - P::lo(w[0][1]), e[3] - P::hi(w[0][1]));
        }
    }
    typedef unsigned wide __attribute__((ext_vector_type(kWords == 1 ? 2 : kWords)));
    u32x4 k[kLoads];
    unsigned v[4][kWords];
    f32x4 ks, vs;

    static __device__ unsigned slot_dim(unsigned f, unsigned quad) {
        return kE4m3 ? 64 * (f / 2) + 16 * quad + 8 * (f % 2) : 32 * f + 8 * quad;
    }
    // Fragment f of the keys.
    __device__ u32x4 key(int f) const {
        if constexpr (kE4m3) {
            const unsigned a = k[f / 2][2 * (f % 2)], b = k[f / 2][2 * (f % 2) + 1];
            return u32x4{T::template from_e4m3<false>(a), T::template from_e4m3<true>(a),
                         T::template from_e4m3<false>(b), T::template from_e4m3<true>(b)};
        } else {
            return k[f];
        }
    }
    // Words w (columns 2 w, 2 w + 1) of value i in 16 bits.
    __device__ unsigned value(int i, int w) const {
        if constexpr (kE4m3)
            return w % 2 ? P::template from_e4m3<true>(v[i][w / 2]) : P::template from_e4m3<false>(v[i][w / 2]);
        else
            return v[i][w];
    }
};

// The lane's constant part of the addresses.
template <class T, int kDim, bool kE4m3>
struct Places {
    typedef Keys<T, kDim, kE4m3> K;
    unsigned col, quad;
    unsigned kd[K::kLoads], vd;     // byte offsets inside a row, 0 behind dim
    __device__ Places(const AttendArgs& A, unsigned lane) {
        col = lane % 16;
        quad = lane / 16;
#pragma unroll
        for (int f = 0; f < K::kLoads; ++f) {
            const unsigned d = K::slot_dim(kE4m3 ? 2 * f : f, quad);
            kd[f] = d < A.dim ? d * (kE4m3 ? 1 : 2) : 0;
        }
        vd = col * K::kCols < A.dim ? col * K::kCols * (kE4m3 ? 1 : 2) : 0;
    }
};

// Loads the 16 keys and values from key `key0` (a multiple of 16) on, whose units
// lie in lanes `at` .. at + 15 of `unit`; tokens that are away are read from unit 0.
// kWide: pages of 16 tokens and more, so the 16 keys are of one unit, the same for all
// lanes, and their addresses differ by a 32-bit offset.
// kOnce: no other item reads them, so they go past the caches (131,071 tokens of one
// agent 111 us, through them 116 us).
template <class T, int kDim, bool kE4m3, bool kWide, bool kOnce>
__device__ __forceinline__ void load_keys(const AttendArgs& A, const Places<T, kDim, kE4m3>& p,
                                          unsigned head, int unit, unsigned at, unsigned key0,
                                          Keys<T, kDim, kE4m3>& x) {
    typedef Keys<T, kDim, kE4m3> K;
    const unsigned mask = (1u << A.shift) - 1u;
    const u64 head_off = (u64)head * A.head_bytes;
    auto read_once = [](auto* from) {
        if constexpr (kOnce) return __builtin_nontemporal_load(from);
        else return *from;
    };
    auto k_from = [&](const char* row) {
#pragma unroll
        for (int f = 0; f < K::kLoads; ++f) x.k[f] = read_once(reinterpret_cast<const u32x4*>(row + p.kd[f]));
    };
    auto v_from = [&](const char* row, int i) {
        if constexpr (K::kWords == 1) {
            x.v[i][0] = *reinterpret_cast<const unsigned*>(row);
        } else {
            const typename K::wide w = read_once(reinterpret_cast<const typename K::wide*>(row));
#pragma unroll
            for (int j = 0; j < K::kWords; ++j) x.v[i][j] = w[j];
        }
    };
    if constexpr (kWide) {
        const u64 u = unit < 0 ? 0 : unit;
        const unsigned slot = key0 & mask;
        const char* kb = A.k + u * A.k_unit + head_off + (u64)slot * A.token_bytes;
        const char* vb = A.v + u * A.v_unit + head_off + (u64)slot * A.token_bytes;
        const unsigned tb = (unsigned)A.token_bytes;
        k_from(kb + p.col * tb);
#pragma unroll
        for (int i = 0; i < 4; ++i) v_from(vb + ((4 * p.quad + i) * tb + p.vd), i);
        if constexpr (kE4m3) {
            const u64 so = A.scale_off + 4 * (((u64)head << A.shift) + slot);
            x.ks = *reinterpret_cast<const f32x4*>(A.k + u * A.k_unit + so + 16 * p.quad);
            x.vs = *reinterpret_cast<const f32x4*>(A.v + u * A.v_unit + so + 16 * p.quad);
        }
    } else {
        const int safe = unit < 0 ? 0 : unit;
        const u64 ku = (u64)__shfl(safe, at + p.col);
        k_from(A.k + ku * A.k_unit + head_off + (u64)((key0 + p.col) & mask) * A.token_bytes);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const u64 vu = (u64)__shfl(safe, at + 4 * p.quad + i);
            const unsigned slot = (key0 + 4 * p.quad + i) & mask;
            v_from(A.v + vu * A.v_unit + head_off + (u64)slot * A.token_bytes + p.vd, i);
            if constexpr (kE4m3) {
                const u64 so = A.scale_off + 4 * (((u64)head << A.shift) + slot);
                x.ks[i] = *reinterpret_cast<const float*>(A.k + vu * A.k_unit + so);
                x.vs[i] = *reinterpret_cast<const float*>(A.v + vu * A.v_unit + so);
            }
        }
    }
}

// What is stored where no token is may be anything: values become zeros (their
// weights are, but 0 * NaN is not).  Bit i of `there`: the lane's value i is a token.
template <class K>
__device__ __forceinline__ void clear_values(K& x, unsigned there) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (!(there >> i & 1)) {
#pragma unroll
            for (int w = 0; w < K::kWords; ++w) x.v[i][w] = 0;
        }
}

// The table's entry for key `key` of a segment, -1 where there is none, as it is read:
// whether it is a unit is asked when it is used, or the read would be waited for.
__device__ __forceinline__ int entry_of(const AttendArgs& A, u64 first, unsigned key, unsigned limit) {
    return key < limit ? A.tab.units[first + (key >> A.shift)] : -1;
}
__device__ __forceinline__ int unit_of(const AttendArgs& A, int entry) {
    return entry >= 0 && (u64)entry < A.tab.capacity ? entry : -1;
}

// The keys that an item reads: blocks [b0, b1) of the prefix's and the own tokens'
// blocks, of which the tile's rows see own tokens below `most`.
struct Range {
    unsigned nb0, most;
    unsigned b0, b1;            // below 2^28 + chunk
    __device__ Range(const AttendArgs& A, const Item& s, unsigned last_row, unsigned split) {
        most = (unsigned)min((long long)s.keys[1], max(0ll, (long long)s.see + last_row + 1));
        nb0 = (s.keys[0] + kBlock - 1) / kBlock;
        b0 = split * s.chunk;
        b1 = min(nb0 + (most + kBlock - 1) / kBlock, b0 + s.chunk);
    }
};

// Queries of one tile of 16 rows: row lane % 16, in the slots of the keys.  A scale of
// zero or less is taken into their bits, so that scores can be compared unscaled.
template <class T, int kDim, bool kE4m3>
__device__ __forceinline__ void load_queries(const AttendArgs& A, const Item& s, unsigned head,
                                             unsigned m, unsigned quad, u32x4* q) {
    const unsigned row = m / A.per, g = m - row * A.per;
    const bool in = m < s.rows * A.per;
    const char* from = A.q + (u64)(s.row0 + (in ? row : 0)) * A.q_row + (u64)(head * A.per + (in ? g : 0)) * A.q_head;
#pragma unroll
    for (int f = 0; f < kDim / 32; ++f) {
        const unsigned d = Keys<T, kDim, kE4m3>::slot_dim(f, quad);
        q[f] = u32x4{0, 0, 0, 0};
        if (in && d < A.dim) q[f] = (*reinterpret_cast<const u32x4*>(from + 2 * d) & A.q_keep) ^ A.q_flip;
    }
}

// Running reference and sum of one row's scores, and its weights.  `top` is an
// unscaled score; weights are 2^(scale (score - top) + lift), and sums are divided by 2^lift
// when they are complete.
struct Softmax {
    float top = -INFINITY, sum = 0.f;
    float off = 0.f;            // what is added to a scaled score
    float gate = -INFINITY;     // `top`, or -infinity in a row far from zero: every block is raised
    // Whether a score passes the reference by more than the slack (in some lane).
    __device__ bool passes(float best, float scale) const {
        return __any(best > gate && !((best - gate) * scale <= kSlack));
    }
    // Takes the largest score of the row (over the lanes that share it) as the new
    // reference; returns what older sums shrink by.  Score and reference are scaled and
    // rounded apart, so the difference of equal ones is off by 2^-24 of them: of a row whose
    // reference is beyond 2^12, it is taken from the scores themselves, block by block (for all
    // rows that is an instruction a score more: 16 prompts 697 us, so 676 us).
    template <int kScores>
    __device__ float raise(float best, float scale, float lift, f32x4* scores) {
        best = fmaxf(best, __shfl_xor(best, 16));
        best = fmaxf(best, __shfl_xor(best, 32));
        best = fmaxf(best, top);
        const float shrink = top == best ? 1.f : __builtin_amdgcn_exp2f((top - best) * scale);
        top = best;
        sum *= shrink;
        off = top == -INFINITY ? 0.f : fmaf(-top, scale, lift);
        const bool far = fabsf(off) > 4096.f;
        gate = far ? -INFINITY : top;
        if (__any(far)) {
#pragma unroll
            for (int j = 0; j < kScores; ++j) scores[j] -= far ? top : 0.f;
            off = far ? lift : off;
        }
        return shrink;
    }
    // log2 of what the row's sums are relative to, -infinity without any score.
    __device__ float reference(float scale) const { return top == -INFINITY ? -INFINITY : top * scale; }
};

// 16 rows and a range of keys.  The four waves take 64-key blocks in turn, each
// with a reference and sum of its own, and join at the end: with so few rows a key
// is used once, so it goes from memory to registers and through the products
// without a stop in LDS.  HBM bounds it; a wave keeps the loads of its next 16 KB in
// flight while it computes (bf16 at dim 128: 32 keys a step).
template <class T, int kDim, bool kE4m3, bool kWide>
__device__ void few_rows(const Item& s, unsigned head, char* lds) {
    const AttendArgs A = again();
    typedef Keys<T, kDim, kE4m3> K;
    typedef typename K::P P;
    constexpr int kCols = K::kCols, kFrags = K::kFrags;
    constexpr int kSub = kDim == 64 ? 4 : 2;            // 16-key pieces of a step
    constexpr unsigned kSteps = 4 / kSub;               // steps of a block
    float* lds_o = reinterpret_cast<float*>(lds);
    float2* lds_ml = reinterpret_cast<float2*>(lds + kWaves * 16 * (kDim + 4) * 4);
    const unsigned lane = own_lane(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const Places<T, kDim, kE4m3> p(A, lane);
    const unsigned col = p.col, quad = p.quad;
    const unsigned total = s.rows * A.per, tile = s.tile, split = s.split;
    const unsigned m = tile * 16 + col;                     // this lane's stack row
    const unsigned row = m / A.per, g = m - row * A.per;
    const unsigned last = min(total - 1, tile * 16 + 15) / A.per;
    const Range range(A, s, last, split);
    // own tokens that this lane's row sees
    const int lim = (int)min((long long)s.keys[1], max(0ll, (long long)s.see + row + 1));
    const unsigned row_first = tile * 16 / A.per;
    const unsigned lim_all = (unsigned)min((long long)s.keys[1], max(0ll, (long long)s.see + row_first + 1));
    u32x4 q[kFrags];
    load_queries<T, kDim, kE4m3>(A, s, head, m, quad, q);
    const float scale = A.scale;
    f32x4 o[kCols];
#pragma unroll
    for (int i = 0; i < kCols; ++i) o[i] = f32x4{0, 0, 0, 0};
    Softmax soft;

    const unsigned blocks = range.b1 > range.b0 + wave ? (range.b1 - range.b0 - wave + kWaves - 1) / kWaves : 0;
    const unsigned steps = blocks * kSteps;
    // step i: whether its keys are own tokens, and the first of them
    auto where = [&](unsigned i, bool* own, unsigned* key0) {
        const unsigned b = range.b0 + wave + i / kSteps * kWaves;
        *own = b >= range.nb0;
        *key0 = (*own ? b - range.nb0 : b) * kBlock + i % kSteps * (16 * kSub);
    };
    // The step's table entries.  Of pages of 16 tokens and more they are the same for all
    // lanes and come through the scalar cache, so that the count of vector reads on their
    // way is that of keys alone, and a step's can be waited for with the next one's out.
    struct Entries {
        int of[kWide ? kSub : 1];
    };
    auto look_up = [&](unsigned i) {
        bool own;
        unsigned key0;
        where(i, &own, &key0);
        const u64 first = own ? s.first[1] : s.first[0];
        const unsigned limit = own ? range.most : s.keys[0];
        Entries e;
        if constexpr (kWide) {
            const auto units = (const __attribute__((address_space(4))) int*)A.tab.units;
#pragma unroll
            for (int j = 0; j < kSub; ++j) {
                const unsigned key = key0 + 16 * j;
                e.of[j] = key < limit ? units[first + (key >> A.shift)] : -1;
            }
        } else {
            e.of[0] = entry_of(A, first, key0 + lane % (16 * kSub), limit);
        }
        return e;
    };
    struct Step {
        K x[kSub];
        u64 there;
    };
    auto load = [&](unsigned i, const Entries& e, Step& t) {
        bool own;
        unsigned key0;
        where(i, &own, &key0);
        if constexpr (kWide) {
            const unsigned limit = own ? range.most : s.keys[0];
            t.there = 0;
#pragma unroll
            for (int j = 0; j < kSub; ++j) {
                const int unit = unit_of(A, e.of[j]);
                const unsigned key = key0 + 16 * j, tokens = unit >= 0 && key < limit ? min(limit - key, 16u) : 0;
                t.there |= (u64)((1u << tokens) - 1u) << (16 * j);
                load_keys<T, kDim, kE4m3, kWide, true>(A, p, head, unit, 0, key, t.x[j]);
            }
        } else {
            const int unit = unit_of(A, e.of[0]);
            t.there = __ballot(unit >= 0);
#pragma unroll
            for (int j = 0; j < kSub; ++j)
                load_keys<T, kDim, kE4m3, kWide, true>(A, p, head, unit, 16 * j, key0 + 16 * j, t.x[j]);
        }
    };
    auto compute = [&](unsigned i, Step& t) {
        bool own;
        unsigned key0;
        where(i, &own, &key0);
        f32x4 st[kSub];
#pragma unroll
        for (int j = 0; j < kSub; ++j) {
            st[j] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int f = 0; f < kFrags; ++f) {
                u32x4 kf = t.x[j].key(f);
                if (A.dim != kDim && K::slot_dim(f, quad) >= A.dim) kf = u32x4{0, 0, 0, 0};
                st[j] = T::mma(kf, q[f], st[j]);
            }
            if constexpr (kE4m3) st[j] *= t.x[j].ks;
        }
        const u64 all = kSub == 4 ? ~0ull : (1ull << (16 * kSub)) - 1;
        if ((t.there & all) != all || (own && key0 + 16 * kSub > lim_all)) {
            // key i of the lane is seen below its row's limit (a few at a time: the compiler
            // would else hold all comparisons in scalar registers)
            const int rest = own ? lim - (int)(key0 + 4 * quad) : 64;
#pragma unroll
            for (int j = 0; j < kSub; ++j) {
                const unsigned bits = (unsigned)(t.there >> (16 * j + 4 * quad)) & 15u;
                clear_values(t.x[j], bits);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const bool seen = (bits >> c & 1) && 16 * j + c < rest;
                    st[j][c] = seen ? st[j][c] : -INFINITY;
                    if constexpr (kE4m3) t.x[j].vs[c] = seen ? t.x[j].vs[c] : 0.f;
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        float best = -INFINITY;
#pragma unroll
        for (int j = 0; j < kSub; ++j)
            best = fmaxf(fmaxf(fmaxf(best, st[j][0]), fmaxf(st[j][1], st[j][2])), st[j][3]);
        if (soft.passes(best, scale)) {
            const float shrink = soft.template raise<kSub>(best, scale, K::kLift, st);
#pragma unroll
            for (int c = 0; c < kCols; ++c) o[c] *= shrink;
        }
        const float off = soft.off;
        unsigned w[kSub][K::kParts][2];
#pragma unroll
        for (int j = 0; j < kSub; ++j) {
            f32x4 e;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                e[c] = __builtin_amdgcn_exp2f(fmaf(st[j][c], scale, off));
                soft.sum += e[c];
            }
            if constexpr (kE4m3) e *= t.x[j].vs;
            K::weights(e, w[j]);
        }
#pragma unroll
        for (int j = 0; j < kSub; j += 2) {
#pragma unroll
            for (int c = 0; c < kCols; ++c) {
                const unsigned sel = c % 2 ? 0x07060302u : 0x05040100u;
                const K &x = t.x[j], &y = t.x[j + 1];
                const u32x4 vf = {__builtin_amdgcn_perm(x.value(1, c / 2), x.value(0, c / 2), sel),
                                  __builtin_amdgcn_perm(x.value(3, c / 2), x.value(2, c / 2), sel),
                                  __builtin_amdgcn_perm(y.value(1, c / 2), y.value(0, c / 2), sel),
                                  __builtin_amdgcn_perm(y.value(3, c / 2), y.value(2, c / 2), sel)};
#pragma unroll
                for (int k = 0; k < K::kParts; ++k)
                    o[c] = P::mma(vf, u32x4{w[j][k][0], w[j][k][1], w[j + 1][k][0], w[j + 1][k][1]}, o[c]);
            }
        }
    };
    // entries are looked up two steps ahead of their use, keys asked for one ahead (where
    // 64 KB of registers hold two steps), with no condition in between that would make
    // the number of reads on their way unknown
    if (steps > 0) {
        if constexpr (kDim <= 128 || kE4m3) {
            Step a, b;
            load(0, look_up(0), a);
            Entries next = look_up(steps > 1 ? 1 : 0);
            unsigned i = 0;
            for (; i + 2 < steps; i += 2) {
                const Entries after = look_up(i + 2);
                load(i + 1, next, b);
                compute(i, a);
                next = look_up(i + 3 < steps ? i + 3 : i + 2);
                load(i + 2, after, a);
                compute(i + 1, b);
            }
            if (i + 1 < steps) {
                load(i + 1, next, b);
                compute(i, a);
                compute(i + 1, b);
            } else {
                compute(i, a);
            }
        } else {
            Entries next = look_up(0);
            for (unsigned i = 0; i < steps; ++i) {
                Step a;
                load(i, next, a);
                if (i + 1 < steps) next = look_up(i + 1);
                compute(i, a);
            }
        }
    }
    float sum = soft.sum * K::kUnlift;
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    const float top = soft.reference(scale);

    // join the four waves: lds_o[wave][row][kDim + 4], lds_ml[wave][row]
    constexpr int kPitch = kDim + 4;
    if (quad == 0) lds_ml[wave * 16 + col] = float2{top, sum};
    __syncthreads();
    float best = -INFINITY, l = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) best = fmaxf(best, lds_ml[w * 16 + col].x);
    const float ref = best == -INFINITY ? 0.f : best;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) l += lds_ml[w * 16 + col].y * exp2f(lds_ml[w * 16 + col].x - ref);
    const bool direct = s.part == ~0ull;
    const float mine = exp2f(top - ref) * K::kUnlift * (direct ? (l == 0.f ? 0.f : 1.f / l) : 1.f);
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int i = 0; i < kCols; ++i)
            lds_o[(wave * 16 + col) * kPitch + (4 * quad + r) * kCols + i] = o[i][r] * mine;
    __syncthreads();
    const u64 part0 = s.part + ((u64)head * s.splits + split) * total;
    for (unsigned e = threadIdx.x; e < 16 * (kDim / 4); e += kWaves * 64) {
        const unsigned mm = e / (kDim / 4), d = e % (kDim / 4) * 4;
        const unsigned sm = tile * 16 + mm;
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
                    (best + log2f(l)) * 0.6931471805599453f;
        } else {
            A.part_ml[part0 + m] = float2{best, l};
        }
    }
}

// A block of 64 keys and values in LDS, in the layout of the products' operands, and
// how it gets there.  A fragment of keys is 64 lanes x 16 bytes, read without bank
// conflicts.  Wave w brings the block's keys 16 w .. 16 w + 15 while the products of the
// block before run.
// Through registers (e4m3, which is converted on the way, and dims that are filled
// up): values are transposed by byte permutes, so their fragments are like the keys'.
template <class T, int kDim, bool kE4m3, bool kWide>
struct ThroughRegisters {
    typedef Keys<T, kDim, kE4m3> K;
    static constexpr int kCols = K::kCols, kFrags = K::kFrags;
    static constexpr unsigned kKeyBytes = 4 * kFrags * 1024, kValueBytes = 2 * kCols * 1024;
    static constexpr unsigned kBuffer = kKeyBytes + kValueBytes + 512;
    Places<T, kDim, kE4m3> p;
    K x;
    unsigned lane, wave;
    __device__ ThroughRegisters(const AttendArgs& A, unsigned l, unsigned w) : p(A, l), lane(l), wave(w) {}
    // Asks for the wave's keys of the block at key0 into buffer `to`.
    __device__ void ask(const AttendArgs& A, unsigned head, int unit, unsigned key0, char*) {
        load_keys<T, kDim, kE4m3, kWide, false>(A, p, head, kWide ? __builtin_amdgcn_readlane(unit, 16 * wave) : unit,
                                         16 * wave, key0 + 16 * wave, x);
    }
    // Has them in the buffer, for all waves; `there`: the block's keys that are tokens.
    __device__ void arrive(const AttendArgs& A, u64 there, char* to) {
        char* const lv = to + kKeyBytes;
        float* const ls = reinterpret_cast<float*>(lv + kValueBytes);
        if (there != ~0ull) {
            const unsigned bits = (unsigned)(there >> (16 * wave + 4 * p.quad)) & 15u;
            clear_values(x, bits);
            if constexpr (kE4m3) {
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (!(bits >> c & 1)) x.ks[c] = x.vs[c] = 0.f;
            }
        }
#pragma unroll
        for (int f = 0; f < kFrags; ++f) {
            u32x4 kf = x.key(f);
            if (A.dim != kDim && K::slot_dim(f, p.quad) >= A.dim) kf = u32x4{0, 0, 0, 0};
            *reinterpret_cast<u32x4*>(to + ((wave * kFrags + f) * 64 + lane) * 16) = kf;
        }
#pragma unroll
        for (int c = 0; c < kCols; ++c) {
            const unsigned sel = c % 2 ? 0x07060302u : 0x05040100u;
            const u32x2 vf = {__builtin_amdgcn_perm(x.value(1, c / 2), x.value(0, c / 2), sel),
                              __builtin_amdgcn_perm(x.value(3, c / 2), x.value(2, c / 2), sel)};
            *reinterpret_cast<u32x2*>(lv + (((wave / 2) * kCols + c) * 64 + lane) * 16 + (wave % 2) * 8) = vf;
        }
        if constexpr (kE4m3) {
            if (p.col == 0) {
                *reinterpret_cast<f32x4*>(ls + 16 * wave + 4 * p.quad) = x.ks;
                *reinterpret_cast<f32x4*>(ls + 64 + 16 * wave + 4 * p.quad) = x.vs;
            }
        }
        __syncthreads();
    }
    // Fragment i of the keys, 16 of them for each kFrags.
    __device__ u32x4 key(const char* from, int i) const {
        return *reinterpret_cast<const u32x4*>(from + (i * 64 + lane) * 16);
    }
    // Fragment c of the values of keys 32 h ..; row r of a lane's product is the column:
    __device__ u32x4 value(const char* from, int h, int c) const {
        return *reinterpret_cast<const u32x4*>(from + kKeyBytes + ((h * kCols + c) * 64 + lane) * 16);
    }
    static constexpr __host__ __device__ unsigned column(unsigned quad, int r, int c) { return (4 * quad + r) * kCols + c; }
    __device__ f32x4 scales(const char* from, unsigned what, unsigned key) const {
        return *reinterpret_cast<const f32x4*>(from + kKeyBytes + kValueBytes + 4 * (64 * what + key));
    }
};

// Straight from memory into LDS, without registers (16-bit caches of the full dim): a
// wave's read puts lane l's 16 bytes at l * 16, so the layout lies in which bytes
// each lane asks for.  Values keep their rows, 16-byte pieces c of key k at c ^ 2 (k % 8)
// (16 rows' 32 bytes would else share their banks), and are transposed when read:
// of four rows that 16 lanes point at, each lane gets one column.
template <class T, int kDim, bool kWide>
struct Straight {
    static constexpr int kCols = kDim / 16, kFrags = kDim / 32, kPieces = kDim / 8;
    static constexpr unsigned kKeyBytes = 64 * kDim * 2;
    static constexpr unsigned kBuffer = 2 * kKeyBytes;
    static constexpr unsigned kTurn = kPieces < 16 ? 3 : 7;       // pieces are turned in pairs
    unsigned lane, wave, col, quad;
    __device__ Straight(const AttendArgs&, unsigned l, unsigned w) : lane(l), wave(w), col(l % 16), quad(l / 16) {}
    typedef const __attribute__((address_space(1))) char* global;
    static __device__ void bring(global from, char* to) {
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                         (__attribute__((address_space(3))) void*)to, 16, 0, 0);
    }
    static __device__ unsigned turn(unsigned key) { return 2 * (key & kTurn); }
    __device__ void ask(const AttendArgs& A, unsigned head, int unit, unsigned key0, char* to) {
        const unsigned mask = (1u << A.shift) - 1u;
        const u64 head_off = (u64)head * A.head_bytes;
        const unsigned first = key0 + 16 * wave;
        // the wave's keys: fragments, then rows of values (kPieces lanes a row)
        char* const lk = to + wave * kFrags * 1024;
        char* const lv = to + kKeyBytes + wave * (16 * kDim * 2);
        constexpr unsigned kRowsAtOnce = 64 / kPieces;
        if constexpr (kWide) {
            const int u0 = __builtin_amdgcn_readlane(unit, 16 * wave);
            const u64 u = u0 < 0 ? 0 : u0;
            const unsigned tb = (unsigned)A.token_bytes;
            const u64 slot = (u64)(first & mask) * A.token_bytes + head_off;
            const global kb = (global)(A.k + (u * A.k_unit + slot)), vb = (global)(A.v + (u * A.v_unit + slot));
            const unsigned k_at = col * tb + 16 * quad;
#pragma unroll
            for (int f = 0; f < kFrags; ++f) bring(kb + 64 * f + k_at, lk + f * 1024);
#pragma unroll
            for (unsigned n = 0; n < 16 / kRowsAtOnce; ++n) {
                const unsigned key = n * kRowsAtOnce + lane / kPieces;
                bring(vb + (key * tb + 16 * (lane % kPieces ^ turn(key))), lv + n * 1024);
            }
        } else {
            const int safe = unit < 0 ? 0 : unit;
            const u64 ku = (u64)__shfl(safe, 16 * wave + col);
            const char* const kb = A.k + ku * A.k_unit + (u64)((first + col) & mask) * A.token_bytes + head_off;
#pragma unroll
            for (int f = 0; f < kFrags; ++f) bring((global)(kb + (64 * f + 16 * quad)), lk + f * 1024);
#pragma unroll
            for (unsigned n = 0; n < 16 / kRowsAtOnce; ++n) {
                const unsigned key = n * kRowsAtOnce + lane / kPieces;
                const u64 vu = (u64)__shfl(safe, 16 * wave + key);
                bring((global)(A.v + vu * A.v_unit + (u64)((first + key) & mask) * A.token_bytes + head_off +
                               16 * (lane % kPieces ^ turn(key))), lv + n * 1024);
            }
        }
    }
    __device__ void arrive(const AttendArgs&, u64 there, char* to) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (there == ~0ull) return;
        // what is stored where no token is may be anything
        for (unsigned i = threadIdx.x; i < 64 * kPieces; i += kWaves * 64)
            if (!(there >> (i / kPieces) & 1))
                *reinterpret_cast<u32x4*>(to + kKeyBytes + i * 16) = u32x4{0, 0, 0, 0};
        __syncthreads();
    }
    __device__ u32x4 key(const char* from, int i) const {
        return *reinterpret_cast<const u32x4*>(from + (i * 64 + lane) * 16);
    }
    __device__ u32x4 value(const char* from, int h, int c) const {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s16x4 lds4;
        // this lane's row of the four that its quarter wave turns, and 8 bytes of it
        const unsigned key = 32 * h + 4 * quad + col / 4, piece = 2 * c + (col % 4) / 2;
        const char* at = from + kKeyBytes + key * (kDim * 2) + 16 * (piece ^ turn(key)) + 8 * (col % 2);
        // 16 keys on, turned alike; written out, as the compiler else takes it for the buffer
        // that the next block comes into and waits for that (16 prompts 776 us)
        const char* at2 = from + kKeyBytes + (key + 16) * (kDim * 2) + 16 * (piece ^ turn(key)) + 8 * (col % 2);
        const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)at);
        const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)at2);
        const u32x2 x = __builtin_bit_cast(u32x2, a), y = __builtin_bit_cast(u32x2, b);
        return u32x4{x[0], x[1], y[0], y[1]};
    }
    static constexpr __host__ __device__ unsigned column(unsigned quad, int r, int c) { return 16 * c + 4 * quad + r; }
    __device__ f32x4 scales(const char*, unsigned, unsigned) const { return f32x4{1, 1, 1, 1}; }
};

// 64 kQ rows and a range of keys: each wave has 16 kQ rows and all keys, and a block of
// 64 keys and values comes into LDS once for the four waves.  From about 150 rows on
// the products bound it, below HBM does.
template <class T, int kDim, bool kE4m3, int kQ, class Blocks>
__device__ void many_rows(const Item& s, unsigned head, char* lds0, char* lds1) {
    const AttendArgs A = again();
    typedef Keys<T, kDim, kE4m3> K;
    typedef typename K::P P;
    constexpr int kCols = kDim / 16, kFrags = kDim / 32;
    const unsigned lane = own_lane(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const unsigned col = lane % 16, quad = lane / 16;
    Blocks keys(A, lane, wave);
    const unsigned total = s.rows * A.per, tile = s.tile, split = s.split;
    const unsigned m0 = tile * 64 * kQ, mw = m0 + wave * 16 * kQ;   // the tile's, the wave's first row
    const unsigned last = min(total - 1, m0 + 64 * kQ - 1) / A.per;
    const Range range(A, s, last, split);
    int lim[kQ];
    u32x4 q[kQ][kFrags];
    f32x4 o[kQ][kCols];
    Softmax soft[kQ];
#pragma unroll
    for (int t = 0; t < kQ; ++t) {
        const unsigned m = mw + 16 * t + col;
        lim[t] = (int)min((long long)s.keys[1], max(0ll, (long long)s.see + m / A.per + 1));
        load_queries<T, kDim, kE4m3>(A, s, head, m, quad, q[t]);
#pragma unroll
        for (int i = 0; i < kCols; ++i) o[t][i] = f32x4{0, 0, 0, 0};
    }
    // own tokens that all rows of the wave see
    const unsigned lim_all = (unsigned)min((long long)s.keys[1],
                                           max(0ll, (long long)s.see + mw / A.per + 1));
    const float scale = A.scale;
    auto look_up = [&](unsigned b) {
        const bool own = b >= range.nb0;
        return entry_of(A, own ? s.first[1] : s.first[0], (own ? b - range.nb0 : b) * kBlock + lane,
                       own ? range.most : s.keys[0]);
    };
    auto key_of = [&](unsigned b) { return (b >= range.nb0 ? b - range.nb0 : b) * kBlock; };
    // units are looked up two blocks ahead of their use, keys asked for one ahead
    int next = -1, after = -1;
    if (range.b0 < range.b1) {
        next = look_up(range.b0);
        if (range.b0 + 1 < range.b1) after = look_up(range.b0 + 1);
        keys.ask(A, head, unit_of(A, next), key_of(range.b0), lds0);
    }
    // One block, in buffer `here`, while the next one comes into `there`.  The products'
    // fragments are read a group ahead of their use: an LDS read takes about as long as
    // eight products, and the compiler by itself waits for each (16 prompts 989 us).
    auto block = [&](unsigned b, char* __restrict__ here, char* __restrict__ beside) {
        const u64 there = __ballot(unit_of(A, next) >= 0);
        next = after;
        keys.arrive(A, there, here);
        if (b + 1 < range.b1) keys.ask(A, head, unit_of(A, next), key_of(b + 1), beside);
        if (b + 2 < range.b1) after = look_up(b + 2);
        // scores
        f32x4 st[kQ][4];
        u32x4 kf[2][kFrags];
#pragma unroll
        for (int f = 0; f < kFrags; ++f) kf[0][f] = keys.key(here, f);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (j < 3) {
#pragma unroll
                for (int f = 0; f < kFrags; ++f) kf[(j + 1) % 2][f] = keys.key(here, (j + 1) * kFrags + f);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < kQ; ++t) st[t][j] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int f = 0; f < kFrags; ++f)
#pragma unroll
                for (int t = 0; t < kQ; ++t) st[t][j] = T::mma(kf[j % 2][f], q[t][f], st[t][j]);
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (kE4m3) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const f32x4 ks = keys.scales(here, 0, 16 * j + 4 * quad);
#pragma unroll
                for (int t = 0; t < kQ; ++t) st[t][j] *= ks;
            }
        }
        // values in groups of kGroup columns' fragments, the first one while the
        // weights are worked out
        constexpr int kGroup = 4, kGroups = 2 * kCols / kGroup;
        u32x4 vf[2][kGroup];
#pragma unroll
        for (int g = 0; g < kGroup; ++g) vf[0][g] = keys.value(here, 0, g);
        const bool own = b >= range.nb0;
        const unsigned key0 = key_of(b);
        if (there != ~0ull || (own && key0 + kBlock > lim_all)) {
            // key i of the lane's 16 is seen below its row's limit (a few at a time: the
            // compiler would else hold 64 comparisons in scalar registers)
#pragma unroll
            for (int t = 0; t < kQ; ++t) {
                const int rest = own ? lim[t] - (int)(key0 + 4 * quad) : 64;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const unsigned bits = (unsigned)(there >> (16 * j + 4 * quad));
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        st[t][j][c] = (bits >> c & 1) && 16 * j + c < rest ? st[t][j][c] : -INFINITY;
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        unsigned w[kQ][4][K::kParts][2];
#pragma unroll
        for (int t = 0; t < kQ; ++t) {
            float best = -INFINITY;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                best = fmaxf(fmaxf(fmaxf(best, st[t][j][0]), fmaxf(st[t][j][1], st[t][j][2])), st[t][j][3]);
            if (soft[t].passes(best, scale)) {
                const float shrink = soft[t].template raise<4>(best, scale, K::kLift, st[t]);
#pragma unroll
                for (int c = 0; c < kCols; ++c) o[t][c] *= shrink;
            }
            const float off = soft[t].off;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                f32x4 e;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    e[c] = __builtin_amdgcn_exp2f(fmaf(st[t][j][c], scale, off));
                    soft[t].sum += e[c];
                }
                if constexpr (kE4m3) e *= keys.scales(here, 1, 16 * j + 4 * quad);
                K::weights(e, w[t][j]);
            }
        }
#pragma unroll
        for (int i = 0; i < kGroups; ++i) {
            if (i + 1 < kGroups) {
#pragma unroll
                for (int g = 0; g < kGroup; ++g)
                    vf[(i + 1) % 2][g] = keys.value(here, (i + 1) * kGroup / kCols, (i + 1) * kGroup % kCols + g);
            }
            __builtin_amdgcn_sched_barrier(0);
            const int h = i * kGroup / kCols, c = i * kGroup % kCols;
#pragma unroll
            for (int g = 0; g < kGroup; ++g)
#pragma unroll
                for (int k = 0; k < K::kParts; ++k)
#pragma unroll
                    for (int t = 0; t < kQ; ++t)
                        o[t][c + g] = P::mma(vf[i % 2][g], u32x4{w[t][2 * h][k][0], w[t][2 * h][k][1],
                                                                 w[t][2 * h + 1][k][0], w[t][2 * h + 1][k][1]},
                                             o[t][c + g]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    for (unsigned b = range.b0; b < range.b1; b += 2) {
        block(b, lds0, lds1);
        if (b + 1 < range.b1) block(b + 1, lds1, lds0);
    }
    const bool direct = s.part == ~0ull;
    const u64 part0 = s.part + ((u64)head * s.splits + split) * total;
#pragma unroll
    for (int t = 0; t < kQ; ++t) {
        const unsigned m = mw + 16 * t + col;
        float sum = soft[t].sum * K::kUnlift;
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        const float top = soft[t].reference(scale);
        if (m >= total) continue;
        const unsigned row = m / A.per, hh = head * A.per + (m - row * A.per);
        const float mine = K::kUnlift * (direct ? (sum == 0.f ? 0.f : 1.f / sum) : 1.f);
        char* to = A.out + (u64)(s.row0 + row) * A.out_row + (u64)hh * A.out_head;
        // four columns next to each other, of one product's rows or of four products
        constexpr bool kByRow = Blocks::column(0, 1, 0) == 1;
#pragma unroll
        for (int r = 0; r < (kByRow ? 1 : 4); ++r)
#pragma unroll
            for (int c = 0; c < kCols; c += kByRow ? 1 : 4) {
                const unsigned d = Blocks::column(quad, r, c);
                if (d >= A.dim) continue;
                const f32x4 y = (kByRow ? o[t][c] : f32x4{o[t][c][r], o[t][c + (kByRow ? 0 : 1)][r],
                                                          o[t][c + (kByRow ? 0 : 2)][r],
                                                          o[t][c + (kByRow ? 0 : 3)][r]}) * mine;
                if (direct)
                    *reinterpret_cast<u32x2*>(to + 2 * d) = u32x2{T::pack(y[0], y[1]), T::pack(y[2], y[3])};
                else
                    *reinterpret_cast<f32x4*>(&A.part_o[(part0 + m) * kDim + d]) = y;
            }
        if (quad == 0) {
            if (direct) {
                if (A.lse) A.lse[(u64)(s.row0 + row) * (A.n_heads * A.per) + hh] =
                    (top + log2f(sum)) * 0.6931471805599453f;
            } else {
                A.part_ml[part0 + m] = float2{top, sum};
            }
        }
    }
}

// kFull: a 16-bit cache whose dim is kDim.
template <class T, int kDim, bool kE4m3, bool kWide, bool kFull>
__global__ __launch_bounds__(kWaves * 64, kDim > 128 ? 1 : 2) void k_attend(AttendArgs A) {
    // two buffers of a block's keys, values and scales, or the waves' sums; two arrays,
    // so that reads of the one do not wait for what comes into the other
    constexpr int kBlocks = kDim * 256 + 512, kSums = kWaves * 16 * (kDim + 4) * 4 + kWaves * 16 * 8;
    __shared__ __align__(16) char lds[kBlocks > kSums ? kBlocks : kSums];
    __shared__ __align__(16) char lds1[kBlocks];
    __shared__ unsigned s_ticket[2];
    const unsigned n = A.counts[0] * A.n_heads;
    // Items are taken as workgroups get free, item i by XCD i % 8 first (workgroups go
    // round the XCDs), so that tiles next to each other, which read the same keys, share a
    // cache.  Which workgroup computes an item changes nothing in its result.  The next
    // number is asked for early and looked at late; asked for two ahead, workgroups hold
    // items that others could take (64 agents over 8,192 tokens 84 us, as it is 70 us).
    unsigned it = blockIdx.x, xcd = blockIdx.x % kXcds;
    for (unsigned turn = 0; it < n; turn ^= 1) {
        unsigned ticket = 0;
        if (threadIdx.x == 0) ticket = atomicAdd(&A.taken[16 * xcd], 1u);
        const unsigned head = it % A.n_heads;
        const Item s = A.items[it / A.n_heads];
        if (s.tile_rows == 16) {
            few_rows<T, kDim, kE4m3, kWide>(s, head, lds);
        } else {
            typedef typename std::conditional<kFull, Straight<T, kDim, kWide>,
                                              ThroughRegisters<T, kDim, kE4m3, kWide>>::type Blocks;
            if (kDim > 128 || s.tile_rows == 64) many_rows<T, kDim, kE4m3, 1, Blocks>(s, head, lds, lds1);
            else if constexpr (kDim <= 128) many_rows<T, kDim, kE4m3, 2, Blocks>(s, head, lds, lds1);
        }
        if (threadIdx.x == 0) {
            // the first gridDim.x items are the workgroups' own
            ticket = gridDim.x + ticket * kXcds + xcd;
            if (ticket >= n) {                  // then those of the XCD that has most left
                unsigned least = ~0u, x = 0;
                for (unsigned k = 0; k < kXcds; ++k) {
                    const unsigned c = __hip_atomic_load(&A.taken[16 * k], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    if (c < least) {
                        least = c;
                        x = k;
                    }
                }
                if (gridDim.x + least * kXcds + x < n)
                    ticket = gridDim.x + atomicAdd(&A.taken[16 * x], 1u) * kXcds + x;
            }
            s_ticket[turn] = ticket;
        }
        __syncthreads();
        it = s_ticket[turn];
    }
}

// Joins the parts of rows that several items share: kTeam waves take a row and query
// head, wave w every kTeam-th part from w on, kDim / 64 columns a lane; a team's waves
// meet in LDS.  Reads that wait for each other bound it (parts come from other XCDs'
// caches), so the parts are read along with their references, eight at a time, and
// small batches get a workgroup a row (one wave took 81 us for 128 parts of 32 rows).
template <class T, int kDim, int kTeam>
__device__ __forceinline__ void join_row(const AttendArgs& A, unsigned w, float (*s_x)[kDim], float2* s_ml) {
    constexpr int kCols = kDim / 64;
    const unsigned lane = threadIdx.x % 64, member = kTeam == 1 ? 0 : threadIdx.x / 64;
    const unsigned heads = A.n_heads * A.per;
    const JoinRow r = A.joins[w / heads];
    const unsigned qh = w % heads, head = qh / A.per, g = qh - head * A.per;
    const u64 first0 = r.first[0] + (u64)head * r.splits[0] * r.total[0] + g;
    const u64 first1 = r.first[1] + (u64)head * r.splits[1] * r.total[1] + g;
    const unsigned parts = r.splits[0] + r.splits[1];
    float top = -INFINITY, sum = 0.f, x[kCols];
#pragma unroll
    for (int c = 0; c < kCols; ++c) x[c] = 0.f;
    constexpr int kRead = kDim > 128 ? 4 : 8;
    for (unsigned i0 = member; i0 < parts; i0 += kTeam * kRead) {
        float2 ml[kRead];
        float y[kRead][kCols];
#pragma unroll
        for (int k = 0; k < kRead; ++k) {
            const unsigned i = min(i0 + k * kTeam, parts - 1);
            const u64 at = i < r.splits[0] ? first0 + (u64)i * r.total[0]
                                           : first1 + (u64)(i - r.splits[0]) * r.total[1];
            ml[k] = A.part_ml[at];
            const float* from = &A.part_o[at * kDim + lane * kCols];
#pragma unroll
            for (int c = 0; c < kCols; ++c) y[k][c] = from[c];
        }
        float best = top;
#pragma unroll
        for (int k = 0; k < kRead; ++k) {
            if (i0 + k * kTeam >= parts) ml[k] = float2{-INFINITY, 0.f};
            best = fmaxf(best, ml[k].x);
        }
        const float ref = best == -INFINITY ? 0.f : best, shrink = exp2f(top - ref);
        top = best;
        sum *= shrink;
#pragma unroll
        for (int c = 0; c < kCols; ++c) x[c] *= shrink;
#pragma unroll
        for (int k = 0; k < kRead; ++k) {
            const float f = exp2f(ml[k].x - ref);
            sum += ml[k].y * f;
            // columns behind dim, and of a part that is not there, may hold anything
#pragma unroll
            for (int c = 0; c < kCols; ++c) x[c] += i0 + k * kTeam < parts ? y[k][c] * f : 0.f;
        }
    }
    if constexpr (kTeam > 1) {
        if (lane == 0) s_ml[member] = float2{top, sum};
#pragma unroll
        for (int c = 0; c < kCols; ++c) s_x[member][lane * kCols + c] = x[c];
        __syncthreads();
        if (member == 0) {
#pragma unroll
            for (int k = 1; k < kTeam; ++k) {
                const float2 ml = s_ml[k];
                const float best = fmaxf(top, ml.x), ref = best == -INFINITY ? 0.f : best;
                const float a = exp2f(top - ref), b = exp2f(ml.x - ref);
                top = best;
                sum = sum * a + ml.y * b;
#pragma unroll
                for (int c = 0; c < kCols; ++c) x[c] = x[c] * a + s_x[k][lane * kCols + c] * b;
            }
        }
    }
    if (member == 0) {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        unsigned short* to = reinterpret_cast<unsigned short*>(A.out + (u64)r.row * A.out_row +
                                                               (u64)qh * A.out_head) + lane * kCols;
        if (lane * kCols < A.dim) {
            if constexpr (kCols == 1) {
                *to = (unsigned short)T::pack(x[0] * inv, 0.f);
            } else {
#pragma unroll
                for (int c = 0; c < kCols; c += 2)
                    reinterpret_cast<unsigned*>(to)[c / 2] = T::pack(x[c] * inv, x[c + 1] * inv);
            }
        }
        if (A.lse && lane == 0) A.lse[(u64)r.row * heads + qh] = (top + log2f(sum)) * 0.6931471805599453f;
    }
    if constexpr (kTeam > 1) __syncthreads();
}

template <class T, int kDim>
__global__ __launch_bounds__(256) void k_attend_join(AttendArgs A) {
    __shared__ float s_x[4][kDim];
    __shared__ float2 s_ml[4];
    const unsigned n = A.counts[1] * (A.n_heads * A.per);      // below 2^30
    if (n <= gridDim.x) {
        if (blockIdx.x < n) join_row<T, kDim, 4>(A, blockIdx.x, s_x, s_ml);
    } else {
        for (unsigned w = blockIdx.x * 4 + threadIdx.x / 64; w < n; w += gridDim.x * 4)
            join_row<T, kDim, 1>(A, w, s_x, s_ml);
    }
}

unsigned padded(unsigned dim) { return dim <= 64 ? 64 : dim <= 128 ? 128 : 256; }
u64 up(u64 x) { return (x + 255) & ~255ull; }

// Partial rows at most: every row once for its own tokens and once for a shared
// prefix, and a tile for each split beyond a stack's first; there are at most
// kTarget of those (and a few for the work's rounding), as every one but a stack's
// last has its share of the work.
constexpr u64 kMoreItems = kTarget + 16;
u64 part_rows(u64 n_rows, u64 n_q_heads) { return 2 * n_rows * n_q_heads + kMoreItems * kMostRows; }

// Items per head at most: a tile of every 16 rows and every stack's last one, once for
// own tokens and once for prefixes, and the splits.
u64 most_items(u64 n_rows, u64 n_stacks, u64 per) { return 2 * (n_rows * per / 16) + n_stacks + kMoreItems; }

struct Layout {
    u64 items, joins, stacks, ml, o, bytes;
};
Layout layout_of(u64 n_rows, u64 n_requests, u64 n_groups, u64 n_heads, u64 per, unsigned dim) {
    Layout l;
    const u64 n = n_requests + n_groups, rows = part_rows(n_rows, n_heads * per);
    l.items = 1024;
    l.joins = up(l.items + sizeof(Item) * most_items(n_rows, n, per));
    l.stacks = up(l.joins + sizeof(JoinRow) * n_rows);
    l.ml = up(l.stacks + sizeof(Stack) * n_groups);
    l.o = up(l.ml + 8 * rows);
    l.bytes = l.o + 4 * rows * padded(dim);
    return l;
}

template <class T, int kDim, bool kE4m3>
void attend_launch(const AttendArgs& A, unsigned cus, hipStream_t st) {
    hipLaunchKernelGGL(k_attend_plan, dim3(1), dim3(kPlanThreads), 0, st, A);
    const dim3 grid((cus * (kDim > 128 ? 1 : 2) + kXcds - 1) / kXcds * kXcds), block(kWaves * 64);
    const bool wide = A.shift >= 4, full = !kE4m3 && A.dim == kDim;
    if (full && wide) hipLaunchKernelGGL((k_attend<T, kDim, kE4m3, true, !kE4m3>), grid, block, 0, st, A);
    else if (full) hipLaunchKernelGGL((k_attend<T, kDim, kE4m3, false, !kE4m3>), grid, block, 0, st, A);
    else if (wide) hipLaunchKernelGGL((k_attend<T, kDim, kE4m3, true, false>), grid, block, 0, st, A);
    else hipLaunchKernelGGL((k_attend<T, kDim, kE4m3, false, false>), grid, block, 0, st, A);
    const u64 rows = (u64)A.n_rows * A.n_heads * A.per;
    hipLaunchKernelGGL((k_attend_join<T, kDim>), dim3((unsigned)std::min<u64>(rows, 8 * cus)), dim3(256), 0,
                       st, A);
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
    if ((u64)b->n_rows * n_q_heads >= (1ull << 30))
        return set_err(SS_ERR_ARG, "n_rows * n_q_heads must be below 2^30");
    const u64 n_stacks = (u64)b->n_requests + b->n_groups;
    if (most_items(b->n_rows, n_stacks, n_q_heads / c->n_heads) * c->n_heads >= (1ull << 31))
        return set_err(SS_ERR_ARG, "(n_requests + n_groups) * n_heads is too large");
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
    return layout_of(batch->n_rows, batch->n_requests, batch->n_groups, cache->n_heads,
                     n_q_heads / cache->n_heads, cache->head_dim).bytes;
}

ss_status ss_prefix_attention(const ss_kv_cache* cache, const ss_batch* batch, const void* q,
                              void* out, float* lse, uint32_t type, uint32_t n_q_heads,
                              uint64_t q_row_stride, uint64_t q_head_stride,
                              uint64_t out_row_stride, uint64_t out_head_stride, float scale,
                              void* workspace, uint64_t workspace_bytes, void* stream) {
    ss_status s = attend_args(cache, batch, type, n_q_heads);
    if (s != SS_OK) return s;
    if (!std::isfinite(scale * 1.4426950408889634f))
        return set_err(SS_ERR_ARG, "scale must be finite, also times log2(e)");
    if (batch->n_rows == 0 || batch->n_requests == 0) return SS_OK;
    const unsigned dim = cache->head_dim;
    const u64 rows = batch->n_rows;
    if ((s = rows_args("q", q, rows, n_q_heads, dim, q_row_stride, q_head_stride, false)) != SS_OK ||
        (s = rows_args("out", out, rows, n_q_heads, dim, out_row_stride, out_head_stride, true)) != SS_OK)
        return s;
    const Layout l = layout_of(rows, batch->n_requests, batch->n_groups, cache->n_heads,
                               n_q_heads / cache->n_heads, dim);
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15))
        return set_err(SS_ERR_ARG, "workspace must be a 16-byte aligned pointer");
    if (workspace_bytes < l.bytes)
        return set_err(SS_ERR_ARG, "workspace_bytes %llu < %llu", (unsigned long long)workspace_bytes,
                       (unsigned long long)l.bytes);
    const u64 q_bytes = rows_bytes(rows, n_q_heads, dim, q_row_stride, q_head_stride);
    const u64 out_bytes = rows_bytes(rows, n_q_heads, dim, out_row_stride, out_head_stride);
    const uintptr_t q0 = reinterpret_cast<uintptr_t>(q), o0 = reinterpret_cast<uintptr_t>(out);
    if (q0 < o0 + out_bytes && o0 < q0 + q_bytes) return set_err(SS_ERR_ARG, "out overlaps q");
    DeviceMemory mem;
    if ((s = mem.current()) != SS_OK || (s = cache_memory(cache, mem)) != SS_OK ||
        (s = batch_memory(batch, true, true, mem)) != SS_OK)
        return s;
    if (!mem.has(q, q_bytes)) return device_error("q", mem.dev);
    if (!mem.has(out, out_bytes)) return device_error("out", mem.dev);
    if (lse && !mem.has(lse, rows * n_q_heads * 4)) return device_error("lse", mem.dev);
    if (!mem.has(workspace, l.bytes)) return device_error("workspace", mem.dev);
    int cus = 256;
    if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, mem.dev) != hipSuccess) {
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
    A.scale = scale == 0.f ? 1.f : fabsf(scale) * 1.4426950408889634f;
    A.q_keep = scale == 0.f ? 0u : ~0u;
    A.q_flip = scale < 0.f ? 0x80008000u : 0u;
    char* ws = static_cast<char*>(workspace);
    A.counts = reinterpret_cast<unsigned*>(ws);
    A.taken = A.counts + 64;
    A.items = reinterpret_cast<Item*>(ws + l.items);
    A.joins = reinterpret_cast<JoinRow*>(ws + l.joins);
    A.most_items = most_items(rows, batch->n_requests + batch->n_groups, n_q_heads / cache->n_heads);
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
