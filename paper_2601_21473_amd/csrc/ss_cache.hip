// Tokens into and out of a pool's KV pages (ss_kv_write, ss_kv_read), and the
// argument checks of every operator over resident units.
//
// Both directions move each byte once and compute next to nothing, so HBM bounds
// them and the layout follows the memory: 16 bytes a lane on the 16-bit side, a
// head's row in 8, 16 or 32 consecutive lanes, so that the largest |x| of a row
// needs 3 to 5 lane exchanges and no memory.
#include <algorithm>
#include <cmath>

#include "ss_model.h"

namespace ss {

namespace {

struct CacheArgs {
    Table tab;
    char* plane[2];                 // keys, values
    u64 unit_bytes[2];
    u64 token_bytes, head_bytes, scale_off;
    char* rows[2];                  // 16-bit rows: read by a write, written by a read
    u64 row_stride, head_stride;    // bytes
    const unsigned* row_off;
    const unsigned* agents;
    const unsigned* lens;
    unsigned n_rows, n_requests;
    unsigned n_heads, dim;
    unsigned shift;                 // page_tokens = 1 << shift
    unsigned rows_per_block;        // 1, 2, 4, 8 or 16
};

constexpr int kCacheThreads = 256;

// Where row t of the batch lies: its unit and token in the page, unit -1 if away
// and -2 if no request has the row.  16 lanes search the requests together.
__device__ inline int place_of(const CacheArgs& A, unsigned t, unsigned sub, unsigned* slot) {
    unsigned lo = 0, n = A.n_requests;
    const unsigned base = __lane_id() & ~15u;
    while (n > 1) {                             // n is the same in the 16 lanes
        const unsigned step = (n + 15) / 16;
        const unsigned at = sub * step;
        const bool p = at < n && A.row_off[lo + (at < n ? at : 0)] <= t;
        const unsigned m = (unsigned)(__ballot(p) >> base) & 0xffffu;
        const unsigned c = m ? 31u - (unsigned)__builtin_clz(m) : 0u;
        lo += c * step;
        n = n - c * step < step ? n - c * step : step;
    }
    const unsigned b = A.row_off[lo], rows = request_rows(A.row_off, lo, A.n_rows);
    if (t >= A.n_rows || t < b || t - b >= rows) return -2;
    const long long token = (long long)A.lens[lo] - rows + (t - b);
    if (token < 0) return -1;
    u64 first;
    const unsigned pages = A.tab.row(A.agents[lo], &first);
    const u64 page = (u64)token >> A.shift;
    *slot = (unsigned)token & ((1u << A.shift) - 1u);
    return page < pages ? A.tab.unit(first + page) : -1;
}

// The largest of a value over kLanes lanes next to each other (8, 16 or 32).
template <int kLanes>
__device__ __forceinline__ float lanes_max(float x) {
#pragma unroll
    for (int m = kLanes / 2; m; m >>= 1) x = fmaxf(x, __shfl_xor(x, m));
    return x;
}

// Eight codes of a row that kLanes lanes hold, and the row's scale.
template <class T, int kLanes>
__device__ __forceinline__ u32x2 quantise(u32x4 w, float* scale) {
    float x[8], top = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        x[2 * j] = T::lo(w[j]);
        x[2 * j + 1] = T::hi(w[j]);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(x[j]));      // not of a NaN
    top = lanes_max<kLanes>(top);
    if (__any(top == INFINITY)) {                                   // not of an infinity either
        float finite = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float y = fabsf(x[j]);
            finite = y < INFINITY && y > finite ? y : finite;
        }
        top = lanes_max<kLanes>(finite);
    }
    const float s = fmaxf(top / 448.f, 0x1p-126f);
    *scale = s;
    // x / s, rounded as a division: the product with 1 / s is at most a unit in the last
    // place off, and its exact rest tells which way (where no rest is denormal)
    const float inv = 1.f / s;
    float q[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float p = x[j] * inv;
        q[j] = fmaf(fmaf(-p, s, x[j]), inv, p);
    }
    bool odd = s < 0x1p-90f;
#pragma unroll
    for (int j = 0; j < 8; ++j) odd |= !(fabsf(x[j]) < INFINITY);
    if (__any(odd)) {                       // tiny scales, infinities (which saturate), NaN
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float p = x[j] / s;
            q[j] = p > 448.f ? 448.f : p < -448.f ? -448.f : p;
        }
    }
    int lo = 0, hi = 0;
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(q[4], q[5], hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(q[6], q[7], hi, true);
    return u32x2{(unsigned)lo, (unsigned)hi};
}

// One workgroup moves rows_per_block rows of keys and values.  kWrite: rows to
// pages.  kLanes lanes hold a head's row, 8 values each (dim <= 8 kLanes).  Such a
// group keeps to one head of the keys or values and goes through the rows, several of
// them in flight (reads of 32,768 tokens: two 48 us, four 59 us; writes of 17,600: four
// 29 us, two 30 us, one 35 us); what depends on the row alone is worked out once, in LDS, as the
// address arithmetic and the division by the scale bounded the write of e4m3 (17,600
// tokens of 8 heads of 128: 263 instructions per four head rows, 43 us).
template <class T, bool kE4m3, bool kWrite, int kLanes>
__global__ __launch_bounds__(kCacheThreads) void k_cache(CacheArgs A) {
    constexpr unsigned kAtOnce = kWrite ? 4 : 2, kGroups = kCacheThreads / kLanes;
    __shared__ u64 s_cell[2][16];               // byte offset of the row's token in its plane
    __shared__ u64 s_scale[2][16];
    __shared__ int s_state[16];                 // -2: no row, -1: away, 0: has a unit
    const unsigned row0 = workgroup() * A.rows_per_block;   // below 2^31 + 2^27
    {
        const unsigned i = threadIdx.x / 16, sub = threadIdx.x % 16;
        unsigned slot = 0;
        int u = -2;
        if (i < A.rows_per_block) u = place_of(A, row0 + i, sub, &slot);
        if (sub < 2) {
            const u64 unit = (u64)(u < 0 ? 0 : u) * A.unit_bytes[sub];
            s_cell[sub][i] = unit + (u64)slot * A.token_bytes;
            s_scale[sub][i] = unit + A.scale_off + 4 * slot;
            s_state[i] = u < 0 ? u : 0;
        }
    }
    __syncthreads();
    const unsigned per_row = 2 * A.n_heads;                 // head rows of keys and values
    // groups side by side on a row's heads, then on rows
    const unsigned wide = per_row < kGroups ? per_row : kGroups, deep = kGroups / wide;
    const unsigned group = threadIdx.x / kLanes, first = group % wide, down = group / wide;
    const unsigned d0 = (threadIdx.x % kLanes) * 8;
    const bool in = d0 < A.dim;
    if (down >= deep) return;
    for (unsigned wh = first; wh < per_row; wh += wide) {
        const unsigned what = wh >= A.n_heads, h = wh - (what ? A.n_heads : 0);
        char* const rows = A.rows[what] + (u64)row0 * A.row_stride + (u64)h * A.head_stride + d0 * 2;
        char* const cells = A.plane[what] + (u64)h * A.head_bytes + d0 * (kE4m3 ? 1 : 2);
        char* const scales = A.plane[what] + (((u64)h * 4) << A.shift);
        for (unsigned i0 = down; i0 < A.rows_per_block; i0 += deep * kAtOnce) {
            u32x4 w[kAtOnce];
            float scale[kAtOnce];
            int state[kAtOnce];
#pragma unroll
            for (unsigned a = 0; a < kAtOnce; ++a) {
                const unsigned i = i0 + a * deep;
                state[a] = i < A.rows_per_block ? s_state[i] : -2;
                w[a] = u32x4{0, 0, 0, 0};
                if (state[a] < 0 || !in) continue;
                if constexpr (kWrite) {
                    w[a] = *reinterpret_cast<const u32x4*>(rows + i * A.row_stride);
                } else if constexpr (!kE4m3) {
                    w[a] = *reinterpret_cast<const u32x4*>(cells + s_cell[what][i]);
                } else {
                    const u32x2 c = *reinterpret_cast<const u32x2*>(cells + s_cell[what][i]);
                    w[a] = u32x4{c[0], c[1], 0, 0};
                    scale[a] = *reinterpret_cast<const float*>(scales + s_scale[what][i]);
                }
            }
#pragma unroll
            for (unsigned a = 0; a < kAtOnce; ++a) {
                const unsigned i = i0 + a * deep;
                if (state[a] < (kWrite ? 0 : -1)) continue;
                if constexpr (!kE4m3) {
                    if (!in) continue;
                    if constexpr (kWrite) *reinterpret_cast<u32x4*>(cells + s_cell[what][i]) = w[a];
                    else store_past(w[a], rows + i * A.row_stride);
                } else if constexpr (kWrite) {
                    float s;
                    const u32x2 codes = quantise<T, kLanes>(w[a], &s);
                    if (in) *reinterpret_cast<u32x2*>(cells + s_cell[what][i]) = codes;
                    if (d0 == 0) *reinterpret_cast<float*>(scales + s_scale[what][i]) = s;
                } else {
                    u32x4 y = {0, 0, 0, 0};
                    if (state[a] >= 0) {
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const auto p = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[a][j], false);
                            const auto q = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[a][j], true);
                            y[2 * j] = T::pack(p[0] * scale[a], p[1] * scale[a]);
                            y[2 * j + 1] = T::pack(q[0] * scale[a], q[1] * scale[a]);
                        }
                    }
                    if (in) store_past(y, rows + i * A.row_stride);
                }
            }
        }
    }
}

template <class T, bool kE4m3, bool kWrite>
void cache_launch(const CacheArgs& A, hipStream_t st) {
    const dim3 grid = grid_of((A.n_rows + A.rows_per_block - 1) / A.rows_per_block), block(kCacheThreads);
    if (A.dim <= 64) hipLaunchKernelGGL((k_cache<T, kE4m3, kWrite, 8>), grid, block, 0, st, A);
    else if (A.dim <= 128) hipLaunchKernelGGL((k_cache<T, kE4m3, kWrite, 16>), grid, block, 0, st, A);
    else hipLaunchKernelGGL((k_cache<T, kE4m3, kWrite, 32>), grid, block, 0, st, A);
}

template <bool kWrite>
ss_status cache_call(const ss_kv_cache* c, const ss_batch* b, const void* k, const void* v,
                     uint32_t type, u64 row_stride, u64 head_stride, void* stream) {
    ss_status s = cache_args(c, type);
    if (s == SS_OK) s = batch_args(b, true, false);
    if (s != SS_OK) return s;
    if (b->n_rows == 0 || b->n_requests == 0) return SS_OK;
    for (const auto& x : {std::make_pair("k", k), std::make_pair("v", v)}) {
        s = rows_args(x.first, x.second, b->n_rows, c->n_heads, c->head_dim, row_stride, head_stride,
                      !kWrite);
        if (s != SS_OK) return s;
    }
    DeviceMemory mem;
    if ((s = mem.current()) != SS_OK || (s = cache_memory(c, mem)) != SS_OK ||
        (s = batch_memory(b, true, false, mem)) != SS_OK)
        return s;
    const u64 bytes = rows_bytes(b->n_rows, c->n_heads, c->head_dim, row_stride, head_stride);
    if (!mem.has(k, bytes)) return device_error("k", mem.dev);
    if (!mem.has(v, bytes)) return device_error("v", mem.dev);
    CacheArgs A{};
    A.tab = table_of(c->units, c->agent_off, c->n_agents, c->n_entries, c->capacity_units);
    A.plane[0] = static_cast<char*>(c->k);
    A.plane[1] = static_cast<char*>(c->v);
    A.unit_bytes[0] = c->k_unit_bytes;
    A.unit_bytes[1] = c->v_unit_bytes;
    A.token_bytes = c->token_bytes;
    A.head_bytes = c->head_bytes;
    A.scale_off = c->scale_off;
    A.rows[0] = static_cast<char*>(const_cast<void*>(k));
    A.rows[1] = static_cast<char*>(const_cast<void*>(v));
    A.row_stride = 2 * row_stride;
    A.head_stride = 2 * head_stride;
    A.row_off = b->row_off;
    A.agents = b->agents;
    A.lens = b->lens;
    A.n_rows = b->n_rows;
    A.n_requests = b->n_requests;
    A.n_heads = c->n_heads;
    A.dim = c->head_dim;
    A.shift = (unsigned)__builtin_ctz(c->page_tokens);
    // the search for the rows' requests costs a block as much for one row as for
    // 16, so blocks take more rows once there are 1,024 blocks
    A.rows_per_block = 1;
    while (A.rows_per_block < 16 && b->n_rows / (2 * A.rows_per_block) >= 1024) A.rows_per_block *= 2;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const bool q = c->type == SS_E4M3;
    if (type == SS_BF16) {
        if (q) cache_launch<Bf16, true, kWrite>(A, st);
        else cache_launch<Bf16, false, kWrite>(A, st);
    } else {
        if (q) cache_launch<F16, true, kWrite>(A, st);
        else cache_launch<F16, false, kWrite>(A, st);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return set_err(SS_ERR_HIP, "%s kernel: %s", kWrite ? "kv write" : "kv read",
                       hipGetErrorString(e));
    return SS_OK;
}

bool aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// a + b * c where every term is nonnegative, or UINT64_MAX beyond 2^62.
u64 madd(u64 a, u64 b, u64 c) {
    const __uint128_t x = (__uint128_t)b * c + a;
    return x > ((__uint128_t)1 << 62) ? UINT64_MAX : (u64)x;
}

// Bytes of a page's codes or values, behind k + unit * k_unit_bytes.
u64 page_bytes(const ss_kv_cache* c) {
    const u64 row = (u64)c->head_dim * (c->type == SS_E4M3 ? 1 : 2);
    return madd(madd(row, c->page_tokens - 1, c->token_bytes), c->n_heads - 1, c->head_bytes);
}
u64 unit_span(const ss_kv_cache* c) {
    const u64 body = page_bytes(c);
    if (c->type != SS_E4M3) return body;
    return std::max(body, madd(c->scale_off, 4ull * c->n_heads, c->page_tokens));
}

}  // namespace

ss_status device_error(const char* name, int dev) {
    return set_err(SS_ERR_ARG, "%s must be device memory of the current device (%d), large enough",
                   name, dev);
}

ss_status table_args(const int32_t* units, const uint64_t* agent_off, uint32_t n_agents,
                     uint64_t n_entries, uint64_t capacity_units) {
    if (!units || !agent_off) return set_err(SS_ERR_ARG, "NULL block table");
    if (n_agents < 1 || n_entries < 1 || n_entries >= (1ull << 40))
        return set_err(SS_ERR_ARG, "n_agents and n_entries must be >= 1");
    if (capacity_units < 1 || capacity_units >= (1ull << 31))
        return set_err(SS_ERR_ARG, "capacity_units must be in [1, 2^31)");
    return SS_OK;
}

ss_status cache_args(const ss_kv_cache* c, uint32_t row_type) {
    if (!c) return set_err(SS_ERR_ARG, "cache is NULL");
    ss_status s = table_args(c->units, c->agent_off, c->n_agents, c->n_entries, c->capacity_units);
    if (s != SS_OK) return s;
    if (!c->k || !c->v || !aligned(c->k) || !aligned(c->v))
        return set_err(SS_ERR_ARG, "cache k and v must be 16-byte aligned pointers");
    if (c->page_tokens < 1 || c->page_tokens > 1024 || (c->page_tokens & (c->page_tokens - 1)))
        return set_err(SS_ERR_ARG, "page_tokens must be a power of two in [1, 1024]");
    if (c->n_heads < 1 || c->n_heads > 1024)
        return set_err(SS_ERR_ARG, "n_heads must be in [1, 1024]");
    if (c->head_dim < 16 || c->head_dim > 256 || c->head_dim % 16)
        return set_err(SS_ERR_ARG, "head_dim must be a multiple of 16 in [16, 256]");
    if (c->type != SS_BF16 && c->type != SS_F16 && c->type != SS_E4M3)
        return set_err(SS_ERR_ARG, "unknown cache type %u", c->type);
    if (row_type != SS_BF16 && row_type != SS_F16)
        return set_err(SS_ERR_ARG, "rows must be SS_BF16 or SS_F16, not type %u", row_type);
    if (c->type != SS_E4M3 && c->type != row_type)
        return set_err(SS_ERR_ARG, "rows of type %u with a cache of type %u", row_type, c->type);
    for (u64 x : {c->k_unit_bytes, c->v_unit_bytes, c->token_bytes, c->head_bytes, c->scale_off})
        if (x % 16) return set_err(SS_ERR_ARG, "cache byte distances must be multiples of 16");
    // tokens within heads or heads within tokens, rows apart from each other
    const u64 row = (u64)c->head_dim * (c->type == SS_E4M3 ? 1 : 2);
    const bool by_head = (c->page_tokens == 1 || c->token_bytes >= row) &&
        (c->n_heads == 1 || c->head_bytes >= madd(row, c->page_tokens - 1, c->token_bytes));
    const bool by_token = (c->n_heads == 1 || c->head_bytes >= row) &&
        (c->page_tokens == 1 || c->token_bytes >= madd(row, c->n_heads - 1, c->head_bytes));
    if (!by_head && !by_token) return set_err(SS_ERR_ARG, "a page's rows overlap");
    if (c->type == SS_E4M3 && c->scale_off < page_bytes(c))
        return set_err(SS_ERR_ARG, "scale_off lies inside the page's codes");
    const u64 span = unit_span(c);
    if (span >= (1ull << 31)) return set_err(SS_ERR_ARG, "a page is too large (2^31 bytes)");
    if (c->capacity_units > 1 && (c->k_unit_bytes < span || c->v_unit_bytes < span))
        return set_err(SS_ERR_ARG, "a page of %llu bytes does not fit into a unit's chunk",
                       (unsigned long long)span);
    if (madd(span, c->capacity_units - 1, std::max(c->k_unit_bytes, c->v_unit_bytes)) == UINT64_MAX)
        return set_err(SS_ERR_ARG, "cache sizes are too large");
    return SS_OK;
}

ss_status batch_args(const ss_batch* b, bool lens, bool groups) {
    if (!b) return set_err(SS_ERR_ARG, "batch is NULL");
    if (b->n_rows >= (1u << 31)) return set_err(SS_ERR_ARG, "n_rows must be below 2^31");
    if (b->n_requests >= (1u << 20)) return set_err(SS_ERR_ARG, "n_requests must be below 2^20");
    if (groups && b->n_groups >= (1u << 20))
        return set_err(SS_ERR_ARG, "n_groups must be below 2^20");
    if (b->n_rows == 0 || b->n_requests == 0) return SS_OK;
    if (!b->row_off || !b->agents || (lens && !b->lens))
        return set_err(SS_ERR_ARG, "NULL array in the batch");
    if (groups && b->n_groups && (!b->group_off || !b->prefix_agents || !b->prefix_lens))
        return set_err(SS_ERR_ARG, "NULL array of the batch's groups");
    return SS_OK;
}

ss_status rows_args(const char* name, const void* ptr, u64 n_rows, u64 n_heads, u64 dim,
                    u64 row_stride, u64 head_stride, bool written) {
    if (!ptr || !aligned(ptr)) return set_err(SS_ERR_ARG, "%s must be a 16-byte aligned pointer", name);
    if (row_stride % 8 || head_stride % 8)
        return set_err(SS_ERR_ARG, "strides of %s must be multiples of 8 elements", name);
    if (row_stride >= (1ull << 40) || head_stride >= (1ull << 40))
        return set_err(SS_ERR_ARG, "strides of %s are too large", name);
    // written rows do not overlap: heads within rows or rows within heads
    if (written && !((n_heads == 1 || head_stride >= dim) &&
                     (n_rows == 1 || row_stride >= madd(dim, n_heads - 1, head_stride))) &&
        !((n_rows == 1 || row_stride >= dim) &&
          (n_heads == 1 || head_stride >= madd(dim, n_rows - 1, row_stride))))
        return set_err(SS_ERR_ARG, "rows of %s overlap", name);
    if (rows_bytes(n_rows, n_heads, dim, row_stride, head_stride) >= (1ull << 62))
        return set_err(SS_ERR_ARG, "%s is too large", name);
    return SS_OK;
}

u64 rows_bytes(u64 n_rows, u64 n_heads, u64 dim, u64 row_stride, u64 head_stride) {
    const u64 n = madd(madd(dim, n_rows - 1, row_stride), n_heads - 1, head_stride);
    return n > (1ull << 61) ? UINT64_MAX : 2 * n;
}

ss_status DeviceMemory::current() {
    if (hipGetDevice(&dev) != hipSuccess) {
        (void)hipGetLastError();
        return set_err(SS_ERR_ARG, "no current device");
    }
    return SS_OK;
}

bool DeviceMemory::has(const void* ptr, u64 bytes) {
    const uintptr_t p = reinterpret_cast<uintptr_t>(ptr);
    for (int i = 0; i < n_known_; ++i)
        if (p >= known_[i].base && p <= known_[i].end && bytes <= known_[i].end - p) return true;
    if (!device_range_ok(ptr, bytes, dev)) return false;
    hipDeviceptr_t base = nullptr;
    size_t size = 0;
    if (hipMemGetAddressRange(&base, &size, const_cast<void*>(ptr)) != hipSuccess) {
        (void)hipGetLastError();                // managed memory, say
    } else if (n_known_ < 4) {
        known_[n_known_++] = {reinterpret_cast<uintptr_t>(base), reinterpret_cast<uintptr_t>(base) + size};
    }
    return true;
}

ss_status table_memory(const int32_t* units, const uint64_t* agent_off, uint32_t n_agents,
                       uint64_t n_entries, DeviceMemory& mem) {
    if (!mem.has(units, n_entries * 4)) return device_error("units", mem.dev);
    if (!mem.has(agent_off, ((u64)n_agents + 1) * 8))
        return device_error("agent_off", mem.dev);
    return SS_OK;
}

ss_status cache_memory(const ss_kv_cache* c, DeviceMemory& mem) {
    const ss_status s = table_memory(c->units, c->agent_off, c->n_agents, c->n_entries, mem);
    if (s != SS_OK) return s;
    const u64 span = unit_span(c);
    if (!mem.has(c->k, madd(span, c->capacity_units - 1, c->k_unit_bytes)))
        return device_error("cache k", mem.dev);
    if (!mem.has(c->v, madd(span, c->capacity_units - 1, c->v_unit_bytes)))
        return device_error("cache v", mem.dev);
    return SS_OK;
}

ss_status batch_memory(const ss_batch* b, bool lens, bool groups, DeviceMemory& mem) {
    if (!mem.has(b->row_off, ((u64)b->n_requests + 1) * 4))
        return device_error("row_off", mem.dev);
    if (!mem.has(b->agents, (u64)b->n_requests * 4)) return device_error("agents", mem.dev);
    if (lens && !mem.has(b->lens, (u64)b->n_requests * 4))
        return device_error("lens", mem.dev);
    if (!groups || b->n_groups == 0) return SS_OK;
    if (!mem.has(b->group_off, ((u64)b->n_groups + 1) * 4))
        return device_error("group_off", mem.dev);
    if (!mem.has(b->prefix_agents, (u64)b->n_groups * 4))
        return device_error("prefix_agents", mem.dev);
    if (!mem.has(b->prefix_lens, (u64)b->n_groups * 4))
        return device_error("prefix_lens", mem.dev);
    return SS_OK;
}

}  // namespace ss

using namespace ss;

extern "C" {

ss_status ss_kv_write(const ss_kv_cache* cache, const ss_batch* batch, const void* k,
                      const void* v, uint32_t type, uint64_t row_stride, uint64_t head_stride,
                      void* stream) {
    return cache_call<true>(cache, batch, k, v, type, row_stride, head_stride, stream);
}

ss_status ss_kv_read(const ss_kv_cache* cache, const ss_batch* batch, void* k, void* v,
                     uint32_t type, uint64_t row_stride, uint64_t head_stride, void* stream) {
    return cache_call<false>(cache, batch, k, v, type, row_stride, head_stride, stream);
}

}  // extern "C"
