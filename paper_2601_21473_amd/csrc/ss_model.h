// What the operators over resident units share (ss_cache.hip, ss_attention.hip,
// ss_adapter.hip): 16-bit and e4m3 values, the block table, the search for a
// row's request, and the host's checks.  Internal to libscalesim.
#pragma once
#include "ss_internal.h"

namespace ss {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// A 16-bit type's pairs, conversions and 16 x 16 x 32 matrix product.
struct Bf16 {
    typedef bf16x8 v8;
    static __device__ unsigned pack(float a, float b) {          // nearest even
        return __builtin_bit_cast(unsigned, bf16x2{(__bf16)a, (__bf16)b});
    }
    static __device__ float lo(unsigned w) { return __uint_as_float(w << 16); }
    static __device__ float hi(unsigned w) { return __uint_as_float(w & 0xffff0000u); }
    // two e4m3 codes (the word's lower or upper half), exactly
    template <bool kHigh>
    static __device__ unsigned from_e4m3(unsigned codes) {
        return __builtin_bit_cast(unsigned,
                                  __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, 1.0f, kHigh));
    }
    static __device__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, a),
                                                       __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
};
struct F16 {
    typedef f16x8 v8;
    static __device__ unsigned pack(float a, float b) {
        return __builtin_bit_cast(unsigned, f16x2{(_Float16)a, (_Float16)b});
    }
    static __device__ float lo(unsigned w) { return (float)__builtin_bit_cast(f16x2, w)[0]; }
    static __device__ float hi(unsigned w) { return (float)__builtin_bit_cast(f16x2, w)[1]; }
    template <bool kHigh>
    static __device__ unsigned from_e4m3(unsigned codes) {
        return __builtin_bit_cast(unsigned,
                                  __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, 1.0f, kHigh));
    }
    static __device__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, a),
                                                      __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
};

// Rows that are written once and not read again by the kernel go past the caches
// (32,768 tokens read back from e4m3: 34 us, kept in the caches 48 us).
__device__ __forceinline__ void store_past(u32x4 x, void* to) {
    __builtin_nontemporal_store(x, static_cast<u32x4*>(to));
}

// A launch's n workgroups (below 2^31), and which of them this one is.  A dimension of a grid
// ends at 2^32 threads, and workgroups behind that are left out without an error, so more
// than a row of them go into a second dimension; the last row's surplus workgroups have
// numbers from n on.
constexpr unsigned kGridRow = 1u << 23;
inline dim3 grid_of(u64 n) {
    return n <= kGridRow ? dim3((unsigned)n) : dim3(kGridRow, (unsigned)((n + kGridRow - 1) / kGridRow));
}
__device__ __forceinline__ unsigned workgroup() { return blockIdx.y * kGridRow + blockIdx.x; }

// A pool's block table: agent a's logical unit j is units[off[a] + j].
struct Table {
    const int* units;
    const u64* off;
    unsigned n_agents;
    unsigned pad;
    u64 n_entries, capacity;
    // Agent a's row: its first entry and their number (0 for no such agent).
    __device__ unsigned row(unsigned a, u64* first) const {
        *first = 0;
        if (a >= n_agents) return 0;
        const u64 b = off[a], e = off[a + 1] < n_entries ? off[a + 1] : n_entries;
        if (b >= e) return 0;
        *first = b;
        return (unsigned)(e - b < (1u << 31) ? e - b : (1u << 31));
    }
    // The unit of a table entry, -1 if it is away.
    __device__ int unit(u64 entry) const {
        const int u = units[entry];
        return u >= 0 && (u64)u < capacity ? u : -1;
    }
};

// The largest r in [0, n) with start(r) <= t (start nondecreasing, start(0) <= t,
// n >= 1), found by all 64 lanes of a wave: log64(n) reads one after the other.
template <class F>
__device__ inline unsigned wave_search(unsigned n, unsigned t, F start) {
    unsigned lo = 0;
    const unsigned lane = __lane_id();
    while (n > 1) {
        const unsigned step = (n + 63) / 64;
        const unsigned at = lane * step;
        const u64 below = __ballot(at < n && start(lo + (at < n ? at : 0)) <= t);
        const unsigned c = below ? 63u - (unsigned)__builtin_clzll(below) : 0u;
        lo += c * step;
        n = n - c * step < step ? n - c * step : step;
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

// Rows of the row arrays that request r has (0 where its offsets break the rules).
__device__ inline unsigned request_rows(const unsigned* row_off, unsigned r, unsigned n_rows) {
    const unsigned b = row_off[r], e = row_off[r + 1];
    return b < e && e <= n_rows ? e - b : 0;
}

// Host checks, defined in ss_cache.hip.
ss_status table_args(const int32_t* units, const uint64_t* agent_off, uint32_t n_agents,
                     uint64_t n_entries, uint64_t capacity_units);
ss_status cache_args(const ss_kv_cache* cache, uint32_t row_type);
ss_status batch_args(const ss_batch* batch, bool lens, bool groups);
// The current device's memory, for one call's checks: arrays in an allocation that the
// call has already asked the runtime about are not asked about again.
class DeviceMemory {
public:
    ss_status current();                        // takes the current device
    bool has(const void* ptr, u64 bytes);       // [ptr, ptr + bytes) in one allocation of it
    int dev = -1;
private:
    struct { uintptr_t base, end; } known_[4];
    int n_known_ = 0;
};
// Arrays in memory of the device: the table and the planes, the batch.
ss_status table_memory(const int32_t* units, const uint64_t* agent_off, uint32_t n_agents,
                       uint64_t n_entries, DeviceMemory& mem);
ss_status cache_memory(const ss_kv_cache* cache, DeviceMemory& mem);
ss_status batch_memory(const ss_batch* batch, bool lens, bool groups, DeviceMemory& mem);
// Rows [n_rows][n_heads][dim] of 16-bit values: strides, alignment and extent.
ss_status rows_args(const char* name, const void* ptr, u64 n_rows, u64 n_heads, u64 dim,
                    u64 row_stride, u64 head_stride, bool written);
u64 rows_bytes(u64 n_rows, u64 n_heads, u64 dim, u64 row_stride, u64 head_stride);
ss_status device_error(const char* name, int dev);
inline Table table_of(const int32_t* units, const uint64_t* off, uint32_t n_agents,
                      uint64_t n_entries, uint64_t capacity) {
    return {units, reinterpret_cast<const u64*>(off), n_agents, 0, n_entries, capacity};
}

}  // namespace ss
