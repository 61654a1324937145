// Device helpers of the key-value cache kernels (gfx950, wave64).
#pragma once

#include <algorithm>
#include <climits>

#include "bdl_device.h"
#include "bdl_kv.h"

namespace bdl {

// two fp32 numbers as bf16, to nearest even (NaN stays)
__device__ __forceinline__ uint32_t pk_bf16(float x, float y) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, y}, bf16x2));
}

// into the range of e4m3 (NaN stays)
__device__ __forceinline__ float clamp_e4m3(float f) { return f != f ? f : fminf(fmaxf(f, -448.f), 448.f); }

__device__ __forceinline__ void kv_error(const KvCache& c) {
    __hip_atomic_store(c.err, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// the entry (index i of sequence row b, kv head h) as an index into the
// pages' entries; -1 (and the error flag) where the table names no page
__device__ __forceinline__ long long kv_entry(const KvCache& c, int b, int h, int i) {
    const int p = c.table[(long long)b * c.tstride + (i >> c.ps_shift)];
    if ((unsigned)p >= (unsigned)c.n_pages) {
        kv_error(c);
        return -1;
    }
    return (((long long)p * c.hkv + h) << c.ps_shift) + (i & ((1 << c.ps_shift) - 1));
}

// length of row b, limited to what its table row can name
__device__ __forceinline__ int kv_len(const KvCache& c, const int* lens, int b) {
    const int n = lens[b];
    const long long most = (long long)c.width << c.ps_shift;
    if (n < 0 || n > most) kv_error(c);
    return n < 0 ? 0 : (int)min((long long)n, most);
}

}  // namespace bdl
