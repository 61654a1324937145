// Device helpers of the key-value cache kernels (gfx950, wave64).
#pragma once

#include "bdl_device.h"
#include "bdl_kv.h"

namespace bdl {

__device__ __forceinline__ float bf2f(uint32_t b) { return __uint_as_float(b << 16); }

// e4m3 bits, round to nearest even, clamped to the largest number (NaN stays)
__device__ __forceinline__ uint32_t f2e4m3(float f) {
    const float c = f != f ? f : fminf(fmaxf(f, -448.f), 448.f);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, c, 0, false) & 0xffu;
}

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
