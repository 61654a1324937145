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

__device__ __forceinline__ void unpack8(u32x4 v, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(v[i] << 16);
        x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    }
}

__device__ __forceinline__ u32x4 pack8(const float (&x)[8]) {
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pk_bf16(x[2 * i], x[2 * i + 1]);
    return v;
}

// Norm of a head of D numbers, 16 a thread (x, in pieces of 8 with their
// weights), its D / 16 threads side by side: x (1 / sqrt(mean x^2 + eps)) w, every
// step rounded by itself
template <int D>
__device__ __forceinline__ void head_norm(float (&x0)[8], float (&x1)[8], u32x4 w0, u32x4 w1, float eps) {
#pragma clang fp contract(off)
    float ss = 0.f, w[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) ss += x0[k] * x0[k] + x1[k] * x1[k];
#pragma unroll
    for (int x = 1; x < D / 16; x *= 2) ss += __shfl_xor(ss, x);
    const float r = 1.f / sqrtf(ss * (1.f / D) + eps);
    unpack8(w0, w);
#pragma unroll
    for (int k = 0; k < 8; ++k) x0[k] = x0[k] * r * w[k];
    unpack8(w1, w);
#pragma unroll
    for (int k = 0; k < 8; ++k) x1[k] = x1[k] * r * w[k];
}

// Rotation of 16 numbers of a head whose angles begin at element `at` of the
// tables: pairs (x0[k], x1[k]), or neighbours, pairs 0..3 in x0 and 4..7 in x1
__device__ __forceinline__ void rotate16(float (&x0)[8], float (&x1)[8], const float* cos, const float* sin, long long at,
                                         bool interleaved) {
#pragma clang fp contract(off)
    float c[8], s[8];
#pragma unroll
    for (int k = 0; k < 8; k += 4) {
        const float4 cc = *reinterpret_cast<const float4*>(cos + at + k), ss = *reinterpret_cast<const float4*>(sin + at + k);
        c[k] = cc.x, c[k + 1] = cc.y, c[k + 2] = cc.z, c[k + 3] = cc.w;
        s[k] = ss.x, s[k + 1] = ss.y, s[k + 2] = ss.z, s[k + 3] = ss.w;
    }
    if (interleaved) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float a0 = x0[2 * k], b0 = x0[2 * k + 1], a1 = x1[2 * k], b1 = x1[2 * k + 1];
            x0[2 * k] = a0 * c[k] - b0 * s[k];
            x0[2 * k + 1] = b0 * c[k] + a0 * s[k];
            x1[2 * k] = a1 * c[k + 4] - b1 * s[k + 4];
            x1[2 * k + 1] = b1 * c[k + 4] + a1 * s[k + 4];
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float a0 = x0[k], b0 = x1[k];
            x0[k] = a0 * c[k] - b0 * s[k];
            x1[k] = b0 * c[k] + a0 * s[k];
        }
    }
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

enum { kBf16, kFp8, kInt8 };     // a cache's format

constexpr float kLn2 = 0.6931471805599453f;
__device__ __forceinline__ int uni(int v) { return __builtin_amdgcn_readfirstlane(v); }

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// what is left of a number without its upper 16 bits
__device__ __forceinline__ float below_bf16(float x) { return x - __uint_as_float(__float_as_uint(x) & 0xffff0000u); }

// the upper 16 bits of two numbers side by side
__device__ __forceinline__ uint32_t upper_halves(float x, float y) {
    return __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);
}

// Where a 16-byte chunk c of row r of a tile lies in LDS: rows of D bf16
// numbers whose chunks are exchanged within the row so that both the 16-byte
// reads of keys (16 rows, one chunk each) and the transposing reads of values
// (8 rows, the two chunks of 16 columns) meet every bank once.
template <int D>
__device__ __forceinline__ int k_at(int r, int c) {
    return r * (D / 8) + (c ^ (D == 128 ? r & 15 : (r >> 1) & 7));
}
template <int D>
__device__ __forceinline__ int v_at(int r, int c) {
    return r * (D / 8) + (c ^ (D == 128 ? 2 * (r & 7) : 2 * ((r >> 1) & 3)));
}

// 8 numbers of an 8-bit cache as bf16 (exact)
__device__ __forceinline__ u32x4 bf16_of(uint32_t a, uint32_t b) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    u32x4 r;
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true));
    return r;
}

// 8 integers as bf16 (exact: 8 significant bits)
__device__ __forceinline__ u32x4 bf16_of_int8(uint32_t a, uint32_t b) {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = (i < 2 ? a : b) >> (16 * (i & 1));
        r[i] = upper_halves((float)(int8_t)w, (float)(int8_t)(w >> 8));
    }
    return r;
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// Shares go past the caches that the compute units do not have in common
// (device scope), 8 or 16 bytes at byte `at` of the workspace
constexpr int kDeviceScope = 16;
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ void store_through(__amdgpu_buffer_rsrc_t r, unsigned at, f32x4 v) {
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), r, (int)at, 0, kDeviceScope);
}

__device__ __forceinline__ void store_through(__amdgpu_buffer_rsrc_t r, unsigned at, float2 v) {
    __builtin_amdgcn_raw_buffer_store_b64(u32x2{__float_as_uint(v.x), __float_as_uint(v.y)}, r, (int)at, 0, kDeviceScope);
}

__device__ __forceinline__ f32x4 load_through4(__amdgpu_buffer_rsrc_t r, unsigned at) {
    return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, (int)at, 0, kDeviceScope));
}

__device__ __forceinline__ float2 load_through2(__amdgpu_buffer_rsrc_t r, unsigned at) {
    const u32x2 v = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, (int)at, 0, kDeviceScope));
    return float2{__uint_as_float(v[0]), __uint_as_float(v[1])};
}

// Shares of a row are added times the factor of their maximum to the row's.  Where that
// is 0 they are left out, since 0 times an infinity is a NaN; but a NaN among a share's
// sums, x, is one of the row's, v, whatever its probability
__device__ __forceinline__ float keep_nan(float v, float x) { return x != x ? x : v; }

typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t min_u16x2(uint32_t x, uint32_t y) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(u16x2, x), __builtin_bit_cast(u16x2, y)));
}

__device__ __forceinline__ uint32_t max_u16x2(uint32_t x, uint32_t y) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, x), __builtin_bit_cast(u16x2, y)));
}

}  // namespace bdl
