// Key-value cache of decoder serving: append and eviction (gfx950, wave64).
#include "bdl_kv_device.h"

namespace bdl {

// ------------------------------------------------------------------ append
// One thread per pair of a q or k row, or per two elements of a v row.
// Rotation: y1 = x1 c - x2 s, y2 = x2 c + x1 s in fp32, every product and sum
// rounded by itself (no fused multiply-add), so that the result is that of
// the two lines as written.
template <bool FP8>
__device__ __forceinline__ void kv_put(char* base, long long entry, int D, int d, float x, float inv) {
    if (FP8)
        reinterpret_cast<uint8_t*>(base)[entry * D + d] = (uint8_t)f2e4m3(x * inv);
    else
        reinterpret_cast<uint16_t*>(base)[entry * D + d] = f2bf(x);
}

template <int D, bool FP8>
__global__ void kv_append_kernel(const KvAppendArgs a) {
#pragma clang fp contract(off)
    const int t = blockIdx.x, H = a.c.hq + 2 * a.c.hkv;
    const int seq = a.seqs[t], i = a.index[t], pos = a.positions[t];
    const bool pad = seq == -1, pos_ok = pos >= 0 && pos < a.n_positions;
    const bool at_ok = seq >= 0 && seq < a.n_seqs && i >= 0 && (long long)i < ((long long)a.c.width << a.c.ps_shift);
    if (threadIdx.x == 0 && (!pos_ok || (!pad && !at_ok))) kv_error(a.c);
    for (int u = threadIdx.x; u < H * (D / 2); u += blockDim.x) {
        const int h = u / (D / 2), j = u % (D / 2);
        const bool v = h >= a.c.hq + a.c.hkv;
        const int d0 = v || a.interleaved ? 2 * j : j, d1 = v || a.interleaved ? 2 * j + 1 : j + D / 2;
        const uint16_t* x = a.qkv + t * a.qkv_stride + h * D;
        float y0 = bf2f(x[d0]), y1 = bf2f(x[d1]);
        if (!v) {
            const float c = pos_ok ? a.cos[(long long)pos * (D / 2) + j] : 0.f, s = pos_ok ? a.sin[(long long)pos * (D / 2) + j] : 0.f;
            const float z0 = y0 * c - y1 * s, z1 = y1 * c + y0 * s;
            y0 = pos_ok ? z0 : 0.f;
            y1 = pos_ok ? z1 : 0.f;
        }
        if (h < a.c.hq) {
            uint16_t* q = a.q_out + t * a.q_stride + h * D;
            q[d0] = f2bf(y0);
            q[d1] = f2bf(y1);
        } else if (at_ok && pos_ok) {
            const int kh = (h - a.c.hq) % a.c.hkv;
            const long long e = kv_entry(a.c, seq, kh, i);
            if (e < 0) continue;
            kv_put<FP8>(v ? a.c.V : a.c.K, e, D, d0, y0, v ? a.v_inv : a.k_inv);
            kv_put<FP8>(v ? a.c.V : a.c.K, e, D, d1, y1, v ? a.v_inv : a.k_inv);
            if (v && j == 0 && a.c.weight) {
                a.c.weight[e] = 0.f;
                a.c.pos[e] = pos;
            }
        }
    }
    if (threadIdx.x == 0 && a.lens && at_ok && pos_ok && kv_entry(a.c, seq, 0, i) >= 0) atomicMax(a.lens + seq, i + 1);
}

hipError_t launch_kv_append(const KvAppendArgs& a, int head_dim, bool fp8, hipStream_t s) {
    if (head_dim == 64)
        fp8 ? kv_append_kernel<64, true><<<a.T, 256, 0, s>>>(a) : kv_append_kernel<64, false><<<a.T, 256, 0, s>>>(a);
    else
        fp8 ? kv_append_kernel<128, true><<<a.T, 256, 0, s>>>(a) : kv_append_kernel<128, false><<<a.T, 256, 0, s>>>(a);
    return hipGetLastError();
}

// ------------------------------------------------------------------ evict
// An entry's rank key: the protected ones above all, then the weights in
// their order, a NaN below all.
__device__ __forceinline__ unsigned kv_key(float w, bool prot) {
    const unsigned u = __float_as_uint(w);
    if (prot) return 0xffffffffu;
    if (w != w) return 0u;
    if (w == 0.f) return 0x80000000u;      // either zero
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ int block_sum(int v, int* red) {
    v = wave_total(wave_incl_scan(v));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return red[0] + red[1] + red[2] + red[3];
}

// Selection: one workgroup per (sequence, kv head).  The budget's smallest
// kept key is found bit by bit; then the entries are passed once in order.
__global__ void kv_select_kernel(const KvEvictArgs a) {
    __shared__ int red[4];
    const int b = blockIdx.x, h = blockIdx.y, n = kv_len(a.c, a.lens, b), M = a.budget;
    if (n <= M) {
        if (threadIdx.x == 0) a.moves[b * a.c.hkv + h] = 0;
        return;
    }
    int last = (int)0x80000000;
    for (int i = threadIdx.x; i < n; i += 256) {
        const long long e = kv_entry(a.c, b, h, i);
        if (e >= 0) last = max(last, a.c.pos[e]);
    }
    for (int k = 32; k; k >>= 1) last = max(last, __shfl_xor(last, k));
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = last;
    __syncthreads();
    last = max(max(red[0], red[1]), max(red[2], red[3]));
    auto key = [&](int i) {
        const long long e = kv_entry(a.c, b, h, i);
        return e < 0 ? 0u : kv_key(a.c.weight[e], (long long)a.c.pos[e] > (long long)last - a.recent);
    };
    // the largest t with at least M keys >= t
    unsigned t = 0;
    for (int bit = 31; bit >= 0; --bit) {
        int v = 0;
        for (int i = threadIdx.x; i < n; i += 256) v += key(i) >= (t | 1u << bit);
        if (block_sum(v, red) >= M) t |= 1u << bit;
    }
    int v = 0;
    for (int i = threadIdx.x; i < n; i += 256) v += key(i) > t;
    const int ties = M - block_sum(v, red);       // of the entries with key t, so many stay
    int eq0 = 0, free0 = 0, move0 = 0;
    for (int i0 = 0; i0 < n; i0 += 256) {
        const int i = i0 + threadIdx.x;
        const unsigned k = i < n ? key(i) : 0u;
        auto scan = [&](int x, int& base) {       // exclusive prefix over the workgroup, continued
            const int incl = wave_incl_scan(x);
            __syncthreads();
            if ((threadIdx.x & 63) == 63) red[threadIdx.x >> 6] = incl;
            __syncthreads();
            int at = base + incl - x;
            for (int q = 0; q < 4; ++q) {
                if (q < (int)(threadIdx.x >> 6)) at += red[q];
                base += red[q];
            }
            return at;
        };
        const int eq = i < n && k == t, r = scan(eq, eq0);
        const bool kept = i < n && (k > t || (eq && r < ties));
        const int fr = i < M && !kept, mv = i >= M && kept;
        const int fk = scan(fr, free0), mk = scan(mv, move0);
        if (fr || mv) {
            const long long e = kv_entry(a.c, b, h, fr ? fk : M + mk);
            if (e >= 0) a.scratch[e] = i;
        }
    }
    if (threadIdx.x == 0) a.moves[b * a.c.hkv + h] = free0;
}

template <int ROW>
__global__ void kv_move_kernel(const KvEvictArgs a) {
    const int b = blockIdx.x, h = blockIdx.y, n = a.moves[b * a.c.hkv + h], l = threadIdx.x & 63;
    for (int k = blockIdx.z * 4 + wave_id(); k < n; k += gridDim.z * 4) {
        const long long ef = kv_entry(a.c, b, h, k), em = kv_entry(a.c, b, h, a.budget + k);
        if (ef < 0 || em < 0) continue;
        const long long to = kv_entry(a.c, b, h, a.scratch[ef]), from = kv_entry(a.c, b, h, a.scratch[em]);
        if (to < 0 || from < 0) continue;
        for (int x = l * 4; x < ROW; x += 256) {
            *reinterpret_cast<uint32_t*>(a.c.K + to * ROW + x) = *reinterpret_cast<const uint32_t*>(a.c.K + from * ROW + x);
            *reinterpret_cast<uint32_t*>(a.c.V + to * ROW + x) = *reinterpret_cast<const uint32_t*>(a.c.V + from * ROW + x);
        }
        if (l == 0) {
            a.c.weight[to] = a.c.weight[from];
            a.c.pos[to] = a.c.pos[from];
        }
    }
    if (h == 0 && blockIdx.z == 0 && threadIdx.x == 0) a.lens[b] = min(kv_len(a.c, a.lens, b), a.budget);
}

hipError_t launch_kv_evict(const KvEvictArgs& a, int head_dim, bool fp8, hipStream_t s) {
    kv_select_kernel<<<dim3(a.B, a.c.hkv), 256, 0, s>>>(a);
    const dim3 grid(a.B, a.c.hkv, 16);
    switch (head_dim * (fp8 ? 1 : 2)) {
    case 64: kv_move_kernel<64><<<grid, 256, 0, s>>>(a); break;
    case 128: kv_move_kernel<128><<<grid, 256, 0, s>>>(a); break;
    default: kv_move_kernel<256><<<grid, 256, 0, s>>>(a); break;
    }
    return hipGetLastError();
}

}  // namespace bdl
