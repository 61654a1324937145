// Attention of one new token per sequence over the paged cache (gfx950,
// wave64).
//
//     s_j = scale <q, k_j>,  out = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m)
//
// in one pass over the entries with a running maximum m.  An entry's key and
// value are read once for all query heads of its kv head (up to 16 of them;
// more take further workgroups), so the kernel is bound by reading the cache:
// 4 G flops per 4 bytes.
//
// Work is cut into tiles of 32 entries.  All tiles of the batch, sequence
// after sequence and head after head, form one line, of which every workgroup
// takes an equal stretch, whatever the sequences' lengths; the four waves of
// a workgroup take every fourth tile and meet in LDS.  A sequence that a
// stretch covers alone is finished there; the others' shares go to the
// workspace, and the workgroup that arrives last adds them in their order (so
// the result does not depend on which one that is).
#include "bdl_kv_device.h"

namespace bdl {

namespace {

constexpr int kNW = 4;                  // waves per workgroup
constexpr float kLn2 = 0.6931471805599453f;

// A sequence: entries first .. len - 1 in tiles that begin at a multiple of 16
// (an empty one has a tile too, which writes its row)
struct Seq {
    int len, first;
    unsigned tiles;
};

__device__ __forceinline__ Seq seq_of(const KvAttendArgs& a, int b) {
    Seq s{0, 0, 0u};
    if (b >= a.B) return s;
    s.len = kv_len(a.c, a.lens, b);
    s.first = a.starts ? max(a.starts[b], 0) : 0;
    if (s.first >= s.len) s.len = s.first = 0;
    s.tiles = max(1u, (unsigned)(s.len - (s.first & ~15) + 31) >> 5);
    return s;
}

// The line of tiles: `total` of them (heads x the sequences' tiles), cut into
// 1 << k stretches
struct Line {
    unsigned long long total;
    int k;
    __device__ __forceinline__ unsigned long long begin(unsigned w) const { return (total * w) >> k; }
    // the stretch that holds tile c
    __device__ __forceinline__ unsigned owner(unsigned long long c) const {
        unsigned w = (unsigned)min((double)((1u << k) - 1), (double)c * (double)(1u << k) / (double)total);
        while (begin(w) > c) --w;
        while (begin(w + 1) <= c) ++w;
        return w;
    }
};

__device__ __forceinline__ unsigned long long wave_sum64(unsigned long long v) {
#pragma unroll
    for (int x = 32; x; x >>= 1) v += __shfl_xor(v, x);
    return v;
}

__device__ __forceinline__ int uni(int v) { return __builtin_amdgcn_readfirstlane(v); }

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ void store_through(float* p, float x, float y) {
    __hip_atomic_store(reinterpret_cast<unsigned long long*>(p),
                       (unsigned long long)__float_as_uint(x) | ((unsigned long long)__float_as_uint(y) << 32),
                       __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ float2 load_through(const float* p) {
    const unsigned long long v =
        __hip_atomic_load(reinterpret_cast<const unsigned long long*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return float2{__uint_as_float((unsigned)v), __uint_as_float((unsigned)(v >> 32))};
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

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// A tile's two blocks of 16 entries, each within one page
struct Tile {
    size_t at[2];     // bytes from the start of K and V
    int lo[2], n[2];  // rows lo .. n - 1 of a block are attended to
    int page[2];
};

template <int D, bool FP8, bool ACC>
__global__ __launch_bounds__(kNW * 64, 2) void kv_attend_kernel(const KvAttendArgs a) {
    constexpr int SZ = FP8 ? 1 : 2, ROW = D * SZ;
    constexpr int NL = 16 * ROW / 1024;             // 16-byte loads of a block
    constexpr int KS = D / 32, DT = D / 16;
    constexpr int BUF = 32 * D / 8;                 // 16-byte pieces of a tile in LDS
    __shared__ u32x4 lds[kNW * BUF];
    __shared__ float stat[kNW][2][kKvHeads];
    __shared__ int last_flag;
    const int w = wave_id(), l = threadIdx.x & 63, lr = l & 15, lg = l >> 4;
    const int G = a.c.hq / a.c.hkv, HT = (G + kKvHeads - 1) / kKvHeads, HH = a.c.hkv * HT;
    const int psh = a.c.ps_shift, pmask = (1 << psh) - 1;

    // this workgroup's stretch and where it begins
    Line line;
    Seq mine = seq_of(a, l);
    unsigned incl = (unsigned)wave_incl_scan((int)mine.tiles);
    unsigned long long total = (unsigned)wave_total((int)incl);
    for (int b = 64 + l; b - l < a.B; b += 64) total += wave_sum64(seq_of(a, b).tiles);
    line.total = total * HH;
    const int kmax = 31 - __builtin_clz(gridDim.x);
    line.k = 0;
    while (line.k < kmax && line.total > ((unsigned long long)kNW << line.k)) ++line.k;
    if (blockIdx.x >= 1u << line.k) return;
    unsigned long long r = line.begin(blockIdx.x);
    const unsigned long long r1 = line.begin(blockIdx.x + 1);
    if (r >= r1) return;
    int b0 = 0;                                     // sequences b0 .. b0 + 63 are in the lanes
    unsigned long long base = 0;                    // tiles of a head before b0
    while ((base + (unsigned)wave_total((int)incl)) * HH <= r) {
        base += (unsigned)wave_total((int)incl);
        b0 += 64;
        mine = seq_of(a, b0 + l);
        incl = (unsigned)wave_incl_scan((int)mine.tiles);
    }
    int bi = __ffsll((long long)__ballot((base + incl) * HH > r)) - 1;
    unsigned long long seq0 = (base + (unsigned)__builtin_amdgcn_readlane((int)(incl - mine.tiles), bi)) * HH;   // its first tile
    int h;
    unsigned t0;
    {
        const unsigned tiles = (unsigned)__builtin_amdgcn_readlane((int)mine.tiles, bi);
        const unsigned long long off = r - seq0;
        unsigned q = (unsigned)((double)off / (double)tiles);
        if ((unsigned long long)q * tiles > off) --q;
        if ((unsigned long long)(q + 1) * tiles <= off) ++q;
        h = (int)q;
        t0 = (unsigned)(off - (unsigned long long)q * tiles);
    }
    u32x4* const buf = lds + w * BUF;

    for (;;) {
        const int b = b0 + bi, kvh = h / HT, ht = h - kvh * HT;
        const int len = __builtin_amdgcn_readlane(mine.len, bi), first = __builtin_amdgcn_readlane(mine.first, bi);
        const unsigned tiles = (unsigned)__builtin_amdgcn_readlane((int)mine.tiles, bi);
        const unsigned t1 = (unsigned)min((unsigned long long)tiles, t0 + (r1 - r));
        const int nh = min(kKvHeads, G - ht * kKvHeads), hq0 = kvh * G + ht * kKvHeads;
        const int e0 = first & ~15;
        typedef const __attribute__((address_space(4))) int* cint;
        const cint trow = (cint)(a.c.table + (long long)b * a.c.tstride);

        // the queries: B operand, lane = head lr, numbers 32 ks + 8 lg on
        u32x4 q[KS];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
            q[ks] = lr < nh ? ld16(a.q + b * a.q_stride + (long long)(hq0 + lr) * D + ks * 32 + lg * 8) : u32x4{0, 0, 0, 0};

        auto pages = [&](unsigned t, int (&pg)[2]) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const long long e = e0 + 32LL * t + 16 * j;
                pg[j] = trow[uni(e < len ? (int)(e >> psh) : 0)];
            }
        };
        auto tile = [&](unsigned t, const int (&pg)[2]) __attribute__((always_inline)) {
            Tile x;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const long long e = e0 + 32LL * t + 16 * j;
                bool ok = t < t1 && e < len;
                if (ok && (unsigned)pg[j] >= (unsigned)a.c.n_pages) {
                    kv_error(a.c);
                    ok = false;
                }
                x.page[j] = ok ? pg[j] : 0;
                x.n[j] = ok ? (int)min(16LL, len - e) : 0;
                x.lo[j] = (int)max(0LL, first - e);
                x.at[j] = ok ? ((((size_t)pg[j] * a.c.hkv + kvh) << psh) + (size_t)((int)e & pmask)) * ROW : 0;
            }
            return x;
        };
        u32x4 kr[2][NL], vr[2][NL];
        auto load = [&](u32x4 (&x)[2][NL], const char* base_, const Tile& tl) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const __amdgpu_buffer_rsrc_t rs = buf_rsrc(base_ + tl.at[j], (unsigned)tl.n[j] * ROW);
#pragma unroll
                for (int i = 0; i < NL; ++i) x[j][i] = buf16(rs, l * 16 + i * 1024);
            }
        };
        // rows as they were loaded (a block is contiguous) into LDS, bf16
        auto put = [&](const u32x4 (&x)[2][NL], const Tile& tl, bool value) __attribute__((always_inline)) {
            constexpr int LPR = ROW / 16;           // lanes of a row
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < NL; ++i) {
                    const int row = i * (64 / LPR) + l / LPR, c = l % LPR, rr = j * 16 + row;
                    u32x4 v = x[j][i];
                    // (a value before the first entry may be NaN, and 0 times NaN is one)
                    if (value && tl.lo[j] > 0 && row < tl.lo[j]) v = u32x4{0, 0, 0, 0};
                    if constexpr (FP8) {
                        const u32x4 y0 = bf16_of(v[0], v[1]), y1 = bf16_of(v[2], v[3]);
                        buf[value ? v_at<D>(rr, 2 * c) : k_at<D>(rr, 2 * c)] = y0;
                        buf[value ? v_at<D>(rr, 2 * c + 1) : k_at<D>(rr, 2 * c + 1)] = y1;
                    } else {
                        buf[value ? v_at<D>(rr, c) : k_at<D>(rr, c)] = v;
                    }
                }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        };

        // state of the wave: lane (head lr) has its maximum, its part of the
        // sum, and out^T: numbers 16 dt + 4 lg + i
        float m = -INFINITY, sum = 0.f;
        f32x4 o[DT];
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};

        int pg[2];
        unsigned t = t0 + w;
        pages(t, pg);
        Tile cur = tile(t, pg);
        load(kr, a.c.K, cur);
        load(vr, a.c.V, cur);
        pages(t + kNW, pg);
        for (; t < t1; t += kNW) {
            const Tile nxt = tile(t + kNW, pg);
            put(kr, cur, false);
            load(kr, a.c.K, nxt);
            pages(t + 2 * kNW, pg);
            // scores^T: lane = head lr, entries 4 lg + i of each block
            f32x4 s[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                s[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) s[j] = mfma(buf[k_at<D>(j * 16 + lr, ks * 4 + lg)], q[ks], s[j]);
            }
            float top = -INFINITY;
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int row = 4 * lg + i;
                    const float x = s[j][i] * a.score_scale;
                    s[j][i] = row >= cur.lo[j] && row < cur.n[j] ? x : -INFINITY;
                    top = fmaxf(top, s[j][i]);
                }
            if constexpr (ACC) {
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    if (lr < nh && cur.n[j] > 0) {
                        const int in_page = (int)(e0 + 32 * t + 16 * j) & pmask;
                        *reinterpret_cast<f32x4*>(a.logits + ((((size_t)cur.page[j] * a.c.hq + hq0 + lr) << psh) + in_page + 4 * lg)) = s[j];
                    }
            }
            // the maximum follows only where a score passes it by 8 (in units of
            // log 2): until then no exponential exceeds 2^8
            if (__any(top > m + 8.f)) {
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                const float mn = fmaxf(m, top), f = m == -INFINITY ? 0.f : exp2_(m - mn);
                m = mn;
                sum *= f;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) o[dt] *= f;
            }
            const float mm = m == -INFINITY ? 0.f : m;
            // exponentials as two bf16 numbers whose sum has 16 significant bits
            u32x4 hi, lo;
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < 4; i += 2) {
                    const float x = exp2_(s[j][i] - mm), y = exp2_(s[j][i + 1] - mm);
                    sum += x + y;
                    const uint32_t ux = __float_as_uint(x), uy = __float_as_uint(y);
                    hi[j * 2 + i / 2] = (ux >> 16) | (uy & 0xffff0000u);
                    const float dx = x - __uint_as_float(ux & 0xffff0000u), dy = y - __uint_as_float(uy & 0xffff0000u);
                    lo[j * 2 + i / 2] = (__float_as_uint(dx) >> 16) | (__float_as_uint(dy) & 0xffff0000u);
                }
            put(vr, cur, true);
            load(vr, a.c.V, nxt);
            // out^T += V^T P^T: the entries' order within the product is that of
            // the scores' lanes
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                s16x4 v[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int row = j * 16 + 4 * lg + (lr >> 2);
                    const short* p = reinterpret_cast<const short*>(buf + v_at<D>(row, 2 * dt + ((lr >> 1) & 1))) + 4 * (lr & 1);
                    v[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
                }
                const u32x4 va = __builtin_bit_cast(u32x4, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
                o[dt] = mfma(va, lo, mfma(va, hi, o[dt]));
            }
            cur = nxt;
        }

        // the workgroup's waves meet
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        f32x4* const ob = reinterpret_cast<f32x4*>(buf);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) ob[dt * 64 + l] = o[dt];
        if (l < kKvHeads) {
            stat[w][0][l] = m;
            stat[w][1][l] = sum;
        }
        __syncthreads();
        const int head = threadIdx.x & 15;
        float M = stat[0][0][head], f[kNW], S = 0.f;
#pragma unroll
        for (int x = 1; x < kNW; ++x) M = fmaxf(M, stat[x][0][head]);
#pragma unroll
        for (int x = 0; x < kNW; ++x) {
            f[x] = stat[x][0][head] == -INFINITY ? 0.f : exp2_(stat[x][0][head] - M);
            S += f[x] * stat[x][1][head];
        }
        auto finish = [&](int hd, int d, f32x4 v, float top, float total_) __attribute__((always_inline)) {
            const float g = total_ == 0.f ? 0.f : a.v_scale / total_;
            uint32_t p[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) p[i] = total_ == 0.f ? 0u : f2bf(v[2 * i] * g) | ((uint32_t)f2bf(v[2 * i + 1] * g) << 16);
            *reinterpret_cast<uint2*>(a.out + b * a.out_stride + (long long)(hq0 + hd) * D + d) = uint2{p[0], p[1]};
            if (d == 0) {
                const float lse2 = total_ == 0.f ? -INFINITY : top + __log2f(total_);
                const long long at = (long long)b * a.c.hq + hq0 + hd;
                if (a.lse) a.lse[at] = lse2 * kLn2;
                if (ACC) a.lse2[at] = lse2;
            }
        };
        const bool whole = t0 == 0 && t1 == tiles;
        const unsigned long long head0 = seq0 + (unsigned long long)h * tiles;      // this sequence and head's first tile
        float* const part = a.part + (size_t)(2 * blockIdx.x + (t0 == 0)) * kv_part_floats(D);
        if (head < nh) {
            for (int u = threadIdx.x; u < DT * 64; u += kNW * 64) {
                f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int x = 0; x < kNW; ++x) {
                    const f32x4 y = reinterpret_cast<const f32x4*>(lds)[x * BUF + u];
                    if (f[x] != 0.f) v += f[x] * y;
                }
                const int d = (u >> 6) * 16 + ((u >> 4) & 3) * 4;
                if (whole) {
                    finish(head, d, v, M, S);
                } else {
                    store_through(part + head * D + d, v[0], v[1]);
                    store_through(part + head * D + d + 2, v[2], v[3]);
                    if (d == 0) store_through(part + kKvHeads * D + 2 * head, M, S);
                }
            }
        }
        if (!whole) {
            const unsigned w0 = line.owner(head0), w1 = line.owner(head0 + tiles - 1);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // the share has reached memory
            __syncthreads();
            if (threadIdx.x == 0) {
                unsigned* const c = a.count + (size_t)b * HH + h;
                const unsigned old = __hip_atomic_fetch_add(c, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                last_flag = old == w1 - w0;
                if (last_flag) __hip_atomic_store(c, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            __syncthreads();
            if (last_flag) {
                // share x of sequence: the first workgroup's second place, the others' first
                const int n = (int)(w1 - w0) + 1;
                auto share = [&](int x) { return a.part + (size_t)(2 * (w0 + x) + (x == 0)) * kv_part_floats(D); };
                float* const fl = reinterpret_cast<float*>(lds);
                float mx = -INFINITY;
                if (head < nh)
                    for (int x = threadIdx.x >> 4; x < n; x += kNW * 4) mx = fmaxf(mx, load_through(share(x) + kKvHeads * D + 2 * head).x);
                fl[threadIdx.x] = mx;
                __syncthreads();
                if (threadIdx.x < kKvHeads) {
                    for (int x = 1; x < kNW * 4; ++x) mx = fmaxf(mx, fl[x * 16 + head]);
                    stat[0][0][head] = mx;
                }
                __syncthreads();
                // one item = 4 numbers of a head; groups of threads take every ng-th share
                const int items = nh * (D / 4), ng = max(1, kNW * 64 / items);
                for (int i0 = 0; i0 < items; i0 += kNW * 64) {
                    const int g = ng == 1 ? 0 : threadIdx.x / items, item = i0 + (ng == 1 ? (int)threadIdx.x : (int)threadIdx.x - g * items);
                    const bool in = item < items && g < ng;
                    const int hd = item / (D / 4), d = item % (D / 4) * 4;
                    f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f};
                    float ss = 0.f;
                    const float top = in ? stat[0][0][hd] : 0.f;
                    if (in)
#pragma unroll 4
                        for (int x = g; x < n; x += ng) {
                            const float* p = share(x);
                            const float2 ms = load_through(p + kKvHeads * D + 2 * hd);
                            const float2 y0 = load_through(p + hd * D + d), y1 = load_through(p + hd * D + d + 2);
                            const float fx = ms.x == -INFINITY ? 0.f : exp2_(ms.x - top);
                            if (fx != 0.f) {
                                ss += fx * ms.y;
                                v += fx * f32x4{y0.x, y0.y, y1.x, y1.y};
                            }
                        }
                    if (ng > 1) {
                        if (in) {
                            reinterpret_cast<f32x4*>(lds)[threadIdx.x] = v;
                            fl[kNW * 64 * 4 + threadIdx.x] = ss;
                        }
                        __syncthreads();
                        if (threadIdx.x < items)
                            for (int x = 1; x < ng; ++x) {
                                v += reinterpret_cast<f32x4*>(lds)[x * items + threadIdx.x];
                                ss += fl[kNW * 64 * 4 + x * items + threadIdx.x];
                            }
                    }
                    if (in && g == 0) finish(hd, d, v, top, ss);
                }
            }
        }
        // on to the next head or sequence
        r += t1 - t0;
        if (r >= r1) return;
        __syncthreads();
        t0 = 0;
        if (++h == HH) {
            h = 0;
            seq0 += (unsigned long long)HH * tiles;
            if (++bi == 64) {
                bi = 0;
                b0 += 64;
                mine = seq_of(a, b0 + l);
            }
        }
    }
}

// Weights: each entry's probabilities from the stored scores and the row's
// log of sums.  The entries of all sequences and kv heads, 256 at a time, form
// a line as above.
__global__ __launch_bounds__(256) void kv_weigh_kernel(const KvAttendArgs a) {
    const int l = threadIdx.x & 63, G = a.c.hq / a.c.hkv, hkv = a.c.hkv, psh = a.c.ps_shift, pmask = (1 << psh) - 1;
    auto blocks = [&](const Seq& s) { return (unsigned)(s.len - (s.first & ~15) + 255) >> 8; };
    unsigned long long at = 0;              // blocks before sequence b0, all heads
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        const Seq mine = seq_of(a, b0 + l);
        const unsigned nb = b0 + l < a.B ? blocks(mine) : 0u;
        const unsigned incl = (unsigned)wave_incl_scan((int)nb), total = (unsigned)wave_total((int)incl);
        // this workgroup's blocks: at + x with (at + x) mod gridDim = blockIdx
        const unsigned long long n = (unsigned long long)total * hkv;
        unsigned long long x = (blockIdx.x + (unsigned long long)gridDim.x - at % gridDim.x) % gridDim.x;
        for (; x < n; x += gridDim.x) {
            const int bi = __ffsll((long long)__ballot((unsigned long long)incl * hkv > x)) - 1;
            const unsigned nbb = (unsigned)__builtin_amdgcn_readlane((int)nb, bi);
            const unsigned off = (unsigned)(x - (unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(incl - nb), bi) * hkv);
            const int h = off / nbb, blk = off - h * nbb, b = b0 + bi;
            const int len = __builtin_amdgcn_readlane(mine.len, bi), first = __builtin_amdgcn_readlane(mine.first, bi);
            const long long e = (first & ~15) + 256LL * blk + threadIdx.x;
            if (e >= first && e < len) {
                const int pg = a.c.table[(long long)b * a.c.tstride + (e >> psh)];
                if ((unsigned)pg < (unsigned)a.c.n_pages) {
                    float v = 0.f;
                    for (int g = 0; g < G; ++g) {
                        const float s = a.logits[(((size_t)pg * a.c.hq + h * G + g) << psh) + ((int)e & pmask)];
                        const float z = a.lse2[(long long)b * a.c.hq + h * G + g];
                        if (z != -INFINITY) v += exp2_(s - z);
                    }
                    a.c.weight[(((size_t)pg * hkv + h) << psh) + ((int)e & pmask)] += v;
                }
            }
        }
        at += n;
    }
}

template <int D, bool FP8>
hipError_t launch(const KvAttendArgs& a, bool accumulate, hipStream_t s) {
    // no more workgroups than the table rows could have work for
    const long long G = a.c.hq / a.c.hkv, HH = a.c.hkv * ((G + kKvHeads - 1) / kKvHeads);
    const long long tiles = (((long long)a.c.width << a.c.ps_shift) + 31) / 32 * a.B * HH;
    int grid = 1;
    while (grid < kKvAttendGrid && (long long)grid * kNW < tiles) grid *= 2;
    if (!accumulate) {
        kv_attend_kernel<D, FP8, false><<<grid, kNW * 64, 0, s>>>(a);
        return hipGetLastError();
    }
    kv_attend_kernel<D, FP8, true><<<grid, kNW * 64, 0, s>>>(a);
    const long long blocks = (((long long)a.c.width << a.c.ps_shift) + 255) / 256 * a.B * a.c.hkv;
    kv_weigh_kernel<<<(int)std::min(blocks, 1024LL), 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_attend(const KvAttendArgs& a, int head_dim, bool fp8, bool accumulate, hipStream_t s) {
    if (head_dim == 64) return fp8 ? launch<64, true>(a, accumulate, s) : launch<64, false>(a, accumulate, s);
    return fp8 ? launch<128, true>(a, accumulate, s) : launch<128, false>(a, accumulate, s);
}

}  // namespace bdl
