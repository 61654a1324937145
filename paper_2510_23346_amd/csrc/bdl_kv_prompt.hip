// Attention of many new tokens of each sequence over the paged cache (gfx950,
// wave64): prompts, chunks of them, drafted tokens.
//
//     s_pj = scale <q_p, k_j>,  out_p = sum_j exp(s_pj - m) v_j / sum_j exp(s_pj - m)
//
// over the entries j that the token of entry p sees (j <= p; with a window the
// last so many of them, and the first few).  One pass over the entries with a
// running maximum m.
//
// The rows of a kv head are (token, query head), heads of one token side by
// side, so that a tile of 128 rows reads an entry's key and value once for all
// its heads.  A workgroup has a tile: four waves of 32 rows, which share tiles
// of 64 entries in LDS, two of them in turn (one is worked on while the next
// one's loads are in flight).
//
// A wave's products are S^T = K Q^T and O^T = V^T P^T (32x32x16, bf16): a row's
// scores lie in one lane (and the one 32 further), so that maximum and sum need
// no exchange, and they are already those of the second product's operand.
#include "bdl_kv_device.h"

namespace bdl {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int NW = 4, NT = NW * 64;     // waves and threads of a workgroup, of which a compute unit holds two
constexpr int kRows = NW * 32;          // rows of a tile
constexpr int kKeys = 64;               // entries of a tile

__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// A sequence's rows of q (of a kv head: `rows`, n tokens' G each) and length
struct Prompt {
    int t0, n, len;
    unsigned tiles;
    bool bad;
};

__device__ __forceinline__ Prompt prompt_of(const KvPromptArgs& a, int b, int G) {
    const int at = min(max(b, 0), a.B - 1), cap = a.c.width << a.c.ps_shift;
    const int u0 = a.q_starts[at], u1 = a.q_starts[at + 1], n = a.lens[at];
    Prompt p;
    p.t0 = min(max(u0, 0), a.T);
    const int t1 = min(max(u1, p.t0), a.T);
    p.n = t1 - p.t0;
    p.len = min(max(n, 0), cap);
    p.bad = p.t0 != u0 || t1 != u1 || p.len != n || p.n > p.len;
    p.tiles = b >= 0 && b < a.B ? (unsigned)(p.n * G + kRows - 1) / kRows : 0u;
    return p;
}

template <int D, int FMT>
__global__ __launch_bounds__(NT, 2) void kv_prompt_kernel(const KvPromptArgs a) {
    constexpr int SZ = FMT == kBf16 ? 2 : 1, ROW = D * SZ, CPR = ROW / 16;
    constexpr int LPT = kKeys * CPR / NT;           // 16-byte loads of a thread for a tile's keys
    constexpr int KS = D / 16, DT = D / 32;
    constexpr int BUF = kKeys * D / 8;              // 16-byte pieces of a tile's keys in LDS
    __shared__ u32x4 lds[2][2][BUF];
    const int w = wave_id(), l = threadIdx.x & 63, lr = l & 31, lh = l >> 5;
    const int hkv = a.c.hkv, G = a.c.hq / hkv, psh = a.c.ps_shift, pmask = (1 << psh) - 1;
    const int kvh = blockIdx.x % hkv;
    const unsigned item = blockIdx.x / hkv;

    // the workgroup's sequence and tile: the last sequence's last tile, which
    // sees most, comes first
    int b = -1, t0 = 0, n = 0, len = 0, r0 = 0;
    {
        unsigned base = 0;
        bool bad = false;
        for (int c0 = 0; c0 < a.B && b < 0; c0 += 64) {
            const Prompt p = prompt_of(a, a.B - 1 - c0 - l, G);
            bad |= p.bad;
            const unsigned incl = base + (unsigned)wave_incl_scan((int)p.tiles);
            const unsigned long long over = __ballot(incl > item);
            if (over) {
                const int i = __ffsll((long long)over) - 1;
                b = a.B - 1 - c0 - i;
                t0 = __builtin_amdgcn_readlane(p.t0, i);
                n = __builtin_amdgcn_readlane(p.n, i);
                len = __builtin_amdgcn_readlane(p.len, i);
                r0 = (int)((unsigned)__builtin_amdgcn_readlane((int)incl, i) - 1 - item) * kRows;
            }
            base = (unsigned)__builtin_amdgcn_readlane((int)incl, 63);
        }
        if (bad) kv_error(a.c);
        if (b < 0) return;
    }
    const int rows = min(kRows, n * G - r0), at0 = len - n;
    const int p_first = at0 + r0 / G, p_last = at0 + (r0 + rows - 1) / G;
    // entries that some row sees: 0 .. sk - 1 and k_begin .. k_end - 1
    const int k_end = max(0, p_last + 1);
    int k_begin = a.window ? min(k_end, max(0, p_first - a.window + 1)) : 0, sk = min(a.sinks, k_begin);
    if (sk == k_begin) sk = k_begin = 0;
    const int nS = (sk + kKeys - 1) / kKeys, base = k_begin & ~15;
    const int tiles = nS + (k_end > k_begin ? (k_end - base + kKeys - 1) / kKeys : 0);

    // this lane's row
    const bool busy = 32 * w < rows;                // the wave has rows
    const int wr0 = r0 + min(32 * w, rows - 1), wr1 = r0 + min(32 * w + 31, rows - 1);
    const int row = min(wr0 + lr, wr1), tok = row / G, hd = row - tok * G, p = at0 + tok;
    const int pw_first = at0 + wr0 / G, pw_last = at0 + wr1 / G;
    u32x4 q[KS];
    {
        const uint16_t* const qp = a.q + (long long)(t0 + tok) * a.q_stride + (kvh * G + hd) * D + 8 * lh;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            q[ks] = ld16(qp + 16 * ks);
#pragma unroll
            for (int i = 0; i < 4; ++i) q[ks][i] ^= a.q_sign;
        }
    }

    struct Tile {
        int e, lo, hi;        // first entry; those lo .. hi - 1 count
    };
    auto tile_at = [&](int ct) __attribute__((always_inline)) {
        const bool s = ct < nS;
        return Tile{s ? kKeys * ct : base + kKeys * (ct - nS), s ? 0 : k_begin, s ? sk : k_end};
    };
    // a thread's loads of a tile: 64 pieces of 16 bytes a wave, of one block of 16 entries
    auto block_of = [&](int i) __attribute__((always_inline)) { return (i * NT + w * 64) / CPR / 16; };
    // Pages (and an int8 cache's scales) of 16 tiles at once, a block of 16 entries
    // a lane; in `ok` those blocks that are there.  Tiles are loaded in order, the
    // next 16 looked up when the first of these is
    const int* const trow = a.c.table + (long long)b * a.c.tstride;
    int page_ = 0, page_next = 0;
    float2 scale_ = float2{1.f, 1.f}, scale_next = scale_;
    unsigned long long ok_ = 0;
    auto look = [&](int ct0) __attribute__((always_inline)) {
        const int ct = ct0 + (l >> 2);
        const Tile t = tile_at(ct);
        const int e = t.e + 16 * (l & 3);
        page_next = ct < tiles && e < t.hi ? trow[e >> psh] : -1;
    };
    auto entry_of = [&](int page, int e) __attribute__((always_inline)) {
        return (((unsigned long long)(unsigned)page * (unsigned)hkv + (unsigned)kvh) << psh) + (unsigned)(e & pmask);
    };
    auto turn = [&](int ct0) __attribute__((always_inline)) {
        page_ = page_next;
        const int ct = ct0 + (l >> 2);
        const Tile t = tile_at(ct);
        const int e = t.e + 16 * (l & 3);
        const bool in = ct < tiles && e < t.hi, there = in && (unsigned)page_ < (unsigned)a.c.n_pages;
        if (in && !there) kv_error(a.c);
        ok_ = __ballot(there);
        if constexpr (FMT == kInt8) scale_ = there ? *reinterpret_cast<const float2*>(a.c.scales + 2 * (entry_of(page_, e) >> 4)) : float2{1.f, 1.f};
        look(ct0 + 16);
    };
    u32x4 kr[LPT], vr[LPT];
    // of the tile being worked on: blocks that are there, and their scales
    unsigned there = 0, there_next = 0;
    float ks[4], vs[4], ks_next[4], vs_next[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) ks[k] = vs[k] = ks_next[k] = vs_next[k] = 1.f;
    auto load = [&](int ct) __attribute__((always_inline)) {
        if ((ct & 15) == 0) turn(ct);
        const Tile t = tile_at(ct);
        const int l0 = 4 * (ct & 15);
        there_next = (unsigned)(ok_ >> l0) & 15u;
#pragma unroll
        for (int i = 0; i < LPT; ++i) {
            const int blk = block_of(i), e = t.e + 16 * blk;
            const bool ok = there_next >> blk & 1;
            const unsigned long long ent = entry_of(ok ? __builtin_amdgcn_readlane(page_, l0 + blk) : 0, e);
            const unsigned lo = (unsigned)uni((int)(unsigned)ent), hi = (unsigned)uni((int)(unsigned)(ent >> 32));
            const unsigned long long at = ((unsigned long long)hi << 32 | lo) * ROW;
            const unsigned bytes = (unsigned)uni(ok ? min(16, t.hi - e) : 0) * ROW;
            const unsigned off = (unsigned)((((i * NT + (int)threadIdx.x) / CPR & 15) * CPR + threadIdx.x % CPR) * 16);
            kr[i] = buf16(buf_rsrc(a.c.K + at, bytes), off);
            vr[i] = buf16(buf_rsrc(a.c.V + at, bytes), off);
        }
        if constexpr (FMT == kInt8)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                ks_next[k] = __uint_as_float((unsigned)__builtin_amdgcn_readlane((int)__float_as_uint(scale_.x), l0 + k));
                vs_next[k] = __uint_as_float((unsigned)__builtin_amdgcn_readlane((int)__float_as_uint(scale_.y), l0 + k));
            }
    };
    auto next = [&]() __attribute__((always_inline)) {
        there = there_next;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            ks[k] = ks_next[k];
            vs[k] = vs_next[k];
        }
    };
    auto put = [&](int buf, int ct) __attribute__((always_inline)) {
        const Tile t = tile_at(ct);
#pragma unroll
        for (int i = 0; i < LPT; ++i) {
            const int id = i * NT + (int)threadIdx.x, r = id / CPR, c = id % CPR;
            u32x4 v = vr[i];
            // (what lies before the first entry may be NaN, and 0 times NaN is one)
            if (t.e + r < t.lo) v = u32x4{0, 0, 0, 0};
            if constexpr (FMT == kBf16) {
                lds[buf][0][k_at<D>(r, c)] = kr[i];
                lds[buf][1][v_at<D>(r, c)] = v;
            } else {
                const u32x4 k = kr[i];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    lds[buf][0][k_at<D>(r, 2 * c + x)] = FMT == kFp8 ? bf16_of(k[2 * x], k[2 * x + 1]) : bf16_of_int8(k[2 * x], k[2 * x + 1]);
                    lds[buf][1][v_at<D>(r, 2 * c + x)] = FMT == kFp8 ? bf16_of(v[2 * x], v[2 * x + 1]) : bf16_of_int8(v[2 * x], v[2 * x + 1]);
                }
            }
        }
    };
    float m = -INFINITY, sum = 0.f;
    f32x16 o[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[dt] = f32x16{};

    if (tiles > 0) {
        look(0);
        load(0);
        put(0, 0);
        next();
    }
    __syncthreads();
    for (int ct = 0; ct < tiles; ++ct) {
        const int buf = ct & 1;
        load(ct + 1);
        const Tile t = tile_at(ct);
        const bool past = t.e > pw_last;                                   // no row of the wave sees it
        const bool gone = a.window && t.e + kKeys - 1 <= pw_first - a.window && t.e >= a.sinks;
        if (busy && !past && !gone) {
            const u32x4* const kb = lds[buf][0];
            const u32x4* const vb = lds[buf][1];
            f32x16 s[2] = {f32x16{}, f32x16{}};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                s[0] = mfma32(kb[k_at<D>(lr, 2 * ks + lh)], q[ks], s[0]);
                s[1] = mfma32(kb[k_at<D>(32 + lr, 2 * ks + lh)], q[ks], s[1]);
            }
            const bool whole = t.e >= t.lo && t.e + kKeys <= t.hi && t.e + kKeys - 1 <= pw_first && there == 15u &&
                               (!a.window || t.e > pw_last - a.window || t.e + kKeys <= a.sinks);
            if (!whole) {
                const int last = min(t.hi - 1, p), first = a.window ? p - a.window + 1 : 0;
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int e = t.e + 32 * j + 8 * (i / 4) + 4 * lh + i % 4;
                        const bool sees = e <= last && e >= t.lo && (e >= first || e < a.sinks) && (there >> (2 * j + i / 8) & 1);
                        s[j][i] = sees ? s[j][i] : -INFINITY;
                    }
            }
            float scale[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) scale[k] = FMT == kInt8 ? a.score_scale * ks[k] : a.score_scale;
            float top = -INFINITY;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float x = -INFINITY;
#pragma unroll
                for (int i = 0; i < 8; ++i) x = fmaxf(x, s[k / 2][8 * (k & 1) + i]);
                top = fmaxf(top, x * scale[k]);
            }
            // the maximum follows only where a score passes it by 8 (in units of
            // log 2): until then no exponential exceeds 2^8
            if (__any(top > m + 8.f)) {
                top = fmaxf(top, __shfl_xor(top, 32));
                const float mn = fmaxf(m, top), f = m == -INFINITY ? 0.f : exp2_(m - mn);
                m = mn;
                sum *= f;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) o[dt] *= f;
            }
            const float mm = m == -INFINITY ? 0.f : m;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                u32x4 pb;
#pragma unroll
                for (int i = 0; i < 8; i += 2) {
                    float x = exp2_(fmaf(s[k / 2][8 * (k & 1) + i], scale[k], -mm)), y = exp2_(fmaf(s[k / 2][8 * (k & 1) + i + 1], scale[k], -mm));
                    sum += x + y;
                    if constexpr (FMT == kInt8) x *= vs[k], y *= vs[k];
                    pb[i / 2] = pk_bf16(x, y);
                }
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    s16x4 v[2];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int r = 16 * k + 8 * j + 4 * lh + ((l & 15) >> 2);
                        const short* const at = reinterpret_cast<const short*>(vb + v_at<D>(r, 4 * dt + 2 * ((l >> 4) & 1) + ((l >> 1) & 1))) + 4 * (l & 1);
                        v[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
                    }
                    const u32x4 va = __builtin_bit_cast(u32x4, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
                    o[dt] = mfma32(va, pb, o[dt]);
                }
            }
        }
        put(buf ^ 1, ct + 1);
        next();
        __syncthreads();
    }
    if (!busy || wr0 + lr > wr1) return;
    sum += __shfl_xor(sum, 32);
    const bool none = sum == 0.f;
    const float g = a.v_scale / sum;
    uint16_t* const out = a.out + (long long)(t0 + tok) * a.out_stride + (kvh * G + hd) * D + 4 * lh;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<uint2*>(out + 32 * dt + 8 * i) =
                uint2{none ? 0u : pk_bf16(o[dt][4 * i] * g, o[dt][4 * i + 1] * g), none ? 0u : pk_bf16(o[dt][4 * i + 2] * g, o[dt][4 * i + 3] * g)};
    if (lh == 0 && a.lse) a.lse[(long long)(t0 + tok) * a.c.hq + kvh * G + hd] = none ? -INFINITY : (m + __log2f(sum)) * kLn2;
}

template <int D>
hipError_t launch(const KvPromptArgs& a, bool fp8, hipStream_t s) {
    const long long G = a.c.hq / a.c.hkv, items = (a.T * G / kRows + std::min(a.T, a.B)) * a.c.hkv;
    if (a.c.scales)
        kv_prompt_kernel<D, kInt8><<<(int)items, NT, 0, s>>>(a);
    else if (fp8)
        kv_prompt_kernel<D, kFp8><<<(int)items, NT, 0, s>>>(a);
    else
        kv_prompt_kernel<D, kBf16><<<(int)items, NT, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_prompt(const KvPromptArgs& a, int head_dim, bool fp8, hipStream_t s) {
    return head_dim == 64 ? launch<64>(a, fp8, s) : launch<128>(a, fp8, s);
}

}  // namespace bdl
