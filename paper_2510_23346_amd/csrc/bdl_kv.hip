// Key-value cache of decoder serving: append and eviction (gfx950, wave64).
#include <type_traits>

#include "bdl_kv_device.h"

namespace bdl {

namespace {

// ------------------------------------------------------------------ append
// Rotation: y1 = x1 c - x2 s, y2 = x2 c + x1 s in fp32, every product and sum
// rounded by itself (no fused multiply-add), so that the result is that of
// the two lines as written.
//
// Bound by its memory traffic, a decode step's by one trip to the token's row and
// its page number and one back.  A thread takes 16 numbers of one head of one
// token, those whose pairs it needs: two 16-byte loads, two 16-byte stores (8
// bytes each into an 8-bit cache).  A workgroup's threads are units x tokens
// (x, y), so that no index needs a division by the number of heads.
// Measured: 64 tokens of 4 + 1 + 1 heads of 128 4.1 us, of which an empty
// kernel takes 3.0; 4288 tokens of 8 + 1 + 1 heads into an 8-bit cache 8.5 us,
// 21 MB read and written.
__device__ __forceinline__ uint2 pack8_e4m3(const float (&x)[8], float inv) {
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        float c[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) c[k] = clamp_e4m3(x[4 * i + k] * inv);
        int r = __builtin_amdgcn_cvt_pk_fp8_f32(c[0], c[1], 0, false);
        w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c[2], c[3], r, true);
    }
    return uint2{w[0], w[1]};
}

// With norms (NORM) a query or key is first taken times 1 / sqrt(mean x^2 + eps)
// and its weight, in fp32 and not rounded before the rotation.  The threads of a
// head (4 or 8 neighbours in a wave) add their squares by exchanges, in an
// order that depends on nothing.  64 tokens of 4 + 1 + 1 heads of 128: 4.1 to 4.6 us,
// as without.
template <int D, bool FP8, bool NORM>
__device__ __forceinline__ void append(const KvAppendArgs& a) {
#pragma clang fp contract(off)
    const int t = blockIdx.x * blockDim.y + threadIdx.y, u = blockIdx.y * blockDim.x + threadIdx.x;
    const int H = a.c.hq + 2 * a.c.hkv, h = u / (D / 16), j = u % (D / 16);
    if (t >= a.T || h >= H) return;
    const bool v = h >= a.c.hq + a.c.hkv, pairs = v || a.interleaved;
    const int d0 = pairs ? 16 * j : 8 * j, d1 = pairs ? 16 * j + 8 : D / 2 + 8 * j;
    const uint16_t* x = a.qkv + t * a.qkv_stride + h * D;
    const u32x4 x0 = ld16(x + d0), x1 = ld16(x + d1);
    const int seq = a.seqs[t], i = a.index[t], pos = a.positions[t];
    const int cap = a.c.width << a.c.ps_shift;
    const bool pos_ok = pos >= 0 && pos < a.n_positions, at_ok = seq >= 0 && seq < a.n_seqs && i >= 0 && i < cap;
    float y0[8], y1[8];
    unpack8(x0, y0);
    unpack8(x1, y1);
    if (NORM && !v) {
        const uint16_t* const w = h < a.c.hq ? a.q_norm : a.k_norm;
        const u32x4 w0 = ld16(w + d0), w1 = ld16(w + d1);
        head_norm<D>(y0, y1, w0, w1, a.eps);
    }
    if (!v) {
        rotate16(y0, y1, a.cos, a.sin, (long long)(pos_ok ? pos : 0) * (D / 2) + 8 * j, a.interleaved);
        if (!pos_ok)
#pragma unroll
            for (int k = 0; k < 8; ++k) y0[k] = y1[k] = 0.f;
    }
    if (h < a.c.hq) {
        uint16_t* q = a.q_out + t * a.q_stride + h * D;
        *reinterpret_cast<u32x4*>(q + d0) = pack8(y0);
        *reinterpret_cast<u32x4*>(q + d1) = pack8(y1);
        if (u == 0) {
            if (!pos_ok || (seq != -1 && !at_ok)) kv_error(a.c);
            if (a.lens && at_ok && pos_ok && kv_entry(a.c, seq, 0, i) >= 0) {
                // (a prompt's tokens would all raise one number: only the last
                // of a run does)
                bool covered = false;
                if (t + 1 < a.T && a.seqs[t + 1] == seq) {
                    const int i1 = a.index[t + 1], p1 = a.positions[t + 1];
                    covered = i1 > i && i1 < cap && p1 >= 0 && p1 < a.n_positions && kv_entry(a.c, seq, 0, i1) >= 0;
                }
                if (!covered) atomicMax(a.lens + seq, i + 1);
            }
        }
        return;
    }
    if (!at_ok || !pos_ok) return;
    const int kh = h - a.c.hq - (v ? a.c.hkv : 0);
    const long long e = kv_entry(a.c, seq, kh, i);
    if (e < 0) return;
    char* const base = (v ? a.c.V : a.c.K) + e * (D * (FP8 ? 1 : 2));
    if constexpr (FP8) {
        const float inv = v ? a.v_inv : a.k_inv;
        *reinterpret_cast<uint2*>(base + d0) = pack8_e4m3(y0, inv);
        *reinterpret_cast<uint2*>(base + d1) = pack8_e4m3(y1, inv);
    } else {
        *reinterpret_cast<u32x4*>(base + 2 * d0) = v ? x0 : pack8(y0);
        *reinterpret_cast<u32x4*>(base + 2 * d1) = v ? x1 : pack8(y1);
    }
    if (v && j == 0 && a.c.weight) {
        a.c.weight[e] = 0.f;
        a.c.pos[e] = pos;
    }
}

template <int D, bool FP8>
__global__ __launch_bounds__(256) void kv_append_kernel(const KvAppendArgs a) {
    append<D, FP8, false>(a);
}

template <int D, bool FP8>
__global__ __launch_bounds__(256) void kv_append_norm_kernel(const KvAppendArgs a) {
    append<D, FP8, true>(a);
}

template <int D, bool FP8>
hipError_t append(const KvAppendArgs& a, hipStream_t s) {
    const int units = (a.c.hq + 2 * a.c.hkv) * (D / 16), x = std::min(units, 256), y = 256 / x;
    const dim3 grid((a.T + y - 1) / y, (units + x - 1) / x), block(x, y);
    if (a.q_norm)
        kv_append_norm_kernel<D, FP8><<<grid, block, 0, s>>>(a);
    else
        kv_append_kernel<D, FP8><<<grid, block, 0, s>>>(a);
    return hipGetLastError();
}

// ------------------------------------------------------------------ evict
// One launch.  The workgroups (sequence, kv head, z) of one sequence and head
// all select the entries that stay (it reads 8 bytes an entry, what an
// exchange between them would cost more than), and each moves its share of the
// keys and values.  Weights and positions, which the selection reads, are moved
// by the workgroup that is the last of its head to have selected; the length is
// set by the last of its sequence.
//
// Selection: the rank key of the last entry that stays, found in up to three
// passes over the keys (11, 11 and 10 bits; histograms in LDS), then places and
// sources by prefix sums.  A thread owns consecutive entries.  Their keys are
// kept in registers (up to 24576 entries of a sequence), or the first 8192 there
// and 28672 more in LDS, and what is left is read again in each pass.
//
// Measured: 64 sequences from 2049 to 2048 entries 9.7 us, of which 2 are the
// way to lengths, pages and weights, 1.1 to 1.5 each pass, 1.3 the places and 1
// the one row that moves: a chain of waits, 64 workgroups, and all of it the
// general selection, though one entry is looked for.  8 sequences of two
// kv heads from 8192 to 2048 18.2 us, 10 of them the same chain over four
// times the entries and 5 the 25 MB that move.
// One of 16384 to 4096 23 us, of 32768 43, of 65536 92; of 131072 to 8192 237,
// most of it the keys read again in each pass, a thread's at a time.
constexpr int kET = 1024, kEW = kET / 64;
constexpr int kFewGroups = 2, kRegGroups = 6, kLdsGroups = 7;      // groups of four entries a thread keeps
constexpr int kFewEntries = 4 * kFewGroups * kET, kRegEntries = 4 * kRegGroups * kET;
constexpr int kListCap = 4096;          // moves whose lists fit LDS; more go through a.scratch

// An entry's rank key: the protected ones above all, then the weights in
// their order, a NaN below all.  (0: the entry's page is none; it ranks below
// every entry that is there)
__device__ __forceinline__ unsigned kv_key(float w, bool prot) {
    const unsigned u = __float_as_uint(w);
    if (prot) return 0xffffffffu;
    if (w != w) return 1u;
    if (w == 0.f) return 0x80000000u;      // either zero
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

struct EvictLds {
    unsigned hist[2048];
    int freed[kListCap], moved[kListCap];
    int wave[2][kEW];
    unsigned digit, need, same;
    int last, lost;         // largest position; entries below the budget whose page is none
    int holes;              // whether there are such pages at all
};

// exclusive prefix sum over the workgroup; total in *total
__device__ __forceinline__ int block_scan(int v, int* total, int* waves) {
    const int incl = wave_incl_scan(v), l = threadIdx.x & 63;
    if (l == 63) waves[threadIdx.x >> 6] = incl;
    __syncthreads();
    const int s = wave_incl_scan(l < kEW ? waves[l] : 0), w = wave_id();
    *total = __builtin_amdgcn_readlane(s, kEW - 1);
    return incl - v + (w ? __builtin_amdgcn_readlane(s, w - 1) : 0);
}

// Entries 4 g .. 4 g + 3 of a sequence (they lie in one page): their first
// place among the entries of all pages, or -1
__device__ __forceinline__ long long four_at(const KvCache& c, int b, int h, int g) {
    return kv_entry(c, b, h, 4 * g);
}

// Pages of a sequence of n entries, and a thread's share of them
__device__ __forceinline__ int pages_of(const KvCache& c, int n) { return (n + (1 << c.ps_shift) - 1) >> c.ps_shift; }
__device__ __forceinline__ int page_share(const KvCache& c, int n) { return (pages_of(c, n) + kET - 1) / kET; }
__device__ __forceinline__ bool page_there(const KvCache& c, int b, int page) {
    return (unsigned)c.table[(long long)b * c.tstride + page] < (unsigned)c.n_pages;
}

// The lists of moves (the places, then the sources: 2 moves in all) that LDS
// does not hold lie in a.scratch, element x in the place of the sequence's x-th
// entry.  Where page numbers are none, these are passed over (at least 2 moves
// entries are there): L.freed then has how many pages are there before each
// thread's share
__device__ __forceinline__ long long list_past_holes(const KvCache& c, int b, int h, int n, int x, const EvictLds& L) {
    int t = 0, left = x >> c.ps_shift;
#pragma unroll 1
    for (int step = kET / 2; step; step /= 2)
        if (L.freed[t + step] <= left) t += step;
    left -= L.freed[t];
    const int share = page_share(c, n), end = min(pages_of(c, n), (t + 1) * share);
    int page = t * share;
#pragma unroll 1
    for (; page < end; ++page)
        if (page_there(c, b, page) && left-- == 0) break;
    return page < end ? kv_entry(c, b, h, (page << c.ps_shift) + (x & ((1 << c.ps_shift) - 1))) : -1;
}

// R groups of a thread in registers; with MORE the next ones in LDS, and what
// is left is read again each time.  Returns how many entries move; -1 where the
// row names pages that are none, which only the form with HOLES can deal with
// (one form for both costs every call 0.3 to 0.7 us)
template <int R, bool MORE, bool HOLES>
__device__ __forceinline__ int kv_select(const KvEvictArgs& a, int b, int h, int n, EvictLds& L, uint4* keys) {
    constexpr int U = 4;                // groups whose loads are in flight at once, behind the first R
    const int tid = threadIdx.x, M = a.budget, groups = (n + 3) / 4;
    const int per = (groups + kET - 1) / kET, g0 = tid * per;
    int mine = min(n - 4 * g0, 4 * per);        // the thread's entries (none: less than one)
    // (false: there is no such group, or its page is none)
    auto get = [&](int k, float4& ww, int4& pp) __attribute__((always_inline)) {
        ww = float4{NAN, NAN, NAN, NAN};
        pp = int4{INT_MIN, INT_MIN, INT_MIN, INT_MIN};
        if (k >= per || g0 + k >= groups) return false;
        const long long e = four_at(a.c, b, h, g0 + k);
        if (e < 0) return false;
        ww = *reinterpret_cast<const float4*>(a.c.weight + e);
        pp = *reinterpret_cast<const int4*>(a.c.pos + e);
        return true;
    };
    // the largest position
    float4 w[R];
    int4 p[R];
    bool there[R];
    int last = INT_MIN, lost = 0;
    bool hole = false;
    auto top = [&](int k, const int4& pp, bool ok) __attribute__((always_inline)) {
        const int i = 4 * k;
        if (!ok && i < mine) {
            hole = true;
            lost += max(0, min(4, min(mine, M - 4 * g0) - i));
        }
        if (i < mine) last = max(last, pp.x);
        if (i + 1 < mine) last = max(last, pp.y);
        if (i + 2 < mine) last = max(last, pp.z);
        if (i + 3 < mine) last = max(last, pp.w);
    };
    // f(k, weights, positions, whether they are there) for the groups from `from` on
    auto read = [&](int from, auto f) __attribute__((always_inline)) {
#pragma unroll 1
        for (int k0 = from; k0 < per; k0 += U) {
            float4 ww[U];
            int4 pp[U];
            bool ok[U];
#pragma unroll
            for (int u = 0; u < U; ++u) ok[u] = get(k0 + u, ww[u], pp[u]);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (k0 + u < per) f(k0 + u, ww[u], pp[u], ok[u]);
        }
    };
    for (int i = tid; i < 2048; i += kET) L.hist[i] = 0;
    if (tid == 0) {
        L.last = INT_MIN;
        L.lost = L.holes = 0;
    }
#pragma unroll
    for (int k = 0; k < R; ++k) there[k] = get(k, w[k], p[k]);
#pragma unroll
    for (int k = 0; k < R; ++k) top(k, p[k], there[k]);
    if constexpr (MORE)
        read(R, [&](int k, const float4&, const int4& pp, bool ok) __attribute__((always_inline)) { top(k, pp, ok); });
#pragma unroll
    for (int x = 32; x; x >>= 1) last = max(last, __shfl_xor(last, x));
    __syncthreads();
    if ((tid & 63) == 0) atomicMax(&L.last, last);
    if (HOLES && lost) atomicAdd(&L.lost, lost);
    if (hole) L.holes = 1;
    __syncthreads();
    if (!HOLES && L.holes) return -1;
    // as many stay as there are places for below the budget: no fewer entries
    // are there, since those from the budget on are n - M or fewer
    const int room = HOLES ? M - L.lost : M;
    if (HOLES && room == 0) return 0;
    const long long floor_ = (long long)L.last - a.recent;
    auto key4 = [&](const float4& ww, const int4& pp, bool ok) __attribute__((always_inline)) {
        if (HOLES && !ok) return uint4{0, 0, 0, 0};
        return uint4{kv_key(ww.x, pp.x > floor_), kv_key(ww.y, pp.y > floor_), kv_key(ww.z, pp.z > floor_), kv_key(ww.w, pp.w > floor_)};
    };
    uint4 key[R];
#pragma unroll
    for (int k = 0; k < R; ++k) key[k] = key4(w[k], p[k], there[k]);
    constexpr int kKept = R + kLdsGroups;
    if constexpr (MORE)
#pragma unroll
        for (int k0 = R; k0 < kKept; k0 += U) {
            float4 ww[U];
            int4 pp[U];
            bool ok[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (k0 + u < kKept) ok[u] = get(k0 + u, ww[u], pp[u]);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (k0 + u < kKept) keys[(k0 + u - R) * kET + tid] = key4(ww[u], pp[u], ok[u]);
        }
    // f(entry, key) for the thread's entries in order
    auto each = [&](auto f) __attribute__((always_inline)) {
        const int i0 = 4 * g0;
        // (the comparisons stay where they are: their results, kept over the
        // passes, would be more masks than there are scalar registers)
        if constexpr (R > kFewGroups || MORE) asm volatile("" : "+v"(mine));
        auto four = [&](int k, const uint4& key) __attribute__((always_inline)) {
            if (4 * k < mine) f(i0 + 4 * k, key.x);
            if (4 * k + 1 < mine) f(i0 + 4 * k + 1, key.y);
            if (4 * k + 2 < mine) f(i0 + 4 * k + 2, key.z);
            if (4 * k + 3 < mine) f(i0 + 4 * k + 3, key.w);
        };
#pragma unroll
        for (int k = 0; k < R; ++k)
            if (k < per) four(k, key[k]);
        if constexpr (MORE) {
#pragma unroll 1
            for (int k = R; k < min(per, kKept); ++k) four(k, keys[(k - R) * kET + tid]);
            read(kKept, [&](int k, const float4& ww, const int4& pp, bool ok) __attribute__((always_inline)) { four(k, key4(ww, pp, ok)); });
        }
    };
    // the room-th largest key (never that of an entry that is not there), 11, 11
    // and 10 bits at a time
    unsigned known = 0, need = room;    // its leading bits; how many of the keys with these bits stay
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, above = pass == 0 ? 32 : pass == 1 ? 21 : 10;
        const unsigned mask = pass == 2 ? 1023u : 2047u;
        each([&](int, unsigned k) __attribute__((always_inline)) {
            if (pass && (k >> above) != known) return;
            const unsigned dgt = (k >> shift) & mask;
            // (where a wave's keys agree, one lane counts them)
            const unsigned first = (unsigned)__builtin_amdgcn_readfirstlane((int)dgt);
            const unsigned long long act = __ballot(1), same = __ballot(dgt == first);
            if (same == act) {
                if ((int)(threadIdx.x & 63) == __ffsll((long long)act) - 1) atomicAdd(&L.hist[first], (unsigned)__popcll(act));
            } else {
                atomicAdd(&L.hist[dgt], 1u);
            }
        });
        __syncthreads();
        // bins from the top: thread t has 2047 - 2 t and 2046 - 2 t
        const unsigned c0 = L.hist[2047 - 2 * tid], c1 = L.hist[2046 - 2 * tid];
        int total;
        const unsigned before = (unsigned)block_scan((int)(c0 + c1), &total, L.wave[0]);
        if (before < need && need <= before + c0) {
            L.digit = 2047 - 2 * tid;
            L.need = need - before;
            L.same = c0;
        } else if (before + c0 < need && need <= before + c0 + c1) {
            L.digit = 2046 - 2 * tid;
            L.need = need - before - c0;
            L.same = c1;
        }
        L.hist[2047 - 2 * tid] = 0;
        L.hist[2046 - 2 * tid] = 0;
        __syncthreads();
        known = pass == 2 ? known << 10 | L.digit : known << 11 | L.digit;
        need = L.need;
        // (where all keys with these bits stay, the rest of the bits decides
        // nothing: weights that differ mostly spare the third pass, 1.1 us)
        if (need == L.same) {
            known <<= shift;
            break;
        }
    }
    // of the entries with that key the first `need` stay (where that is not
    // all of them, a thread has to know how many come before its own)
    const bool all_same = need == L.same;
    int eq0 = 0, total;
    if (!all_same) {
        int eq = 0;
        each([&](int, unsigned k) __attribute__((always_inline)) { eq += k == known; });
        eq0 = block_scan(eq, &total, L.wave[0]);
    }
    int eq = all_same ? INT_MIN / 2 : eq0, fr = 0, mv = 0;
    each([&](int i, unsigned k) __attribute__((always_inline)) {
        const bool kept = k > known || (k == known && eq++ < (int)need);
        fr += i < M && !kept && (!HOLES || k);
        mv += i >= M && kept;
    });
    // (both counts in one scan where they fit 16 bits)
    int moves;
    if (n < 1 << 16) {
        const int s = block_scan(fr | mv << 16, &moves, L.wave[1]);
        fr = s & 0xffff;
        mv = s >> 16 & 0xffff;
        moves &= 0xffff;
    } else {
        fr = block_scan(fr, &moves, L.wave[1]);
        __syncthreads();
        mv = block_scan(mv, &total, L.wave[0]);
    }
    eq = all_same ? INT_MIN / 2 : eq0;
    // (half of the entries at most)
    const bool in_lds = (!MORE && 2 * R * kET <= kListCap) || moves <= kListCap;
    auto put = [&](int i, unsigned k, auto place) __attribute__((always_inline)) {
        const bool kept = k > known || (k == known && eq++ < (int)need);
        const bool f = i < M && !kept && (!HOLES || k), m = i >= M && kept;
        if (!f && !m) return;
        const int at = f ? fr++ : mv++;
        if (in_lds) {
            (f ? L.freed : L.moved)[at] = i;
        } else {
            const long long e = place(f ? at : moves + at);
            if (e >= 0) a.scratch[e] = i;
        }
    };
    if (!HOLES || in_lds) {
        each([&](int i, unsigned k) __attribute__((always_inline)) { put(i, k, [&](int x) { return kv_entry(a.c, b, h, x); }); });
        return moves;
    }
    // (an entry at a time from memory: nothing but a wrong page table comes here)
    const int share = page_share(a.c, n), p0 = tid * share, p1 = min(pages_of(a.c, n), p0 + share);
    int pages = 0;
#pragma unroll 1
    for (int j = p0; j < p1; ++j) pages += page_there(a.c, b, j);
    __syncthreads();
    L.freed[tid] = block_scan(pages, &total, L.wave[0]);
    __syncthreads();
#pragma unroll 1
    for (int i = 4 * g0; i < 4 * g0 + mine; ++i) {
        const long long e = kv_entry(a.c, b, h, i);
        put(i, e < 0 ? 0u : kv_key(a.c.weight[e], a.c.pos[e] > floor_), [&](int x) { return list_past_holes(a.c, b, h, n, x, L); });
    }
    return moves;
}

// LONG: rows of the page table that can name more than kFewEntries
template <int ROW, bool LONG>
__global__ __launch_bounds__(kET) void kv_evict_kernel(const KvEvictArgs a) {
    __shared__ EvictLds L;
    __shared__ uint4 keys[LONG ? kLdsGroups * kET : 1];
    __shared__ bool last_head;
    const int b = blockIdx.x, h = blockIdx.y, z = blockIdx.z, Z = gridDim.z, M = a.budget;
    const int raw = a.lens[b], n = kv_len(a.c, a.lens, b);
    if (n <= M) {
        // (a length that is none becomes one; reading it before or after is the same)
        if (h == 0 && z == 0 && threadIdx.x == 0 && raw != n) a.lens[b] = n;
        return;
    }
    int moves;
    if (!LONG || n <= kFewEntries)
        moves = kv_select<kFewGroups, false, false>(a, b, h, n, L, keys);
    else if (n <= kRegEntries)
        moves = kv_select<kRegGroups, false, false>(a, b, h, n, L, keys);
    else
        moves = kv_select<kFewGroups, true, false>(a, b, h, n, L, keys);
    if (moves < 0) {
        __syncthreads();
        moves = kv_select<kFewGroups, LONG, true>(a, b, h, n, L, keys);
    }
    // this workgroup has read what it needs of weights, positions and lengths
    __syncthreads();
    const bool alone = Z == 1;              // of its head
    if (threadIdx.x == 0) {
        unsigned* const ch = a.count + ((size_t)b * a.c.hkv + h) * kKvCount;
        unsigned* const cs = a.count + ((size_t)gridDim.x * a.c.hkv + b) * kKvCount;
        const unsigned nh = Z, ns = Z * a.c.hkv;
        // (both counted at once)
        const unsigned at_h = nh > 1 ? __hip_atomic_fetch_add(ch, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0u;
        const unsigned at_s = ns > 1 ? __hip_atomic_fetch_add(cs, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0u;
        last_head = !alone && at_h == nh - 1;
        if (last_head) __hip_atomic_store(ch, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (at_s == ns - 1) {
            if (ns > 1) __hip_atomic_store(cs, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            a.lens[b] = M;
        }
    }
    const bool in_lds = !LONG || moves <= kListCap;
    // place and source of move k, as entries of all pages; false where a page is
    // none.  (past_holes: a list in memory of a row that names such pages)
    auto move = [&](auto past_holes, int k, long long& to, long long& from) __attribute__((always_inline)) {
        int i, j;
        if (!past_holes.value && in_lds) {
            i = L.freed[k];
            j = L.moved[k];
        } else {
            auto at = [&](int x) __attribute__((always_inline)) {
                return past_holes.value ? list_past_holes(a.c, b, h, n, x, L) : kv_entry(a.c, b, h, x);
            };
            const long long ef = at(k), em = at(moves + k);
            if (ef < 0 || em < 0) return false;
            i = a.scratch[ef];
            j = a.scratch[em];
        }
        to = kv_entry(a.c, b, h, i);
        from = kv_entry(a.c, b, h, j);
        return to >= 0 && from >= 0;
    };
    // keys and values: LPR lanes a row, four moves in flight (and weights and
    // positions, where no other workgroup is still to read them)
    constexpr int LPR = ROW / 16, RPP = kET / LPR;
    const int k1 = (int)((long long)moves * (z + 1) / Z), c = threadIdx.x % LPR * 16;
    auto rows = [&](auto past_holes) __attribute__((always_inline)) {
        constexpr int U = decltype(past_holes)::value ? 1 : 4;
        for (int k0 = (int)((long long)moves * z / Z) + threadIdx.x / LPR; k0 < k1; k0 += U * RPP) {
            long long to[U], from[U];
            bool ok[U];
            u32x4 x[U], y[U];
            float w[U];
            int p[U];
#pragma unroll
            for (int u = 0; u < U; ++u) ok[u] = k0 + u * RPP < k1 && move(past_holes, k0 + u * RPP, to[u], from[u]);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (ok[u]) {
                    x[u] = *reinterpret_cast<const u32x4*>(a.c.K + from[u] * ROW + c);
                    y[u] = *reinterpret_cast<const u32x4*>(a.c.V + from[u] * ROW + c);
                    if (alone && c == 0) {
                        w[u] = a.c.weight[from[u]];
                        p[u] = a.c.pos[from[u]];
                    }
                }
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (ok[u]) {
                    *reinterpret_cast<u32x4*>(a.c.K + to[u] * ROW + c) = x[u];
                    *reinterpret_cast<u32x4*>(a.c.V + to[u] * ROW + c) = y[u];
                    if (alone && c == 0) {
                        a.c.weight[to[u]] = w[u];
                        a.c.pos[to[u]] = p[u];
                    }
                }
        }
    };
    const bool holes = !in_lds && L.holes;
    if (holes)
        rows(std::true_type{});
    else
        rows(std::false_type{});
    if (alone) return;
    __syncthreads();
    auto weights = [&](auto past_holes) __attribute__((always_inline)) {
        for (int k = threadIdx.x; k < moves; k += kET) {
            long long to, from;
            if (!move(past_holes, k, to, from)) continue;
            a.c.weight[to] = a.c.weight[from];
            a.c.pos[to] = a.c.pos[from];
        }
    };
    if (!last_head) return;
    if (holes)
        weights(std::true_type{});
    else
        weights(std::false_type{});
}

}  // namespace

hipError_t launch_kv_append(const KvAppendArgs& a, int head_dim, bool fp8, hipStream_t s) {
    if (a.c.scales) return launch_kv_store(a, head_dim, s);
    if (head_dim == 64) return fp8 ? append<64, true>(a, s) : append<64, false>(a, s);
    return fp8 ? append<128, true>(a, s) : append<128, false>(a, s);
}

namespace {

template <int ROW>
void evict(const KvEvictArgs& a, const dim3& grid, bool many, hipStream_t s) {
    if (many)
        kv_evict_kernel<ROW, true><<<grid, kET, 0, s>>>(a);
    else
        kv_evict_kernel<ROW, false><<<grid, kET, 0, s>>>(a);
}

}  // namespace

hipError_t launch_kv_evict(const KvEvictArgs& a, int head_dim, bool fp8, hipStream_t s) {
    // a workgroup per compute unit, and no more of a head than the moves could
    // feed that a row of this width allows.  (Up to 256 moves: one; the counting
    // that several need costs what they save, 11.1 against 12.4 us at 236 moves,
    // and 15.1 against 15.7 at 1024.  Lengths are not known here: where rows are
    // wider than their sequences, few moves get several workgroups all the same:
    // 64 sequences from 2049 to 2048 take 11.9 us in rows of 2064 entries, 13.1 to
    // 13.4 in rows of 8192 to 131072)
    const long long heads = (long long)a.B * a.c.hkv, cap = (long long)a.c.width << a.c.ps_shift;
    const long long most = std::min<long long>(a.budget, std::max(0LL, cap - a.budget));
    const int z = most <= 256 ? 1 : (int)std::max(1LL, std::min({a.n_cu / heads, (most + 63) / 64, 64LL}));
    const dim3 grid(a.B, a.c.hkv, z);
    const bool many = cap > kFewEntries;
    switch (head_dim * (fp8 ? 1 : 2)) {
    case 64: evict<64>(a, grid, many, s); break;
    case 128: evict<128>(a, grid, many, s); break;
    default: evict<256>(a, grid, many, s); break;
    }
    return hipGetLastError();
}

}  // namespace bdl
