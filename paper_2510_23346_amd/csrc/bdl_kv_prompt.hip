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
// side, so that a tile of rows reads an entry's key and value once for all its
// heads.  A wave's products are S^T = K Q^T and O^T = V^T P^T (32x32x16, bf16): a
// row's scores lie in one lane (and the one 32 further), so that maximum and sum
// need no exchange, and they are already those of the second product's operand.
// In wide tiles the probabilities are rounded to bf16 for it (their sum is not): half a
// step of 2^-8 each, which the sum of many averages out: outputs are off by 0.0022 to
// 0.0024 (root of the mean square, relative), 0.0017 of it their own rounding.  Two
// bf16 numbers for each take the second product twice: 8192 tokens 733 us in place of
// 539, 16384 with a window 373 for 274, 8 prompts of 512 17.8 for 16.4.  Narrow tiles,
// single and drafted tokens, have three for each, all 24 bits, as the call for single
// tokens has, so that a token's numbers do not depend on the call its batch takes (64
// sequences of 5 tokens over int8 26.4 us in place of 24.3).
//
// Wide tiles: a workgroup has 128 (or 64) rows, 32 a wave, whose four waves share
// tiles of 64 entries in LDS, two of them in turn: one is worked on while the next
// one's loads are in flight.  (64 rows: two waves share a tile's entries, half each.)
// Narrow tiles, of sequences of up to 32 rows: the four waves have the same rows and
// every fourth tile of 32 entries each, through their own parts of LDS, and wait for
// each other at the end only.
//
// Where there are few tiles of rows, or a long sequence among not too many short ones, a
// tile's entries are cut into stretches for several workgroups.  They leave sums, maxima
// and outputs in the workspace; the last one to come adds them, in the order of the
// entries.  Calls of 1024 workgroups and more are not cut: there a long sequence's rows
// stay with one workgroup a kv head (8 kv heads, 128 single tokens behind 2000 entries each and one
// behind 32768: 511 us, where the 2000 everywhere take 212, and 119 of them and the long
// one, which is cut, 218).
//
// Measured: one prompt of 8192 with 32 query heads of 128 on 8 kv heads 517 to 560 us
// (several cards), 0.98 to 1.06 PFLOP/s, where a large matrix product has 1.25; the
// matrix units are busy half of the time, at a clock that power holds near 2.0 GHz
// (32 cycles a product beside 5.6 vector instructions, so what one wave does not
// cover another one has to).  16384 with a window of 4096 beside 4 sinks, 8 heads on
// one 263 to 281 us.  4 prompts of 1024 beside 192 single tokens, e4m3, 36.5 us; 8 of
// 512, 4 heads on one, 16.4; 64 sequences of 5 new tokens behind 2100 entries each,
// int8, 26.4: about 8 us are the chain to the first tile (starts and lengths, pages,
// entries) and the end, and 8 more where stretches are joined.
#include <type_traits>

#include "bdl_kv_device.h"

namespace bdl {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int NW = 4, NT = NW * 64;     // waves and threads of a workgroup, of which a compute unit holds two
constexpr int kKeys = 64;               // entries of a wide tile
constexpr int kNarrow = 32;             // rows, and entries of a wave's tile, of a narrow one

// Stretches: about as many as give this many workgroups work, two a compute unit (a
// share takes a slot of the workspace for each 16 rows).  A wide tile's beginning counts
// as this many units, the end of one that is cut as kJoin
constexpr int kCutItems = 512, kCutNarrow = 384;
constexpr float kEnds = 6.f, kJoin = 8.f;

__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Where chunk c of row r of a tile's values lies in LDS: the transposing reads of
// 32 lanes (4 rows, 4 chunks) meet every bank once
template <int D>
__device__ __forceinline__ int v32_at(int r, int c) {
    return r * (D / 8) + (c ^ (D == 128 ? 4 * (r & 3) : 2 * (r & 2)));
}

// x y, but 0 where one of them is 0 whatever the other.  (The compiler's instruction and
// not one of an asm statement: x is an exponential, which needs a pause before it is
// used, and before asm statements the compiler puts none)
extern "C" __device__ float bdl_mul_legacy(float x, float y) __asm("llvm.amdgcn.fmul.legacy");

// 64 pieces of 16 bytes, the lanes' at byte offsets `off` of a buffer, into LDS at
// `to` (the wave's; lane l's lands 16 l bytes on).  Written out because the compiler
// waits for all such copies before it reads LDS at all, the other buffer's too; here
// copies_done waits, and what a wait of the compiler's own finds under way besides
// can only make it longer
__device__ __forceinline__ u32x4 rsrc_of(const char* p, unsigned bytes) {
    return u32x4{(unsigned)(uintptr_t)p, (unsigned)((uintptr_t)p >> 32), bytes, (unsigned)kRawBufferWord3};
}

__device__ __forceinline__ unsigned lds_address(const void* p) {
    return (unsigned)uni((int)(unsigned)(uintptr_t)(const __attribute__((address_space(3))) void*)p);
}

// (m0 is named as written, so that the compiler keeps nothing there across it; its
// warning is that it would not save one of its own there, which it has not)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void copy_to_lds(u32x4 rsrc, unsigned off, unsigned at) {
    // (the pause: a vector instruction may just have written the descriptor)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : : "s"(at), "v"(off), "s"(rsrc) : "m0", "memory");
}
#pragma clang diagnostic pop

__device__ __forceinline__ void copies_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

__device__ __forceinline__ unsigned lane_of(unsigned v, int i) { return (unsigned)__builtin_amdgcn_readlane((int)v, i); }

// Entries that some row of entries p_first .. p_last sees: 0 .. sinks - 1 and
// begin .. end - 1, in tiles of `size` that begin at its multiples
struct Span {
    int end, begin, sinks;
    __device__ __forceinline__ Span(const KvPromptArgs& a, int p_first, int p_last) {
        end = max(0, p_last + 1);
        begin = a.window ? min(end, max(0, p_first - a.window + 1)) : 0;
        sinks = min(a.sinks, begin);
        if (sinks == begin) sinks = begin = 0;
    }
    __device__ __forceinline__ int sink_tiles(int size) const { return (sinks + size - 1) / size; }
    __device__ __forceinline__ int tiles(int size) const {
        return sink_tiles(size) + (end > begin ? (end - (begin & -size) + size - 1) / size : 0);
    }
};

// A tile of entries: its first; those lo .. hi - 1 count
struct Tile {
    int e, lo, hi;
};

__device__ __forceinline__ Tile tile_at(const Span& s, int size, int ct) {
    const int ns = s.sink_tiles(size);
    const bool sink = ct < ns;
    return Tile{sink ? size * ct : (s.begin & -size) + size * (ct - ns), sink ? 0 : s.begin, sink ? s.sinks : s.end};
}

// A sequence: its first row of q, new tokens, length; its tiles of rows and the
// stretches' units (of 64 entries, narrow 128) of the last of them and of the first
struct Prompt {
    int t0, n, len;
    unsigned tiles, units, units0;
    bool narrow, bad;
    // what follows from n and len
    template <int ROWS>
    __device__ __forceinline__ void count(const KvPromptArgs& a, int G) {
        const int rows = n * G, size = rows <= kNarrow ? kNarrow : ROWS, at0 = len - n;
        narrow = rows <= kNarrow;
        tiles = (unsigned)(rows + size - 1) / size;
        const Span s(a, at0 + (int)((max(tiles, 1u) - 1) * size / (unsigned)G), len - 1), s0(a, at0, at0 + (min(rows, size) - 1) / G);
        units = tiles == 0 ? 0u : narrow ? (unsigned)(s.tiles(kNarrow) + NW - 1) / NW : (unsigned)s.tiles(kKeys);
        units0 = tiles == 0 || narrow ? units : (unsigned)s0.tiles(kKeys);
    }
    // of all tiles, about (a wide one's beginning and end take as long as kEnds units)
    __device__ __forceinline__ float work() const { return (float)tiles * (0.5f * (float)(units + units0) + (narrow ? 0.f : kEnds)); }
};

template <int ROWS>
__device__ __forceinline__ Prompt prompt_of(const KvPromptArgs& a, int b, int G) {
    const int at = min(max(b, 0), a.B - 1), cap = a.c.width << a.c.ps_shift;
    const int u0 = a.q_starts[at], u1 = a.q_starts[at + 1], n = a.lens[at];
    Prompt p;
    p.t0 = min(max(u0, 0), a.T);
    const int t1 = min(max(u1, p.t0), a.T);
    p.n = t1 - p.t0;
    p.len = min(max(n, 0), cap);
    p.bad = p.t0 != u0 || t1 != u1 || p.len != n || p.n > p.len;
    if (b < 0 || b >= a.B) p.n = 0;
    p.template count<ROWS>(a, G);
    return p;
}

// The last `tiles` of a sequence's tiles of rows are cut into `parts` stretches, where
// `part` units each give all workgroups work: no more than about the root of the units,
// since the last one reads all shares, and none of short tiles, since leaving and
// joining takes about 8 us, and a unit 1 to 1.5.  (With one bf16 number a probability: 64 tokens of 4 heads behind 2048, 4096 and
// 32768 entries: 24, 27 and 55 us; up to twice as many stretches 27, 33 and 75, none
// 33, 56 and 380.)  Of a wide sequence those of more than a stretch's units are cut, and
// into longer ones where the shares would take more than the sequence's `slots`.  (One
// prompt of 2000, 4096, 6000 and 8192 tokens of 4 heads 26, 47, 68 and 109 us, not cut 29,
// 62, 88 and 121; with no account of the tiles' ends 4 prompts of 2000 take 50 for 41)
struct Cut {
    unsigned tiles, parts;
};

__device__ __forceinline__ Cut cut_of(const Prompt& p, float part, float slots, float per, int split) {
    const float units = (float)p.units, tiles = (float)p.tiles;
    if (p.narrow) {
        const unsigned parts = !split || units < 8.f ? 1u : max(1u, (unsigned)fminf(ceilf(units / part), 1.4f * __fsqrt_rn(units)));
        return Cut{parts > 1 ? p.tiles : 0u, parts};
    }
    Cut c{0u, 1u};
    if (!split || units < 16.f) return c;
    float size = fmaxf(part, 1.5f * __fsqrt_rn(units));
    bool done = false;
#pragma unroll 1
    for (int i = 0; i < 6 && __any(!done); ++i) {
        const float parts = ceilf(units / size), over = units - fmaxf(size, 12.f), slope = units - (float)p.units0;
        const float x = slope <= over ? tiles : ceilf(tiles * over / slope);
        if (!done && (parts < 2.f || x * parts * per <= slots)) {
            done = true;
            if (parts >= 2.f && x > 0.f) c = Cut{(unsigned)x, (unsigned)parts};
        }
        size *= 1.4f;
    }
    return c;
}

// What a workgroup does: a tile of rows (r0 on) of sequence b, of its entries'
// tiles the part-th of `parts` stretches
struct Item {
    int b, t0, n, len, r0;
    unsigned part, parts;
    int slot;             // the first share's, of the tile's
    bool narrow;
};

// The workgroup's item; b -1: there is none.  All workgroups see the same plan.
// Wide tiles come first; the last sequence's last tile, which sees most, before
// the others.  Up to kMine sequences each wave looks up by itself; of more, the first
// HELD (from the last on) are looked up by the four waves together and kept in LDS, with
// the tiles of each 64 of them.  (All looked up by each wave, again for each kind: 300
// sequences of 16 tokens 27.5 us where these take 16, 1500 of 8 tokens 158 and 59)
constexpr int kMine = 256;

template <int ROWS, int HELD>
__device__ __forceinline__ Item item_of(const KvPromptArgs& a, int G, unsigned item, int kvh, u32x4* held, int (*groups)[64], float2 (*stat)[32]) {
    constexpr int C = kMine / 64;       // sequences a lane has at once
    const int l = threadIdx.x & 63, hkv = a.c.hkv;
    const float heads = (float)hkv;
    const bool together = a.B > kMine;
    Prompt p[C];
    auto at = [&](int c0) __attribute__((always_inline)) {
#pragma unroll
        for (int x = 0; x < C; ++x) p[x] = prompt_of<ROWS>(a, a.B - 1 - c0 - 64 * x - l, G);
    };
    auto again = [&](int c0) __attribute__((always_inline)) {
        if (c0 >= HELD) return at(c0);
#pragma unroll
        for (int x = 0; x < C; ++x) {
            const u32x4 v = held[c0 + 64 * x + l];
            p[x].t0 = (int)v[0], p[x].n = (int)v[1], p[x].len = (int)v[2];
            p[x].template count<ROWS>(a, G);
        }
    };
    Item it;
    it.b = -1;
    it.t0 = it.n = it.len = it.r0 = 0;
    it.part = 0;
    it.parts = 1;
    it.slot = 0;
    it.narrow = false;
    // units of work of either kind
    float units[2] = {0.f, 0.f};
    bool bad = false;
    // (together: a wave's share of the sequences, the sums of all of them at the end)
    const int w = wave_id();
    for (int c0 = together ? kMine * w : 0; c0 < a.B; c0 += together ? kMine * NW : kMine) {
        at(c0);
        if (together && c0 < HELD)
#pragma unroll
            for (int y = 0; y < C; ++y) {
                held[c0 + 64 * y + l] = u32x4{(unsigned)p[y].t0, (unsigned)p[y].n, (unsigned)p[y].len, 0u};
                const int n0 = wave_total(wave_incl_scan(p[y].narrow ? 0 : (int)p[y].tiles));
                const int n1 = wave_total(wave_incl_scan(p[y].narrow ? (int)p[y].tiles : 0));
                if (l == 0) groups[0][c0 / 64 + y] = n0, groups[1][c0 / 64 + y] = n1;
            }
        float x[2] = {0.f, 0.f};
#pragma unroll
        for (int y = 0; y < C; ++y) {
            bad |= p[y].bad;
            const float u = p[y].work();
            x[0] += p[y].narrow ? 0.f : u;
            x[1] += p[y].narrow ? u : 0.f;
        }
        if (a.split)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
#pragma unroll
                for (int y = 32; y; y >>= 1) x[k] += __shfl_xor(x[k], y);
                units[k] += x[k];
            }
    }
    if (bad) kv_error(a.c);
    if (together) {
        if (l == 0) stat[w][0] = float2{units[0], units[1]};
        const bool some = __any(bad);
        if (l == 0) stat[w][1] = float2{some ? 1.f : 0.f, 0.f};
        __syncthreads();
        units[0] = units[1] = 0.f;
#pragma unroll
        for (int y = 0; y < NW; ++y) {
            units[0] += stat[y][0].x, units[1] += stat[y][0].y;
            bad |= stat[y][1].x != 0.f;
        }
    }
    // (starts that do not ascend can name more rows than the grid is for, and a share
    // that nobody brings would be waited for in the next call: nothing is cut then)
    const int split = __any(bad) ? 0 : a.split;
    const int both = units[0] > 0.f && units[1] > 0.f ? 2 : 1;
    const float part_of[2] = {fmaxf(1.f, units[0] * heads / (float)(kCutItems / both)) + kJoin,
                              fmaxf(1.f, units[1] * heads / (float)(kCutNarrow / both))};
    if (together && !split && a.B <= HELD) {
        // nothing is cut: the group of 64 sequences, then the one of them
        const bool in = 64 * l < (a.B + kMine - 1) / kMine * kMine;
        unsigned left = item;
#pragma unroll 1
        for (int kind = 0; kind < 2; ++kind) {
            const unsigned n = in ? (unsigned)groups[kind][l] : 0u, incl = (unsigned)wave_incl_scan((int)n);
            const unsigned long long over = __ballot(incl > left);
            if (over) {
                const int g = __ffsll((long long)over) - 1;
                left -= lane_of(incl - n, g);
                Prompt q;
                const u32x4 v = held[64 * g + l];
                q.t0 = (int)v[0], q.n = (int)v[1], q.len = (int)v[2];
                q.template count<ROWS>(a, G);
                const unsigned tiles = q.narrow == (kind == 1) ? q.tiles : 0u, upto = (unsigned)wave_incl_scan((int)tiles);
                const int i = __ffsll((long long)__ballot(upto > left)) - 1;
                it.b = a.B - 1 - 64 * g - i;
                it.t0 = __builtin_amdgcn_readlane(q.t0, i);
                it.n = __builtin_amdgcn_readlane(q.n, i);
                it.len = __builtin_amdgcn_readlane(q.len, i);
                it.narrow = kind == 1;
                it.r0 = (int)((lane_of(upto, i) - 1 - left) * (kind ? kNarrow : ROWS));
                return it;
            }
            left -= lane_of(incl, 63);
        }
        return it;
    }
    unsigned before = 0, slots = 0;
#pragma unroll 1
    for (int kind = 0; kind < 2; ++kind) {
        const unsigned per = kind ? 2 : ROWS / 16;                // slots of a share
#pragma unroll 1
        for (int c0 = 0; c0 < a.B; c0 += kMine) {
            if (together) again(c0);
#pragma unroll
            for (int x = 0; x < C; ++x) {
                if (x > 0 && c0 + 64 * x >= a.B) continue;
                const unsigned tiles = p[x].narrow == (kind == 1) ? p[x].tiles : 0u;
                Cut cut{0u, 1u};
                if (tiles) cut = cut_of(p[x], part_of[kind], (float)(kKvPromptSlots / both) * p[x].work() / units[kind], heads * (float)per, split);
                const unsigned need = (unsigned)fminf((float)cut.tiles * (float)cut.parts * heads * (float)per, 1e6f);
                const unsigned slot_incl = slots + (unsigned)wave_incl_scan((int)need);
                if (slot_incl > (unsigned)kKvPromptSlots) cut = Cut{0u, 1u};  // (what finds no slots is not cut)
                const unsigned incl = before + (unsigned)wave_incl_scan((int)(tiles + cut.tiles * (cut.parts - 1)));
                const unsigned long long over = __ballot(incl > item);
                if (over) {
                    const int i = __ffsll((long long)over) - 1;
                    it.b = a.B - 1 - c0 - 64 * x - i;
                    it.t0 = __builtin_amdgcn_readlane(p[x].t0, i);
                    it.n = __builtin_amdgcn_readlane(p[x].n, i);
                    it.len = __builtin_amdgcn_readlane(p[x].len, i);
                    it.narrow = kind == 1;
                    const unsigned z = lane_of(incl, i) - 1 - item, parts = lane_of(cut.parts, i), uncut = lane_of(tiles - cut.tiles, i);
                    unsigned tile = z;
                    if (z >= uncut) {
                        const unsigned k = (z - uncut) / parts;
                        it.parts = parts;
                        it.part = z - uncut - k * parts;
                        it.slot = (int)(lane_of(slot_incl - need, i) + (k * (unsigned)hkv + (unsigned)kvh) * parts * per);
                        tile = uncut + k;
                    }
                    it.r0 = (int)(tile * (kind ? kNarrow : ROWS));
                    return it;
                }
                before = lane_of(incl, 63);
                slots = min(lane_of(slot_incl, 63), 2u * kKvPromptSlots);
            }
        }
    }
    return it;
}

// A wave's 32 rows: queries, running maximum and sum, output.  Lane: row lr = l % 32
// (both halves of the wave; they have the sum in parts); o[dt][i]: number
// 32 dt + 8 (i / 4) + 4 (l / 32) + i % 4 of it
template <int D, int FMT>
struct Rows {
    static constexpr int KS = D / 16, DT = D / 32;
    u32x4 q[KS];
    f32x16 o[DT];
    float m, sum;
    int l, lr, lh;
    int p;                    // the row's own entry
    long long row;            // of q and out
    int hq;                   // its query head
    int first, last;          // own entries of the wave's first and last row

    // rows r0 + lr of a tile's, those from r1 on are r1 - 1 again
    __device__ __forceinline__ void init(const KvPromptArgs& a, const Item& it, int kvh, int G, int r0, int r1) {
        l = threadIdx.x & 63;
        lr = l & 31;
        lh = l >> 5;
        const int r = min(r0 + lr, r1 - 1), tok = r / G, h = r - tok * G, at0 = it.len - it.n;
        p = at0 + tok;
        first = at0 + r0 / G;
        last = at0 + min(r0 + 31, r1 - 1) / G;
        row = it.t0 + tok;
        hq = kvh * G + h;
        const uint16_t* const qp = a.q + row * a.q_stride + hq * D + 8 * lh;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            q[ks] = ld16(qp + 16 * ks);
#pragma unroll
            for (int i = 0; i < 4; ++i) q[ks][i] ^= a.q_sign;
        }
        m = -INFINITY;
        sum = 0.f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt] = f32x16{};
    }

    // products with 32 keys of LDS, rows r on: lane has entries 8 (i / 4) + 4 lh + i % 4
    // (ln: the lane, for LDS addresses)
    __device__ __forceinline__ void read(const u32x4* keys, int r, u32x4 (&k)[KS], int ln) const {
#pragma unroll
        for (int x = 0; x < KS; ++x) k[x] = keys[k_at<D>(r + (ln & 31), 2 * x + (ln >> 5))];
    }
    __device__ __forceinline__ f32x16 products(const u32x4 (&k)[KS]) const {
        f32x16 s = f32x16{};
#pragma unroll
        for (int x = 0; x < KS; ++x) s = mfma32(k[x], q[x], s);
        return s;
    }
    // those of entries e0 on, blocks of 16 that are there in `there`, to be seen or not;
    // times the scales of an int8 cache's blocks (which may be NaN: what does not see
    // the block must not)
    __device__ __forceinline__ void mask(const KvPromptArgs& a, f32x16& s, const Tile& t, int e0, unsigned there, const float* ks) const {
        int hh = lh;
        asm volatile("" : "+v"(hh));            // (a branch: not done and thrown away where all are seen; no registers across the tiles)
        const int to = min(t.hi - 1, p), from = a.window ? p - a.window + 1 : 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int e = e0 + 8 * (i / 4) + 4 * hh + i % 4;
            const bool sees = (e <= to) & (e >= t.lo) & ((e >= from) | (e < a.sinks)) & (bool)(there >> (i / 8) & 1);
            s[i] = sees ? FMT == kInt8 ? s[i] * ks[i / 8] : s[i] : -INFINITY;
        }
    }
    __device__ __forceinline__ float top_of(const f32x16& s, float scale0, float scale1) const {
        float x[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            x[k] = s[8 * k];
#pragma unroll
            for (int i = 1; i < 8; ++i) x[k] = fmaxf(x[k], s[8 * k + i]);
        }
        return FMT == kInt8 ? fmaxf(x[0] * scale0, x[1] * scale1) : fmaxf(x[0], x[1]) * scale0;
    }
    // The maximum follows only where a score passes it by 8 (in units of log 2):
    // until then no exponential exceeds 2^8.  follow: the factor of the output so far
    __device__ __forceinline__ bool passes(float top) const { return __any(top > m + 8.f); }
    __device__ __forceinline__ float follow(float top) {
        top = fmaxf(top, __shfl_xor(top, 32));
        const float mn = fmaxf(m, top), f = m == -INFINITY ? 0.f : exp2_(m - mn);
        m = mn;
        sum *= f;
        return f;
    }
    __device__ __forceinline__ void rescale(float f) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt] *= f;
    }
    // exponentials, summed, and as the second product's operand; vs: an int8 cache's
    // scales of the values
    __device__ __forceinline__ void exponentials(const f32x16& s, float scale0, float scale1, const float* vs, u32x4 (&pb)[2]) {
        const float mm = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const float f = FMT == kInt8 && k ? scale1 : scale0;
                float x = exp2_(fmaf(s[8 * k + i], f, -mm)), y = exp2_(fmaf(s[8 * k + i + 1], f, -mm));
                sum += x + y;
                if constexpr (FMT == kInt8) x = bdl_mul_legacy(x, vs[k]), y = bdl_mul_legacy(y, vs[k]);
                pb[k][i / 2] = pk_bf16(x, y);
            }
        // (computed here, beside the products that go on, and not where they are used)
        asm volatile("" : "+v"(pb[0]), "+v"(pb[1]), "+v"(sum));
    }
    // part dt of 16 transposed values of LDS, rows r on
    __device__ __forceinline__ u32x4 values_of(const u32x4* values, int r, int dt, int ln) const {
        s16x4 v[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int at = v32_at<D>(r + 8 * x + 4 * (ln >> 5) + ((ln & 15) >> 2), 4 * dt + 2 * ((ln >> 4) & 1) + ((ln >> 1) & 1));
            v[x] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(reinterpret_cast<const short*>(values + at) + 4 * (ln & 1)));
        }
        return __builtin_bit_cast(u32x4, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
    }
    // out^T += V^T P^T over 32 values of LDS, rows r on
    __device__ __forceinline__ void add(const u32x4* values, int r, const u32x4 (&pb)[2], int ln) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) o[dt] = mfma32(values_of(values, r + 16 * k, dt, ln), pb[k], o[dt]);
    }
    // Exponentials and their product with 32 values of LDS, rows 0 on, where they are kept
    // as three bf16 numbers whose sum they are, all 24 bits: each cut towards zero, what
    // is left over is exact.  Where the first is not 0 the others are at least 2^-133, so
    // that an infinite value gives an infinite sum and no NaN (int8 has none).  (64 single
    // tokens of 4 heads of 128 behind 2048, 4096 and 32768 entries each: bf16 26.2, 35.4
    // and 204 us, int8 22.9, 29.6 and 130; one number 24.6, 33.2 and 199, 21.1, 26.5 and 112)
    __device__ __forceinline__ void add_exponentials(const f32x16& s, float scale0, float scale1, const float* vs, const u32x4* values) {
        const float mm = m == -INFINITY ? 0.f : m;
        int ln = l;
        asm volatile("" : "+v"(ln));                // (no addresses kept in registers across the tiles)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            u32x4 pb[3];
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const float f = FMT == kInt8 && k ? scale1 : scale0;
                float x = exp2_(fmaf(s[8 * k + i], f, -mm)), y = exp2_(fmaf(s[8 * k + i + 1], f, -mm));
                sum += x + y;
                if constexpr (FMT == kInt8) x = bdl_mul_legacy(x, vs[k]), y = bdl_mul_legacy(y, vs[k]);
                const float x1 = below_bf16(x), y1 = below_bf16(y);
                const uint32_t h = upper_halves(x, y), some = FMT == kInt8 ? 0u : min_u16x2(h, 0x00010001u);
                pb[0][i / 2] = h;
                pb[1][i / 2] = max_u16x2(upper_halves(x1, y1), some);
                pb[2][i / 2] = max_u16x2(upper_halves(below_bf16(x1), below_bf16(y1)), some);
            }
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                const u32x4 v = values_of(values, 16 * k, dt, ln);
#pragma unroll
                for (int n = 0; n < 3; ++n) o[dt] = mfma32(v, pb[n], o[dt]);
            }
        }
    }
    // the maximum follows the scores of 32 keys of LDS, rows r on, which stand for entries e0 on of tile t
    __device__ __forceinline__ void follow_tile(const KvPromptArgs& a, const u32x4* keys, int r, const Tile& t, int e0, unsigned there) {
        const float ones[2] = {1.f, 1.f};
        int ln = l;
        asm volatile("" : "+v"(ln));
        // (registers: one read at a time)
        f32x16 s = f32x16{};
#pragma unroll
        for (int x = 0; x < KS; ++x) {
            s = mfma32(keys[k_at<D>(r + (ln & 31), 2 * x + (ln >> 5))], q[x], s);
            __builtin_amdgcn_sched_barrier(0);
        }
        mask(a, s, t, e0, there, ones);
        const float top = top_of(s, a.score_scale, a.score_scale);
        if (passes(top)) rescale(follow(top));
    }
    // Infinities and NaN among the values of LDS, rows k0 .. k1 - 1 of tile t, are added
    // to the rows that see them as they are (any probability times them is they).  After
    // the rows' maximum has followed the tile's scores: infinity times a factor that
    // vanishes, or the 0 that stands for no maximum yet, is a NaN
    __device__ __forceinline__ void poison(const KvPromptArgs& a, const u32x4* values, int k0, int k1, const Tile& t, unsigned there) {
        int hh = lh;
        asm volatile("" : "+v"(hh));
#pragma unroll 1
        for (int k = k0; k < k1; ++k) {
            const int e = t.e + k;
            const bool in = e <= min(t.hi - 1, p) && e >= t.lo && (!a.window || e > p - a.window || e < a.sinks) && (there >> (k / 16) & 1);
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint2 v = reinterpret_cast<const uint2*>(values + v32_at<D>(k, 4 * dt + i))[hh];
                    const float x[4] = {__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16),
                                        __uint_as_float(v.y & 0xffff0000u)};
#pragma unroll
                    for (int z = 0; z < 4; ++z) o[dt][4 * i + z] += in && !(fabsf(x[z]) < INFINITY) ? x[z] : 0.f;
                    __builtin_amdgcn_sched_barrier(0);          // (registers: one read at a time)
                }
        }
    }
    // A block of an int8 cache that stands for NaN, entries e0 on of tile t: rows that see
    // one of them are NaN, also where its probability is 0
    __device__ __forceinline__ void nan_block(const KvPromptArgs& a, const Tile& t, int e0) {
        const int lo = max(t.lo, e0), to = min(min(t.hi - 1, p), e0 + 15), from = a.window ? p - a.window + 1 : 0;
        const bool sees = max(lo, from) <= to || lo <= min(to, a.sinks - 1);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[dt][i] = sees ? NAN : o[dt][i];
    }
    // output numbers of part dt of the row, and with the first its lse
    __device__ __forceinline__ void finish(const KvPromptArgs& a, int dt, const f32x16& v, float top, float total) const {
        const bool none = total == 0.f;
        const float g = a.v_scale / total;
        uint16_t* const out = a.out + row * a.out_stride + hq * D + 32 * dt + 4 * lh;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<uint2*>(out + 8 * i) =
                uint2{none ? 0u : pk_bf16(v[4 * i] * g, v[4 * i + 1] * g), none ? 0u : pk_bf16(v[4 * i + 2] * g, v[4 * i + 3] * g)};
        if (dt == 0 && lh == 0 && a.lse) a.lse[row * a.c.hq + hq] = none ? -INFINITY : (top + __log2f(total)) * kLn2;
    }
};

// A tile's shares in the workspace: [part][rows][D] sums, then [rows][2] maxima and
// sums.  Byte offset of part x's, and how its rows are written and read
template <int D>
struct Shares {
    __amdgpu_buffer_rsrc_t r;
    unsigned base, size, stats;
    __device__ __forceinline__ Shares(const KvPromptArgs& a, const Item& it, int rows16) {
        r = buf_rsrc(a.part, (unsigned)kKvPromptSlots * 16u * (D + 2) * 4u);
        size = (unsigned)rows16 * 16u * (D + 2) * 4u;
        stats = (unsigned)rows16 * 16u * D * 4u;
        base = (unsigned)it.slot * (16u * (D + 2) * 4u);
    }
    __device__ __forceinline__ unsigned at(unsigned part, int row, int dt, int lh) const {
        return base + part * size + (unsigned)(row * D + 32 * dt + 4 * lh) * 4u;
    }
    __device__ __forceinline__ void put(unsigned part, int row, int dt, int lh, const f32x16& v) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) store_through(r, at(part, row, dt, lh) + 32 * i, f32x4{v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]});
    }
    __device__ __forceinline__ void put_stat(unsigned part, int row, float m, float sum) const {
        store_through(r, base + part * size + stats + row * 8u, float2{m, sum});
    }
    __device__ __forceinline__ float2 stat(unsigned part, int row) const { return load_through2(r, base + part * size + stats + row * 8u); }
    // N parts of the output from dt on, of a row from all of its shares, in their order
    template <int N>
    __device__ __forceinline__ void sum(unsigned parts, int row, int dt, int lh, f32x16 (&v)[N], float& top, float& total) const {
        constexpr int U = N == 1 ? 8 : N == 2 ? 4 : 2;      // shares whose loads are in flight at once
#pragma unroll
        for (int z = 0; z < N; ++z) v[z] = f32x16{};
        top = -INFINITY;
        total = 0.f;
#pragma unroll 1
        for (unsigned x0 = 0; x0 < parts; x0 += U) {
            float2 ms[U];
            f32x4 y[U][N][4];
#pragma unroll
            for (int x = 0; x < U; ++x) {
                const bool in = x0 + x < parts;
                ms[x] = stat(in ? x0 + x : x0, row);
                if (!in) ms[x] = float2{-INFINITY, 0.f};
#pragma unroll
                for (int z = 0; z < N; ++z)
#pragma unroll
                    for (int i = 0; i < 4; ++i) y[x][z][i] = load_through4(r, in ? at(x0 + x, row, dt + z, lh) + 32 * i : kOob);
            }
            float tn = top;
#pragma unroll
            for (int x = 0; x < U; ++x) tn = fmaxf(tn, ms[x].x);
            const float fo = top == -INFINITY ? 0.f : exp2_(top - tn);
            top = tn;
            total *= fo;
#pragma unroll
            for (int z = 0; z < N; ++z) v[z] *= fo;
            bool out = false;                               // some are left out
#pragma unroll
            for (int x = 0; x < U; ++x) {
                const float f = ms[x].x == -INFINITY ? 0.f : exp2_(ms[x].x - top);
                total += f * ms[x].y;
                out |= f == 0.f && ms[x].x != -INFINITY;
                if (f != 0.f)
#pragma unroll
                    for (int z = 0; z < N; ++z)
#pragma unroll
                        for (int i = 0; i < 16; ++i) v[z][i] += f * y[x][z][i / 4][i % 4];
            }
            if (out)
#pragma unroll
                for (int x = 0; x < U; ++x)
#pragma unroll
                    for (int z = 0; z < N; ++z)
#pragma unroll
                        for (int i = 0; i < 16; ++i) v[z][i] = keep_nan(v[z][i], y[x][z][i / 4][i % 4]);
        }
    }
};

// this workgroup's share has reached memory: whether it is the tile's last
__device__ __forceinline__ bool last_share(const KvPromptArgs& a, const Item& it, int* flag) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) {
        unsigned* const c = a.count + (it.slot >> 1) * kKvCount;
        const bool last = __hip_atomic_fetch_add(c, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == it.parts - 1;
        if (last) __hip_atomic_store(c, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        *flag = last;
    }
    __syncthreads();
    return uni(*flag);
}

// Where the blocks of 16 entries of several tiles lie (and an int8 cache's scales), a
// block a lane; in `ok` those that are there.  `bytes`: what counts from the block on,
// of up to SPAN entries
template <int D, int FMT, int SPAN>
struct Blocks {
    static constexpr int ROW = D * (FMT == kBf16 ? 2 : 1);
    int page_next = -1;
    unsigned at_lo = 0, at_hi = 0, bytes = 0;
    float2 scale = float2{1.f, 1.f};
    unsigned long long ok = 0;
    // in: whether the lane's block at entry e, of a tile whose entries lo .. hi - 1
    // count, will be loaded: its page's number is asked for
    __device__ __forceinline__ bool counts(bool in, int e, const Tile& t) const { return in && e < t.hi && e + SPAN > t.lo; }
    __device__ __forceinline__ void look(const KvPromptArgs& a, int b, bool in, int e, const Tile& t) {
        page_next = counts(in, e, t) ? a.c.table[(long long)b * a.c.tstride + (e >> a.c.ps_shift)] : -1;
    }
    __device__ __forceinline__ void turn(const KvPromptArgs& a, int kvh, bool in, int e, const Tile& t) {
        const int page = page_next;
        const bool some = counts(in, e, t), there = some && (unsigned)page < (unsigned)a.c.n_pages;
        if (some && !there) kv_error(a.c);
        ok = __ballot(there);
        const unsigned long long entry = there ? (((unsigned long long)(unsigned)page * (unsigned)a.c.hkv + (unsigned)kvh) << a.c.ps_shift) +
                                                     (unsigned)(e & ((1 << a.c.ps_shift) - 1)) : 0ull;
        at_lo = (unsigned)(entry * ROW);
        at_hi = (unsigned)(entry * ROW >> 32);
        bytes = there ? (unsigned)min(SPAN, t.hi - e) * ROW : 0u;
        if constexpr (FMT == kInt8) scale = there ? *reinterpret_cast<const float2*>(a.c.scales + 2 * (entry >> 4)) : float2{1.f, 1.f};
    }
    __device__ __forceinline__ unsigned long long at(int x) const { return (unsigned long long)lane_of(at_hi, x) << 32 | lane_of(at_lo, x); }
};

// Whether a bf16 number of eight is an infinity or a NaN, and zeros in place of such
__device__ __forceinline__ uint32_t size_of(u32x4 v) {
    return max_u16x2(max_u16x2(v[0] & 0x7fff7fffu, v[1] & 0x7fff7fffu), max_u16x2(v[2] & 0x7fff7fffu, v[3] & 0x7fff7fffu));
}
__device__ __forceinline__ bool infinite(uint32_t size) { return (size & 0xffffu) >= 0x7f80u || size >= 0x7f800000u; }
__device__ __forceinline__ u32x4 finite_only(u32x4 v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if ((v[i] & 0x7f80u) == 0x7f80u) v[i] &= 0xffff0000u;
        if ((v[i] & 0x7f800000u) == 0x7f800000u) v[i] &= 0xffffu;
    }
    return v;
}

template <int FMT>
__device__ __forceinline__ u32x4 widen(u32x4 v, int half) {
    return FMT == kFp8 ? bf16_of(v[2 * half], v[2 * half + 1]) : bf16_of_int8(v[2 * half], v[2 * half + 1]);
}

// ------------------------------------------------------------------ wide
// PAGE: pages hold whole tiles (64 entries or more), else blocks of 16.  RW waves
// have rows of their own, and 4 / RW the same rows and a part of a tile's entries each
template <int D, int FMT, bool PAGE, int RW>
__device__ __forceinline__ void wide(const KvPromptArgs& a, const Item& it, int kvh, int G, u32x4 (*lds)[2][kKeys * D / 8], float2 (*stat)[32],
                                     int* flag) {
    constexpr int ROWS = RW * 32, SPAN = PAGE ? kKeys : 16;
    constexpr int ROW = D * (FMT == kBf16 ? 2 : 1), CPR = ROW / 16;
    constexpr int LPT = kKeys * CPR / NT;           // 16-byte loads of a thread for a tile's keys
    constexpr int DT = D / 32;
    const int w = wave_id(), l = threadIdx.x & 63, rw = w % RW, half = w / RW;
    const int rows = min(ROWS, it.n * G - it.r0), at0 = it.len - it.n;
    const Span span(a, at0 + it.r0 / G, at0 + (it.r0 + rows - 1) / G);
    const int tiles = span.tiles(kKeys), nS = span.sink_tiles(kKeys), base = span.begin & -kKeys;
    const int c0 = (int)((unsigned long long)tiles * it.part / it.parts), c1 = (int)((unsigned long long)tiles * (it.part + 1) / it.parts);
    const bool busy = 32 * rw < rows;               // the wave has rows
    const int wr0 = it.r0 + min(32 * rw, rows - 1), r1 = it.r0 + rows;
    Rows<D, FMT> R;
    R.init(a, it, kvh, G, wr0, r1);
    // tiles that no row of the wave sees are passed over: those before `gone` (but
    // the sinks') and from `past` on; those from whole0 to whole1 are seen whole by all
    // of them (rounded down, numbers may be < 0)
    const int past = nS + ((R.last - base) >> 6) + 1;
    const int gone = a.window && a.sinks <= base ? nS + ((R.first - a.window + 1 - base) >> 6) : nS;
    const int whole1 = nS + ((R.first + 1 - base) >> 6);
    const int whole0 = nS + ((max(span.begin, a.window ? R.last - a.window + 1 : 0) - base + kKeys - 1) >> 6);

    // 16 tiles' blocks.  Tiles are loaded in order; the pages of the next 16 are asked
    // for when the first of these is loaded
    Blocks<D, FMT, SPAN> blocks;
    auto look = [&](int x0) __attribute__((always_inline)) {
        const Tile t = tile_at(span, kKeys, x0 + (l >> 2));
        blocks.look(a, it.b, x0 + (l >> 2) < c1, t.e + 16 * (l & 3), t);
    };
    auto turn = [&](int x0) __attribute__((always_inline)) {
        const Tile t = tile_at(span, kKeys, x0 + (l >> 2));
        blocks.turn(a, kvh, x0 + (l >> 2) < c1, t.e + 16 * (l & 3), t);
        look(x0 + 16);
    };
    // of the tile being worked on: blocks that are there, and their scales.  (With a bit
    // where a value's scale is NaN: such a tile is not one of the whole ones)
    constexpr unsigned kNanBlock = 16u;
    unsigned there = 0, there_next = 0;
    float ks[4], vs[4], ks_next[4], vs_next[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) ks[k] = vs[k] = ks_next[k] = vs_next[k] = 1.f;
    u32x4 kr[LPT], vr[LPT];                         // (8-bit formats)
    // Where this lane's pieces lie in a tile, or in a block.  bf16 goes straight into
    // LDS, lane after lane, and the pieces of a row are exchanged on the way; what
    // lies before the first entry may be NaN, and 0 times NaN is one: zeros in its place
    constexpr int BUF = kKeys * D / 8;
    const unsigned lds_w = lds_address(lds) + (unsigned)w * 1024u;
    unsigned ko[LPT], vo[LPT];
#pragma unroll
    for (int i = 0; i < LPT; ++i) {
        const int id = i * NT + (int)threadIdx.x, r = id / CPR, c = id % CPR, from = (PAGE ? r : r & 15) * CPR;
        ko[i] = (unsigned)(from + (FMT == kBf16 ? k_at<D>(r, c) % CPR : c)) * 16;
        vo[i] = (unsigned)(from + v32_at<D>(r, c) % CPR) * 16;
    }
    // the next tile: where it is, then its loads piece by piece
    const char *pk = nullptr, *pv = nullptr;
    unsigned size = 0;
    int from = 0;                                   // (its place in the tile of the first entry that counts)
    auto find = [&](int ct) __attribute__((always_inline)) {
        if ((ct & 15) == 0 && ct > c0) turn(ct);
        const int l0 = 4 * (ct & 15);
        there_next = (unsigned)(blocks.ok >> l0) & 15u;
        if constexpr (FMT == kBf16) {
            const Tile t = tile_at(span, kKeys, ct);
            from = t.lo - t.e;
        }
        if constexpr (PAGE) {
            const unsigned long long at = blocks.at(l0);
            size = lane_of(blocks.bytes, l0);
            pk = a.c.K + at;
            pv = a.c.V + at;
        }
        if constexpr (FMT == kInt8)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                ks_next[k] = __uint_as_float(lane_of(__float_as_uint(blocks.scale.x), l0 + k));
                vs_next[k] = __uint_as_float(lane_of(__float_as_uint(blocks.scale.y), l0 + k));
                if (vs_next[k] != vs_next[k]) there_next |= kNanBlock;
            }
    };
    constexpr int PIECES = 2 * LPT;
    auto piece = [&](auto buf, int ct, int x) __attribute__((always_inline)) {
        const int i = x >> 1;
        if (!PAGE && (x & 1) == 0) {
            // 64 pieces of 16 bytes a wave, of one block of 16 entries
            const int y = 4 * (ct & 15) + (i * NT + w * 64) / CPR / 16;
            const unsigned long long at = blocks.at(y);
            size = lane_of(blocks.bytes, y);
            pk = a.c.K + at;
            pv = a.c.V + at;
        }
        if constexpr (FMT == kBf16) {
            const unsigned to = lds_w + (unsigned)(buf * 2 * BUF + i * NT) * 16u;
            if (x & 1)
                copy_to_lds(rsrc_of(pv, size), (i * NT + (int)threadIdx.x) / CPR < from ? kOob : vo[i], to + BUF * 16u);
            else
                copy_to_lds(rsrc_of(pk, size), ko[i], to);
        } else if (x & 1) {
            vr[i] = buf16(buf_rsrc(pv, size), ko[i]);
        } else {
            kr[i] = buf16(buf_rsrc(pk, size), ko[i]);
        }
    };
    auto load = [&](auto buf, int ct) __attribute__((always_inline)) {
        find(ct);
#pragma unroll
        for (int x = 0; x < PIECES; ++x) piece(buf, ct, x);
    };
    // A tile that not all of the workgroup's rows see whole: an infinite value must not
    // reach those that do not see it, as 0 times it would.  It is added to those that
    // do apart, and then is zero for the products
    const int all1 = nS + ((at0 + it.r0 / G + 1 - base) >> 6);
    const int all0 = nS + ((max(span.begin, a.window ? at0 + (it.r0 + rows - 1) / G - a.window + 1 : 0) - base + kKeys - 1) >> 6);
    auto edge = [&](int ct) __attribute__((always_inline)) { return FMT != kInt8 && (ct < all0 || ct >= all1); };
    auto some_see = [&](int ct) __attribute__((always_inline)) { return busy && ct < past && (ct < nS || ct >= gone); };
    auto clean = [&](int buf, int ct) __attribute__((always_inline)) {
        u32x4* const values = lds[buf][1];
        uint32_t size = 0;
#pragma unroll 1
        for (int i = 0; i < BUF / NT; ++i) size = max_u16x2(size, size_of(values[i * NT + (int)threadIdx.x]));
        if (infinite(size)) *flag = 1;              // (stays so: the tiles behind this one are looked at for nothing)
        __syncthreads();
        if (!*flag) return;
        const Tile t = tile_at(span, kKeys, ct);
        if (some_see(ct)) {
            const int h0 = RW == 4 ? 0 : half, h1 = RW == 4 ? 2 : half + 1;
#pragma unroll 1
            for (int h = h0; h < h1; ++h) R.follow_tile(a, lds[buf][0], 32 * h, t, t.e + 32 * h, there >> (2 * h));
            R.poison(a, values, 32 * h0, 32 * h1, t, there);
        }
        __syncthreads();
#pragma unroll 1
        for (int i = 0; i < BUF / NT; ++i) values[i * NT + (int)threadIdx.x] = finite_only(values[i * NT + (int)threadIdx.x]);
        __syncthreads();
    };
    // the loaded tile is in LDS for all waves
    auto arrive = [&](auto buf, int ct) __attribute__((always_inline)) {
        if constexpr (FMT != kBf16) {
            const Tile t = tile_at(span, kKeys, ct);
#pragma unroll
            for (int i = 0; i < LPT; ++i) {
                const int id = i * NT + (int)threadIdx.x, r = id / CPR, c = id % CPR;
                u32x4 v = vr[i];
                if (FMT == kFp8 && t.e + r < t.lo) v = u32x4{0, 0, 0, 0};
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    lds[buf][0][k_at<D>(r, 2 * c + x)] = widen<FMT>(kr[i], x);
                    lds[buf][1][v32_at<D>(r, 2 * c + x)] = widen<FMT>(v, x);
                }
            }
        } else {
            copies_done();
        }
        there = there_next;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            ks[k] = ks_next[k];
            vs[k] = vs_next[k];
        }
        __syncthreads();
    };
    // A tile that all rows of the wave see whole, and the next one's loads, spread
    // among the products
    auto whole = [&](auto buf, int ct) __attribute__((always_inline)) {
        constexpr std::integral_constant<int, 1 - decltype(buf)::value> other{};
        const u32x4 *const keys = lds[buf][0], *const values = lds[buf][1];
        constexpr int KS = Rows<D, FMT>::KS, HALVES = RW == 4 ? 2 : 1, PER = HALVES * KS / PIECES;
        auto scale = [&](int k) __attribute__((always_inline)) { return FMT == kInt8 ? a.score_scale * ks[k] : a.score_scale; };
        find(ct + 1);
        if constexpr (RW == 4) {
            // two halves of 32 entries, so that the matrix products of one go on
            // beside the exponentials of the other
            u32x4 k0[KS], k1[KS], p0[2], p1[2];
            R.read(keys, 0, k0, l);
            if (FMT == kBf16) R.read(keys, 32, k1, l);
            f32x16 s0 = f32x16{}, s1 = f32x16{};
#pragma unroll
            for (int x = 0; x < 2 * KS; ++x) {
                // (8-bit formats: the loads' registers leave no room for it sooner)
                if (FMT != kBf16 && x == KS) R.read(keys, 32, k1, l);
                if (x < KS)
                    s0 = mfma32(k0[x], R.q[x], s0);
                else
                    s1 = mfma32(k1[x - KS], R.q[x - KS], s1);
                if (x % PER == PER - 1 && x / PER < PIECES) {
                    __builtin_amdgcn_sched_barrier(0x406);
                    piece(other, ct + 1, x / PER);
                    __builtin_amdgcn_sched_barrier(0x406);
                }
            }
            const float before = R.sum;
            R.exponentials(s0, scale(0), scale(1), vs, p0);
            const float top = fmaxf(R.top_of(s0, scale(0), scale(1)), R.top_of(s1, scale(2), scale(3)));
            if (R.passes(top)) {                    // (rarely: done again with the new maximum)
                R.sum = before;
                R.rescale(R.follow(top));
                R.exponentials(s0, scale(0), scale(1), vs, p0);
            }
            R.add(values, 0, p0, l);
            R.exponentials(s1, scale(2), scale(3), vs + 2, p1);
            R.add(values, 32, p1, l);
            // (reads of LDS well ahead of the products, and the exponentials among
            // them: without this order, which the compiler leaves where registers are
            // short, 532 us take the place of 517)
            __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);
#pragma unroll
            for (int x = 0; x < 4 * DT; ++x) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                __builtin_amdgcn_sched_group_barrier(0x402, 6, 0);
            }
        } else {
            const float k2[2] = {half ? ks[2] : ks[0], half ? ks[3] : ks[1]}, v2[2] = {half ? vs[2] : vs[0], half ? vs[3] : vs[1]};
            const float f0 = FMT == kInt8 ? a.score_scale * k2[0] : a.score_scale, f1 = FMT == kInt8 ? a.score_scale * k2[1] : a.score_scale;
            u32x4 k[KS], pb[2];
            R.read(keys, 32 * half, k, l);
            f32x16 s = f32x16{};
#pragma unroll
            for (int x = 0; x < KS; ++x) {
                s = mfma32(k[x], R.q[x], s);
                if (x % PER == PER - 1 && x / PER < PIECES) {
                    __builtin_amdgcn_sched_barrier(0x406);
                    piece(other, ct + 1, x / PER);
                    __builtin_amdgcn_sched_barrier(0x406);
                }
            }
            const float top = R.top_of(s, f0, f1);
            if (R.passes(top)) R.rescale(R.follow(top));
            R.exponentials(s, f0, f1, v2, pb);
            R.add(values, 32 * half, pb, l);
        }
    };
    // Any tile: half by half
    auto any = [&](int buf, int ct) __attribute__((always_inline)) {
        const bool some = some_see(ct);
        const bool late = FMT == kBf16 && some;     // the next tile's loads behind the first reads of this one
        if (!late) load(buf ^ 1, ct + 1);
        if (edge(ct)) clean(buf, ct);
        if (!some) return;
        const u32x4 *const keys = lds[buf][0], *const values = lds[buf][1];
        const Tile t = tile_at(span, kKeys, ct);
        const bool all = there == 15u && ct >= whole0 && ct < whole1;
        int ln = l;
        asm volatile("" : "+v"(ln));                // (addresses of its own, that take no registers of the other tiles)
#pragma unroll 1
        for (int h = RW == 4 ? 0 : half; h < (RW == 4 ? 2 : half + 1); ++h) {
            const float k2[2] = {h ? ks[2] : ks[0], h ? ks[3] : ks[1]}, v2[2] = {h ? vs[2] : vs[0], h ? vs[3] : vs[1]};
            const float f0 = FMT == kInt8 && all ? a.score_scale * k2[0] : a.score_scale, f1 = FMT == kInt8 && all ? a.score_scale * k2[1] : a.score_scale;
            u32x4 k[Rows<D, FMT>::KS], pb[2];
            R.read(keys, 32 * h, k, ln);
            if (late && (RW < 4 || h == 0)) load(buf ^ 1, ct + 1);
            f32x16 s = R.products(k);
            if (!all) R.mask(a, s, t, t.e + 32 * h, there >> (2 * h), k2);
            const float top = R.top_of(s, f0, f1);
            if (R.passes(top)) R.rescale(R.follow(top));
            R.exponentials(s, f0, f1, v2, pb);
            R.add(values, 32 * h, pb, ln);
            if (FMT == kInt8 && (there & kNanBlock))
#pragma unroll 1
                for (int k = 0; k < 2; ++k)
                    if ((k ? v2[1] : v2[0]) != (k ? v2[1] : v2[0])) R.nan_block(a, t, t.e + 32 * h + 16 * k);
        }
    };
    constexpr std::integral_constant<int, 0> buf0{};
    constexpr std::integral_constant<int, 1> buf1{};
    if (threadIdx.x == 0) *flag = 0;                // (behind the first tile's barrier it is so for all)
    if (c1 > c0) {
        look(c0 & ~15);
        turn(c0 & ~15);
        load(0, c0);
    }
    arrive(0, c0);
    // (waves leave the inner loop at tiles of their own: each passes as many barriers.
    // Tiles that some row of the workgroup does not see whole are not for it)
    const int from_whole = busy ? max(c0, max(whole0, all0)) : c1, to_whole = busy ? min(c1, min(whole1, all1)) : c0;
    int ct = c0;
#pragma unroll 1
    while (ct < c1) {
        if (ct >= from_whole && ((ct - c0) & 1) == 0) {
#pragma unroll 1
            while (ct < to_whole && there == 15u) {
                whole(buf0, ct);
                arrive(buf1, ++ct);
                if (ct >= to_whole || there != 15u) break;
                whole(buf1, ct);
                arrive(buf0, ++ct);
            }
            if (ct >= c1) break;
        }
        any((ct - c0) & 1, ct);
        ++ct;
        arrive((ct - c0) & 1, ct);
    }
    R.sum += __shfl_xor(R.sum, 32);
    bool mine = busy && wr0 + R.lr < r1;
    if constexpr (RW < 4) {
        // the other half's sums, through LDS (nobody reads tiles any more)
        f32x4* const x = reinterpret_cast<f32x4*>(lds) + rw * (D / 8 * 64);
        if (half) {
            if (l < 32) stat[rw][l] = float2{R.m, R.sum};
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int i = 0; i < 4; ++i) x[(4 * dt + i) * 64 + l] = f32x4{R.o[dt][4 * i], R.o[dt][4 * i + 1], R.o[dt][4 * i + 2], R.o[dt][4 * i + 3]};
        }
        __syncthreads();
        mine = mine && half == 0;
        if (half == 0) {
            const float2 y = stat[rw][R.lr];
            const float M = fmaxf(R.m, y.x), f0 = R.m == -INFINITY ? 0.f : exp2_(R.m - M), f1 = y.x == -INFINITY ? 0.f : exp2_(y.x - M);
            R.m = M;
            R.sum = f0 * R.sum + f1 * y.y;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f32x4 v = x[(4 * dt + i) * 64 + l];
#pragma unroll
                    for (int k = 0; k < 4; ++k) R.o[dt][4 * i + k] = f0 * R.o[dt][4 * i + k] + f1 * v[k];
                }
        }
    }
    const int row = wr0 - it.r0 + R.lr;
    if (it.parts > 1) {
        const Shares<D> sh(a, it, ROWS / 16);
        if (mine) {
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) sh.put(it.part, row, dt, R.lh, R.o[dt]);
            if (R.lh == 0) sh.put_stat(it.part, row, R.m, R.sum);
        }
        // (the waves that have the same rows take their parts of the output)
        constexpr int N = DT * RW / 4;
        if (!last_share(a, it, flag) || !busy || wr0 + R.lr >= r1) return;
        f32x16 v[N];
        float top, total;
        sh.template sum<N>(it.parts, row, half * N, R.lh, v, top, total);
#pragma unroll
        for (int z = 0; z < N; ++z) R.finish(a, half * N + z, v[z], top, total);
        return;
    }
    if (!mine) return;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) R.finish(a, dt, R.o[dt], R.m, R.sum);
}

// ------------------------------------------------------------------ narrow
template <int D, int FMT>
__device__ __forceinline__ void narrow(const KvPromptArgs& a, const Item& it, int kvh, int G, u32x4* lds_, float2 (*stat)[32], int* flag) {
    constexpr int ROW = D * (FMT == kBf16 ? 2 : 1), CPR = ROW / 16;
    constexpr int LPT = kNarrow * CPR / 64;         // 16-byte loads of a lane for a tile's keys
    constexpr int DT = D / 32, BUF = kNarrow * D / 8;
    const int w = wave_id(), l = threadIdx.x & 63;
    const int rows = min(kNarrow, it.n * G - it.r0), at0 = it.len - it.n;
    const Span span(a, at0 + it.r0 / G, at0 + (it.r0 + rows - 1) / G);
    const int tiles = span.tiles(kNarrow), units = (tiles + NW - 1) / NW;
    const int c0 = NW * (int)((unsigned long long)units * it.part / it.parts) + w;
    const int c1 = min(tiles, NW * (int)((unsigned long long)units * (it.part + 1) / it.parts));
    u32x4 *const keys = lds_ + w * 2 * BUF, *const values = keys + BUF;
    Rows<D, FMT> R;
    R.init(a, it, kvh, G, it.r0, it.r0 + rows);

    // 32 of the wave's tiles' blocks, two of a tile; tile i is c0 + NW i
    Blocks<D, FMT, 16> blocks;
    auto look = [&](int i0) __attribute__((always_inline)) {
        const int ct = c0 + NW * (i0 + (l >> 1));
        const Tile t = tile_at(span, kNarrow, ct);
        blocks.look(a, it.b, ct < c1, t.e + 16 * (l & 1), t);
    };
    auto turn = [&](int i0) __attribute__((always_inline)) {
        const int ct = c0 + NW * (i0 + (l >> 1));
        const Tile t = tile_at(span, kNarrow, ct);
        blocks.turn(a, kvh, ct < c1, t.e + 16 * (l & 1), t);
        look(i0 + 32);
    };
    u32x4 kr[LPT], vr[LPT];
    unsigned there = 0;
    float ks[2] = {1.f, 1.f}, vs[2] = {1.f, 1.f};
    auto load = [&](int i) __attribute__((always_inline)) {
        if ((i & 31) == 0) turn(i);
        const int l0 = 2 * (i & 31);
        there = (unsigned)(blocks.ok >> l0) & 3u;
#pragma unroll
        for (int k = 0; k < LPT; ++k) {
            // (64 pieces, all of one block)
            const int x = l0 + k * 64 / CPR / 16, id = k * 64 + l;
            const unsigned off = (unsigned)((id / CPR & 15) * CPR + id % CPR) * 16, size = lane_of(blocks.bytes, x);
            kr[k] = buf16(buf_rsrc(a.c.K + blocks.at(x), size), off);
            vr[k] = buf16(buf_rsrc(a.c.V + blocks.at(x), size), off);
        }
        if constexpr (FMT == kInt8)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                ks[k] = __uint_as_float(lane_of(__float_as_uint(blocks.scale.x), l0 + k));
                vs[k] = __uint_as_float(lane_of(__float_as_uint(blocks.scale.y), l0 + k));
            }
    };
    if (c0 < c1) {
        look(0);
        load(0);
    }
    for (int i = 0, ct = c0; ct < c1; ++i, ct += NW) {
        const Tile t = tile_at(span, kNarrow, ct);
        const unsigned here = there;
        const float k2[2] = {ks[0], ks[1]}, v2[2] = {vs[0], vs[1]};
        // (the wave's LDS operations run in order)
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int k = 0; k < LPT; ++k) {
            const int id = k * 64 + l, r = id / CPR, c = id % CPR;
            u32x4 v = vr[k];
            if (FMT != kInt8 && t.e + r < t.lo) v = u32x4{0, 0, 0, 0};
            if constexpr (FMT == kBf16) {
                keys[k_at<D>(r, c)] = kr[k];
                values[v32_at<D>(r, c)] = v;
            } else {
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    keys[k_at<D>(r, 2 * c + x)] = widen<FMT>(kr[k], x);
                    values[v32_at<D>(r, 2 * c + x)] = widen<FMT>(v, x);
                }
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const bool whole = here == 3u && t.e >= t.lo && t.e + kNarrow <= t.hi && t.e + kNarrow - 1 <= R.first &&
                           (!a.window || t.e > R.last - a.window || t.e + kNarrow <= a.sinks);
        if (FMT != kInt8 && !whole) {
            // (as for wide tiles)
            uint32_t size = 0;
#pragma unroll 2
            for (int k = 0; k < BUF / 64; ++k) size = max_u16x2(size, size_of(values[k * 64 + l]));
            if (__any(infinite(size))) {
                R.follow_tile(a, keys, 0, t, t.e, here);
                R.poison(a, values, 0, kNarrow, t, here);
#pragma unroll 1
                for (int k = 0; k < BUF / 64; ++k) values[k * 64 + l] = finite_only(values[k * 64 + l]);
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            }
        }
        load(i + 1);
        const float f0 = FMT == kInt8 && whole ? a.score_scale * k2[0] : a.score_scale, f1 = FMT == kInt8 && whole ? a.score_scale * k2[1] : a.score_scale;
        u32x4 k[Rows<D, FMT>::KS];
        R.read(keys, 0, k, l);
        f32x16 s = R.products(k);
        if (!whole) R.mask(a, s, t, t.e, here, k2);
        const float top = R.top_of(s, f0, f1);
        if (R.passes(top)) R.rescale(R.follow(top));
        R.add_exponentials(s, f0, f1, v2, values);
        if (const float both = v2[0] + v2[1]; FMT == kInt8 && both != both)
#pragma unroll 1
            for (int k = 0; k < 2; ++k)
                if ((k ? v2[1] : v2[0]) != (k ? v2[1] : v2[0])) R.nan_block(a, t, t.e + 16 * k);
    }
    // the four waves' sums, each in its own part of LDS, added in order; wave dt has
    // part dt of the outputs
    R.sum += __shfl_xor(R.sum, 32);
    f32x4* const x = reinterpret_cast<f32x4*>(lds_);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (l < 32) stat[w][l] = float2{R.m, R.sum};
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i) x[w * 2 * BUF + (4 * dt + i) * 64 + l] = f32x4{R.o[dt][4 * i], R.o[dt][4 * i + 1], R.o[dt][4 * i + 2], R.o[dt][4 * i + 3]};
    __syncthreads();
    const bool mine = w < DT && R.lr < rows;
    const int dt = w;
    f32x16 v = f32x16{};
    float top = -INFINITY, total = 0.f;
    if (mine) {
        float2 st[NW];
#pragma unroll
        for (int z = 0; z < NW; ++z) {
            st[z] = stat[z][R.lr];
            top = fmaxf(top, st[z].x);
        }
#pragma unroll
        for (int z = 0; z < NW; ++z) {
            const float f = st[z].x == -INFINITY ? 0.f : exp2_(st[z].x - top);
            total += f * st[z].y;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x4 y = x[z * 2 * BUF + (4 * dt + i) * 64 + l];
                if (f != 0.f)
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[4 * i + k] += f * y[k];
                else
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[4 * i + k] = keep_nan(v[4 * i + k], y[k]);
            }
        }
    }
    if (it.parts > 1) {
        const Shares<D> sh(a, it, kNarrow / 16);
        if (mine) {
            sh.put(it.part, R.lr, dt, R.lh, v);
            if (dt == 0 && R.lh == 0) sh.put_stat(it.part, R.lr, top, total);
        }
        if (!last_share(a, it, flag) || !mine) return;
        f32x16 u[1];
        sh.template sum<1>(it.parts, R.lr, dt, R.lh, u, top, total);
        v = u[0];
    }
    if (mine) R.finish(a, dt, v, top, total);
}

template <int D, int FMT, bool PAGE, int RW>
__global__ __launch_bounds__(NT, 2) void kv_prompt_kernel(const KvPromptArgs a) {
    __shared__ u32x4 lds[2][2][kKeys * D / 8];
    __shared__ float2 stat[NW][32];
    __shared__ int flag, groups[2][64];
    const int hkv = a.c.hkv, G = a.c.hq / hkv, kvh = blockIdx.x % hkv;
    const Item it = item_of<RW * 32, 4 * kKeys * D / 8>(a, G, blockIdx.x / hkv, kvh, lds[0][0], groups, stat);
    if (it.b < 0) return;
    if (a.B > kMine) __syncthreads();               // (LDS is for tiles from here on)
    if (it.narrow)
        narrow<D, FMT>(a, it, kvh, G, lds[0][0], stat, &flag);
    else
        wide<D, FMT, PAGE, RW>(a, it, kvh, G, lds, stat, &flag);
}

template <int D, int FMT, bool PAGE>
hipError_t launch(KvPromptArgs a, hipStream_t s) {
    const long long G = a.c.hq / a.c.hkv, seqs = std::min(a.T, a.B);
    auto tiles = [&](int rows) { return (a.T * G / rows + seqs) * a.c.hkv; };
    // 64 rows a workgroup where 128 would leave compute units without, or with one long
    // tile beside a short one.  (Single tokens beside prompts are not counted in the second
    // number.  4 heads of 128 on one kv head, 64 and 128 rows: 8 prompts of
    // 1024 29.0 and 30.4 us, 12 of them 46.8 and 42.3, 24 71.8 and 61.9; of 4096, 2 72.7 and
    // 80.3, 4 107 and 119; 4 of 1024 beside 192 single tokens 28 and 35, with 8 heads 37 and
    // 37, in e4m3 40 and 37.5)
    const long long wide = tiles(128);
    const bool half = wide < 320 || a.T * G * a.c.hkv < 256 * 128 || (wide < 768 && a.T * G / 128 >= 64 * seqs);
    const long long items = half ? tiles(64) : wide;
    a.split = items < 1024 && (a.c.width << a.c.ps_shift) > 15 * kKeys;     // (shorter ones are not cut)
    // (a wide stretch takes slots, of which there are so many; narrow ones are at most one a
    // tile more than the items they are made for)
    const int grid = (int)(items + (a.split ? kKvPromptSlots / (half ? 4 : 8) + kCutNarrow + 16 : 0));
    if (half)
        kv_prompt_kernel<D, FMT, PAGE, 2><<<grid, NT, 0, s>>>(a);
    else
        kv_prompt_kernel<D, FMT, PAGE, 4><<<grid, NT, 0, s>>>(a);
    return hipGetLastError();
}

template <int D>
hipError_t launch(const KvPromptArgs& a, bool fp8, hipStream_t s) {
    if (a.c.scales) return launch<D, kInt8, false>(a, s);
    if (fp8) return launch<D, kFp8, false>(a, s);
    return 1 << a.c.ps_shift >= kKeys ? launch<D, kBf16, true>(a, s) : launch<D, kBf16, false>(a, s);
}

}  // namespace

hipError_t launch_kv_prompt(const KvPromptArgs& a, int head_dim, bool fp8, hipStream_t s) {
    return head_dim == 64 ? launch<64>(a, fp8, s) : launch<128>(a, fp8, s);
}

}  // namespace bdl
