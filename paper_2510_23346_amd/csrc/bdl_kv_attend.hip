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
// after sequence and head after head, form one line, of which every wave takes
// an equal stretch, whatever the sequences' lengths.  Its loads run one tile
// ahead, its page numbers two, across the ends of sequences.  A sequence
// within one stretch is finished there; the waves of a workgroup, which have
// neighbouring stretches, meet in LDS once at the end; what a workgroup shares
// with others goes to the workspace, and the one that arrives last adds the
// shares in the line's order (so the result does not depend on which one that
// is).
//
// A wave's products are S^T = K Q^T and O^T = V^T P^T on the matrix units
// (16x16x32, bf16), so that the scores' lanes are already those of the second
// product's operand: P never leaves the registers.  Keys and values go through
// a wave's own part of LDS, which turns the 1 KB loads of whole rows into
// operands; between waves nothing is waited for until the end.
//
// Measured, one launch: 305 MB of keys and values in bf16 (256 sequences of up
// to 4353 entries, 8 query heads of 128 on one kv head) 63.9 us, 4.8 TB/s; 134 MB of
// one sequence of 131072 34.4 us; 72 MB of 64 sequences 21.2 us, in 8 bits
// 22.3 us; one sequence of 509 entries 8.6 us.  What is over the copy's rate in
// the 72 MB is the join (pieces in LDS, their way through memory, the sum of the
// shares: 4 us) and that stretches are whole tiles: 4440 tiles on 2048 waves
// are 2.2 a wave, but 3 for a sixth of them, and a tile of one entry counts
// like a full one.  (The third matrix instruction of the second product: 0.1 to
// 0.5 us.)
#include "bdl_kv_device.h"

namespace bdl {

namespace {

constexpr float kLn2 = 0.6931471805599453f;
constexpr int NW = 4, NT = NW * 64;     // waves and threads of a workgroup, of which a compute unit holds two

// A sequence: entries first .. len - 1 in tiles that begin at a multiple of 16
// (an empty one has a tile too, which writes its row)
struct Seq {
    int len, first;
    unsigned tiles;
    bool bad;         // the given length was none
};

__device__ __forceinline__ Seq seq_of(const KvAttendArgs& a, int b) {
    const int at = min(b, a.B - 1), cap = a.c.width << a.c.ps_shift;     // (at most 2^30)
    const int n = a.lens[at], st = a.starts[at];
    Seq s;
    s.len = min(max(n, 0), cap);
    s.bad = s.len != n;
    s.first = a.has_starts ? max(st, 0) : 0;
    if (s.first >= s.len) s.len = s.first = 0;
    s.tiles = b < a.B ? max(1u, (unsigned)(s.len - (s.first & ~15) + 31) >> 5) : 0u;
    return s;
}

// The line of tiles: `total` (< 2^31: heads x the sequences' tiles) of them, cut
// into 1 << k stretches
struct Line {
    unsigned total;
    int k;
    __device__ __forceinline__ unsigned begin(unsigned w) const { return (unsigned)(((unsigned long long)total * w) >> k); }
    // the stretch that holds tile c
    __device__ __forceinline__ unsigned owner(unsigned c) const {
        unsigned w = min((1u << k) - 1, (unsigned)((float)c * __builtin_amdgcn_rcpf((float)total) * (float)(1u << k)));
        while (begin(w) > c) --w;
        while (begin(w + 1) <= c) ++w;
        return w;
    }
};

__device__ __forceinline__ int uni(int v) { return __builtin_amdgcn_readfirstlane(v); }

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// What is left of a number without its upper 16 bits, those of two numbers side
// by side, and the smaller or larger one of each half
__device__ __forceinline__ float below_bf16(float x) { return x - __uint_as_float(__float_as_uint(x) & 0xffff0000u); }

__device__ __forceinline__ uint32_t upper_halves(float x, float y) {
    return __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);
}

typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t min_u16x2(uint32_t x, uint32_t y) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(u16x2, x), __builtin_bit_cast(u16x2, y)));
}

__device__ __forceinline__ uint32_t max_u16x2(uint32_t x, uint32_t y) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, x), __builtin_bit_cast(u16x2, y)));
}

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

// A tile: two blocks of 16 entries, each within one page, of one head of one
// sequence
struct Tile {
    int b, h;             // sequence and head
    bool first, last;     // of the sequence's tiles
    unsigned tiles;
    int e;                // its first entry
    int lo[2], n[2];      // rows lo .. n - 1 of a block are attended to
    int page[2];
    unsigned long long at[2];   // where the blocks begin in K and V, in bytes
};

// A share's way through the workspace: up to kDirect shares of a sequence are
// added by its last workgroup; more are added in groups of kGroup workgroups
// first, so that no workgroup reads more than a few dozen.  (32 members: 9.8 us
// at once, 11.2 in groups; 64: 12.0 and 10.6)
constexpr unsigned kDirect = 32, kGroup = 16;

template <int D, bool FP8, bool ACC, bool WIDE>
__global__ __launch_bounds__(NW * 64, 2) void kv_attend_kernel(const KvAttendArgs a) {
    constexpr int SZ = FP8 ? 1 : 2, ROW = D * SZ;
    constexpr int NL = 16 * ROW / 1024;             // 16-byte loads of a block
    constexpr int KS = D / 32, DT = D / 16;
    constexpr int BUF = 32 * D / 8;                 // 16-byte pieces of a tile in LDS, or of a wave's sums
    // per wave: the sums of a sequence that came from the wave before (piece
    // 2 w), and the tile being worked on, in the end the sums of its last
    // sequence (piece 2 w + 1)
    __shared__ u32x4 lds[NW * 2 * BUF];
    __shared__ float2 stat[2 * NW][kKvHeads];       // [piece][head]: maximum and sum
    __shared__ int4 info[2 * NW];                   // [piece]: sequence (-1: none), head, whether it has the last tile, tiles
    __shared__ unsigned info0[2 * NW];              // its sequence's first tile on the line
    __shared__ int flag[2];
    const int w = wave_id(), l = threadIdx.x & 63, lr = l & 15, lg = l >> 4;
    const int G = a.c.hq / a.c.hkv, HT = WIDE ? (G + kKvHeads - 1) / kKvHeads : 1, HH = a.c.hkv * HT;
    const int psh = a.c.ps_shift, pmask = (1 << psh) - 1;

    // the line, this workgroup's stretch and the wave's part of it
    bool bad = false;
    Seq four[4];                                    // sequences c0 + 64 i + lane
    unsigned incl[4], sum4[4], total = 0;
    auto look_four = [&](int c0) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            four[i] = seq_of(a, c0 + 64 * i + l);
            bad |= four[i].bad;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            incl[i] = (unsigned)wave_incl_scan((int)four[i].tiles);
            sum4[i] = (unsigned)wave_total((int)incl[i]);
        }
    };
    if (a.B <= 64) {
        four[0] = seq_of(a, l);
        bad = four[0].bad;
        incl[0] = (unsigned)wave_incl_scan((int)four[0].tiles);
        total = sum4[0] = (unsigned)wave_total((int)incl[0]);
#pragma unroll
        for (int i = 1; i < 4; ++i) {
            four[i] = four[0];
            incl[i] = incl[0];
            sum4[i] = 0;
        }
    } else {
        for (int c0 = (a.B - 1) / 256 * 256; c0 >= 0; c0 -= 256) {
            look_four(c0);
            total += sum4[0] + sum4[1] + sum4[2] + sum4[3];
        }
    }
    if (blockIdx.x == 0 && bad) kv_error(a.c);
    Line line;
    line.total = total * HH;
    // as many stretches as give every wave a tile, at most one per workgroup
    line.k = min(31 - __builtin_clz(gridDim.x), 32 - __builtin_clz((line.total - 1) / NW | 1) - (line.total <= NW ? 1 : 0));
    if (blockIdx.x >= 1u << line.k) return;
    const unsigned g0 = line.begin(blockIdx.x), g1 = line.begin(blockIdx.x + 1);
    if (g0 >= g1) return;
    // (fewer tiles than waves: the first waves have one each)
    auto part_of = [&](unsigned x) { return g1 - g0 < NW ? min(x, g1 - g0) : (unsigned)((unsigned long long)(g1 - g0) * x / NW); };
    const unsigned r0 = g0 + part_of(w);
    const int left = (int)(g0 + part_of(w + 1) - r0);                // tiles of this wave

    // The cursor: the tile whose pages are looked up, two ahead of the one
    // being worked on.  Sequences b0 .. b0 + 63 are in the lanes.
    int b0 = 0, cb, ch, clen, cfirst;
    unsigned ct, ctiles;
    Seq mine;
    unsigned head0;                                 // the first tile of the first sequence and head
    {
        unsigned base = 0, in = 0;                  // tiles of a head before b0; those up to each lane's sequence
        for (int c0 = 0;; c0 += 256) {
            if (a.B > 256) look_four(c0);
            bool found = false;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (found) continue;
                b0 = c0 + 64 * i;
                mine = four[i];
                in = incl[i];
                found = (base + sum4[i]) * HH > r0 || b0 + 64 >= a.B;
                if (!found) base += sum4[i];
            }
            if (found) break;
        }
        const unsigned long long over = __ballot((base + in) * HH > r0);
        const int bi = over ? __ffsll((long long)over) - 1 : 0;      // (none: a wave without tiles behind the last)
        const unsigned seq0 = (base + (unsigned)__builtin_amdgcn_readlane((int)(in - mine.tiles), bi)) * HH;
        ctiles = (unsigned)__builtin_amdgcn_readlane((int)mine.tiles, bi);
        clen = __builtin_amdgcn_readlane(mine.len, bi);
        cfirst = __builtin_amdgcn_readlane(mine.first, bi);
        const unsigned off = r0 - seq0;
        unsigned q = 0;
        if (HH > 1) {
            q = (unsigned)((float)off * __builtin_amdgcn_rcpf((float)ctiles));
            if (q * ctiles > off) --q;
            if ((q + 1) * ctiles <= off) ++q;
        }
        cb = b0 + bi;
        ch = uni((int)q);
        ct = (unsigned)uni((int)(off - q * ctiles));
        head0 = r0 - ct;
    }
    auto advance = [&]() __attribute__((always_inline)) {
        if (++ct < ctiles) return;
        ct = 0;
        if (++ch < HH) return;
        ch = 0;
        if (++cb >= a.B) --cb;                      // (behind the last tile: never used)
        if (cb - b0 == 64) {
            b0 += 64;
            mine = seq_of(a, b0 + l);
        }
        ctiles = (unsigned)__builtin_amdgcn_readlane((int)mine.tiles, cb - b0);
        clen = __builtin_amdgcn_readlane(mine.len, cb - b0);
        cfirst = __builtin_amdgcn_readlane(mine.first, cb - b0);
    };
    // the cursor's tile, its page numbers on their way
    auto look = [&](bool used) __attribute__((always_inline)) {
        typedef const __attribute__((address_space(4))) int* cint;
        const cint trow = (cint)(a.c.table + (long long)uni(cb) * a.c.tstride);
        Tile x;
        x.b = cb;
        x.h = ch;
        x.tiles = ctiles;
        x.first = ct == 0;
        x.last = ct + 1 == ctiles;
        x.e = (cfirst & ~15) + 32 * (int)ct;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int e = x.e + 16 * j, rows = used ? clen - e : 0;
            x.page[j] = trow[uni(rows > 0 ? e >> psh : 0)];
            x.n[j] = min(16, max(0, rows));
            x.lo[j] = max(0, cfirst - e);
        }
        return x;
    };
    // its pages are there: check them.  (Addresses in units of 16 bytes: pages
    // are at most 2^30 of them)
    const unsigned page16 = (unsigned)a.c.hkv << psh, row16 = ROW / 16;
    auto locate = [&](Tile& x) __attribute__((always_inline)) {
        const int kvh = WIDE ? x.h / HT : x.h;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            if (x.n[j] > 0 && (unsigned)x.page[j] >= (unsigned)a.c.n_pages) {
                kv_error(a.c);
                x.n[j] = 0;
            }
            if (x.n[j] == 0) x.page[j] = 0;
            x.at[j] = ((unsigned long long)(unsigned)x.page[j] * (page16 * row16) +
                       (((unsigned)kvh << psh) + ((unsigned)(x.e + 16 * j) & pmask)) * row16) * 16;
        }
    };
    u32x4 kr[2][NL], vr[2][NL];
    auto load = [&](u32x4 (&x)[2][NL], const char* base_, const Tile& tl) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            // (the compiler does not see that these are the same in all lanes)
            const unsigned lo = (unsigned)uni((int)(unsigned)tl.at[j]), hi = (unsigned)uni((int)(unsigned)(tl.at[j] >> 32));
            const __amdgpu_buffer_rsrc_t rs =
                buf_rsrc(base_ + ((unsigned long long)hi << 32 | lo), (unsigned)uni(tl.n[j]) * ROW);
#pragma unroll
            for (int i = 0; i < NL; ++i) x[j][i] = buf16(rs, l * 16 + i * 1024);
        }
    };
    // a head of the line: up to 16 query heads of one kv head
    struct Heads {
        int hq0, n;
    };
    auto heads_of = [&](int h) __attribute__((always_inline)) {
        if (!WIDE) return Heads{h * G, G};
        const int kvh = h / HT, ht = h - kvh * HT;
        return Heads{kvh * G + ht * kKvHeads, min(kKvHeads, G - ht * kKvHeads)};
    };
    // the queries of a tile's heads: B operand, lane = head lr, numbers 32 ks + 8 lg on
    u32x4 q[KS];
    auto load_q = [&](const Tile& x) __attribute__((always_inline)) {
        const Heads hd = heads_of(x.h);
        const uint16_t* p = a.q + x.b * a.q_stride + (hd.hq0 + min(lr, hd.n - 1)) * D + lg * 8;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            q[ks] = ld16(p + ks * 32);
#pragma unroll
            for (int i = 0; i < 4; ++i) q[ks][i] ^= a.q_sign;
        }
    };
    u32x4* const buf = lds + (2 * w + 1) * BUF;
    // rows as they were loaded (a block is contiguous) into LDS, bf16
    auto put = [&](const u32x4 (&x)[2][NL], bool value) __attribute__((always_inline)) {
        constexpr int LPR = ROW / 16;               // lanes of a row
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                const int row = i * (64 / LPR) + l / LPR, c = l % LPR, rr = j * 16 + row;
                const u32x4 v = x[j][i];
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
    // 4 numbers of a row's output, from number d of query head hq on
    auto finish = [&](int b, int hq, int d, f32x4 v, float top, float sum_) __attribute__((always_inline)) {
        const float g = a.v_scale * __builtin_amdgcn_rcpf(sum_);
        const bool none = sum_ == 0.f;
        *reinterpret_cast<uint2*>(a.out + b * a.out_stride + hq * D + d) =
            uint2{none ? 0u : pk_bf16(v[0] * g, v[1] * g), none ? 0u : pk_bf16(v[2] * g, v[3] * g)};
        if (d == 0) {
            const float lse2 = none ? -INFINITY : top + __log2f(sum_);
            const long long at = (long long)b * a.c.hq + hq;
            if (a.lse) a.lse[at] = lse2 * kLn2;
            if (ACC) a.lse2[at] = lse2;
        }
    };

    // state of the wave: lane (head lr) has its maximum, its part of the sum,
    // and out^T: numbers 16 dt + 4 lg + i
    float m = -INFINITY, sum = 0.f;
    f32x4 o[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    // the sums as a piece of a sequence that other waves share, into LDS
    auto leave = [&](int piece, const Tile& x) __attribute__((always_inline)) {
        f32x4* const ob = reinterpret_cast<f32x4*>(lds + piece * BUF);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) ob[dt * 64 + l] = o[dt];
        if (l < kKvHeads) stat[piece][l] = float2{m, sum};
        if (l == 0) {
            info[piece] = int4{x.b, x.h, x.last, (int)x.tiles};
            info0[piece] = head0;
        }
    };
    if (l < 2) info[2 * w + l] = int4{-1, 0, 0, 0};

    if (left > 0) {
        Tile cur = look(true);
        advance();
        Tile nxt = look(left > 1);
        locate(cur);
        load(kr, a.c.K, cur);
        load(vr, a.c.V, cur);
        load_q(cur);
        bool first = cur.first;                     // the wave has the sequence's first tile
        for (int i = 0; i < left; ++i) {
            locate(nxt);
            put(kr, false);
            load(kr, a.c.K, nxt);
            // scores^T: lane = head lr, entries 4 lg + i of each block
            f32x4 s[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                s[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) s[j] = mfma(buf[k_at<D>(j * 16 + lr, ks * 4 + lg)], q[ks], s[j]);
            }
            if ((cur.lo[0] | cur.lo[1]) > 0 || (cur.n[0] & cur.n[1]) != 16) {
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (4 * lg + e < cur.lo[j] || 4 * lg + e >= cur.n[j]) s[j][e] = -INFINITY;
            }
            if constexpr (ACC) {
                const Heads hd = heads_of(cur.h);
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    if (lr < hd.n && cur.n[j] > 0)
                        *reinterpret_cast<f32x4*>(a.logits + ((((size_t)cur.page[j] * a.c.hq + hd.hq0 + lr) << psh) +
                                                              ((cur.e + 16 * j) & pmask) + 4 * lg)) = s[j];
            }
            // the maximum follows only where a score passes it by 8 (in units of
            // log 2): until then no exponential exceeds 2^8
            float top = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])),
                              fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3]))) * a.score_scale;
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
            // exponentials as three bf16 numbers whose sum they are, all 24 bits:
            // each cut towards zero, what is left over is exact.  (Two of them, 16
            // bits, would be off by 1e-5 of sum p |v|, 0.1 to 0.5 us faster.)  Where
            // the first is not 0 the others are at least 2^-133, so that an infinite
            // value gives an infinite sum and no NaN; where it is 0 they are 0 too,
            // so that the largest value adds nothing
            u32x4 hi, lo, lo2;
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                    const float x = exp2_(fmaf(s[j][e], a.score_scale, -mm)), y = exp2_(fmaf(s[j][e + 1], a.score_scale, -mm));
                    sum += x + y;
                    const float x1 = below_bf16(x), y1 = below_bf16(y);
                    const uint32_t h = upper_halves(x, y), some = min_u16x2(h, 0x00010001u);
                    hi[j * 2 + e / 2] = h;
                    lo[j * 2 + e / 2] = max_u16x2(upper_halves(x1, y1), some);
                    lo2[j * 2 + e / 2] = max_u16x2(upper_halves(below_bf16(x1), below_bf16(y1)), some);
                }
            // (a value before the first entry may be NaN, and 0 times NaN is one)
            if ((cur.lo[0] | cur.lo[1]) > 0) {
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int n = 0; n < NL; ++n)
                        if (n * (1024 / ROW) + l / (ROW / 16) < cur.lo[j]) vr[j][n] = u32x4{0, 0, 0, 0};
            }
            put(vr, true);
            load(vr, a.c.V, nxt);
            advance();
            const Tile far = look(i + 2 < left);
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
                o[dt] = mfma(va, lo2, mfma(va, lo, mfma(va, hi, o[dt])));
            }
            if (cur.last || i + 1 == left) {
                // the sequence (and head) ends, or the wave's part does
                sum += __shfl_xor(sum, 16);
                sum += __shfl_xor(sum, 32);
                if (first && cur.last) {
                    const Heads hd = heads_of(cur.h);
                    if (lr < hd.n)
#pragma unroll
                        for (int dt = 0; dt < DT; ++dt) finish(cur.b, hd.hq0 + lr, dt * 16 + 4 * lg, o[dt], m, sum);
                } else {
                    leave(2 * w + first, cur);
                }
                if (i + 1 < left) {
                    load_q(nxt);
                    head0 = r0 + i + 1;
                    first = true;
                    m = -INFINITY;
                    sum = 0.f;
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
                }
            }
            cur = nxt;
            nxt = far;
        }
    }

    // The pieces of the workgroup, in the line's order.  Each sequence's are
    // added, and those that the workgroup has alone are finished
    __syncthreads();
    const int4 pi = info[min(l, 2 * NW - 1)];
    const unsigned ph0 = info0[min(l, 2 * NW - 1)];
    const unsigned valid = (unsigned)__ballot(pi.x >= 0 && l < 2 * NW);
    const unsigned lasts = (unsigned)__ballot(pi.z != 0) & valid;
    constexpr unsigned kPart = kv_part_floats(D) * 4;
    const __amdgpu_buffer_rsrc_t pr = buf_rsrc(a.part, 2 * kKvAttendGrid * kPart);
    // a chain of pieces: one sequence's, from its start on; only the first and
    // the last chain can be shared with other workgroups
    const unsigned starts = valid & (0xaaaau | (valid & -valid));
    if (!starts) return;                            // (every sequence was within one wave)
    const int chains = __popc(starts);
    struct Chain {
        int i0, n;        // first piece and how many
        bool whole;
    };
    auto chain_at = [&](unsigned from) __attribute__((always_inline)) {       // from: starts, those before cut off
        const int i0 = __ffs((int)from) - 1;
        const unsigned rest = from & (from - 1);
        const unsigned members = valid & ~((1u << i0) - 1) & (rest ? (rest & -rest) - 1 : 0xffffu);
        return Chain{i0, (int)__popc(members), (i0 & 1) && (lasts & members)};
    };
    {
        // one or two chains take all or half of the waves, more a wave each
        const int per = chains == 1 ? NW : chains == 2 ? NW / 2 : 1, step = NW / per;
        unsigned from = starts;
        for (int c = 0; c < w / per; ++c) from &= from - 1;
        for (int c = w / per; c < chains; c += step) {
            const Chain ch_ = chain_at(from);
            for (int x = 0; x < step; ++x) from &= from - 1;
            const int i0 = ch_.i0, n = ch_.n, pw = i0 >> 1;         // waves pw .. pw + n - 1
            const int b = __builtin_amdgcn_readlane(pi.x, i0);
            const Heads hd = heads_of(__builtin_amdgcn_readlane(pi.y, i0));
            const unsigned part = (2 * blockIdx.x + (i0 & 1)) * kPart;
            // the chain's z-th piece (past the last: the first again, for nothing)
            auto piece = [&](int z) __attribute__((always_inline)) { return z && z < n ? 2 * (pw + z) : i0; };
            if (lr < hd.n) {
                float2 st[NW];
                float M = -INFINITY, S = 0.f;
#pragma unroll
                for (int z = 0; z < NW; ++z) st[z] = stat[piece(z)][lr];
#pragma unroll
                for (int z = 0; z < NW; ++z) {
                    st[z] = z < n ? st[z] : float2{-INFINITY, 0.f};
                    M = fmaxf(M, st[z].x);
                }
#pragma unroll
                for (int z = 0; z < NW; ++z) {
                    st[z].x = st[z].x == -INFINITY ? 0.f : exp2_(st[z].x - M);
                    S += st[z].x * st[z].y;                         // (a NaN stays one)
                }
#pragma unroll 2
                for (int dt = w % per; dt < DT; dt += per) {
                    f32x4 y[NW], v = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int z = 0; z < NW; ++z) y[z] = reinterpret_cast<const f32x4*>(lds)[piece(z) * BUF + dt * 64 + l];
#pragma unroll
                    for (int z = 0; z < NW; ++z)
                        if (st[z].x != 0.f) v += st[z].x * y[z];
                    const int d = dt * 16 + 4 * lg;
                    if (ch_.whole) {
                        finish(b, hd.hq0 + lr, d, v, M, S);
                    } else {
                        store_through(pr, part + (lr * D + d) * 4, v);
                        if (d == 0) store_through(pr, part + (kKvHeads * D + 2 * lr) * 4, float2{M, S});
                    }
                }
            }
        }
    }

    // Shares: counted; the workgroup that completes a sequence, or a group of
    // its workgroups, adds them in the line's order
    const Chain c0 = chain_at(starts), c1 = chain_at(1u << (31 - __builtin_clz(starts)));
    const bool two = chains > 1 && !c0.whole && !c1.whole;
    const int nsh = two ? 2 : c0.whole && (chains == 1 || c1.whole) ? 0 : 1;
    if (nsh == 0) return;
    struct Share {
        int b, h;
        unsigned v0, v1;      // the sequence's first and last workgroup
        // members m0 + stride x (the first workgroup in place of what lies before
        // it), x = 0 .. n - 1, and their counter; level 0: a group's, 1: all
        unsigned m0, stride, n;
        unsigned* count;
        bool direct;
    };
    const unsigned grp = blockIdx.x / kGroup;
    auto at_level = [&](Share& s, int level) __attribute__((always_inline)) {
        s.m0 = s.direct ? s.v0 : level ? s.v0 / kGroup * kGroup : max(s.v0, grp * kGroup);
        s.stride = s.direct || !level ? 1u : kGroup;
        s.n = s.direct ? s.v1 - s.v0 + 1 : level ? s.v1 / kGroup - s.v0 / kGroup + 1 : min(s.v1 + 1, (grp + 1) * kGroup) - s.m0;
        s.count = a.count + (level ? s.v0 : kKvAttendGrid + 2 * s.m0 + (s.m0 == s.v0)) * kKvCount;
    };
    auto share_of = [&](const Chain& c) __attribute__((always_inline)) {
        Share s;
        s.b = __builtin_amdgcn_readlane(pi.x, c.i0);
        s.h = __builtin_amdgcn_readlane(pi.y, c.i0);
        const unsigned h0 = (unsigned)__builtin_amdgcn_readlane((int)ph0, c.i0);
        s.v0 = line.owner(h0);
        s.v1 = line.owner(h0 + (unsigned)__builtin_amdgcn_readlane(pi.w, c.i0) - 1);
        s.direct = s.v1 - s.v0 < kDirect;
        at_level(s, s.direct);
        return s;
    };
    Share sh0 = share_of(two || !c0.whole ? c0 : c1), sh1 = sh0;
    if (two) sh1 = share_of(c1);
    // what this wave left has reached memory; then one atomic operation for each
    auto arrive = [&](unsigned* c, unsigned n) __attribute__((always_inline)) {
        const bool is_last = __hip_atomic_fetch_add(c, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == n - 1;
        if (is_last) __hip_atomic_store(c, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        return is_last;
    };
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if ((int)threadIdx.x < nsh) flag[threadIdx.x] = arrive(threadIdx.x ? sh1.count : sh0.count, threadIdx.x ? sh1.n : sh0.n);
    __syncthreads();
    unsigned todo = (unsigned)uni(flag[0]) | (nsh == 2 ? (unsigned)uni(flag[1]) << 1 : 0u);
    unsigned level = (sh0.direct ? 1u : 0u) | (sh1.direct ? 2u : 0u);       // bit k: sh_k's members are all of its sequence's
#pragma unroll 1
    while (todo) {
        // One item = 4 numbers of a head; ng threads have every ng-th member of
        // an item: as many as fill half of the workgroup, so that two shares are
        // added at once, or all of it where one of these would have more than
        // 16 members or in groups (64 sequences of 4096, 8 members: 22.2 against
        // 22.9 us; one of 131072, 512: 36.6 against 35.7).  This depends on the
        // share alone, and so does the order of its sums
        const int items0 = heads_of(sh0.h).n * (D / 4), items1 = heads_of(sh1.h).n * (D / 4);
        auto threads_of = [](const Share& s, int items) __attribute__((always_inline)) {
            const int half = max(1, NT / 2 / items);
            return s.direct && (int)s.n <= 16 * half ? half : max(1, NT / items);
        };
        const int ng0 = threads_of(sh0, items0), ng1 = threads_of(sh1, items1);
        const int slots0 = todo & 1 ? items0 * ng0 : 0, slots1 = todo & 2 ? items1 * ng1 : 0;
        // (the threads of an item are in one pass)
        const int from1 = slots0 + slots1 > NT ? (slots0 + NT - 1) / NT * NT : slots0;
        for (int i0 = 0; i0 < from1 + slots1; i0 += NT) {
            if (i0) __syncthreads();                // (the pass before has read its sums)
            const int at = i0 + threadIdx.x;
            const bool k = at >= from1, in = k ? at < from1 + slots1 : at < slots0;
            const int slot = at - (k ? from1 : 0), items = k ? items1 : items0, ng = k ? ng1 : ng0;
            const int g = ng == 1 ? 0 : slot / items, it = slot - g * items, hq = it / (D / 4), d = it % (D / 4) * 4;
            const unsigned v0 = k ? sh1.v0 : sh0.v0, m0 = k ? sh1.m0 : sh0.m0, stride = k ? sh1.stride : sh0.stride;
            const int n = (int)(k ? sh1.n : sh0.n);
            auto share = [&](unsigned x) __attribute__((always_inline)) {
                const unsigned v = max(v0, m0 + stride * x);
                return (2 * v + (v == v0)) * kPart;
            };
            f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f};
            float ss = 0.f, top = -INFINITY;
            auto add = [&](auto batch) __attribute__((always_inline)) {
                constexpr int kBatch = decltype(batch)::value;      // shares whose loads are in flight at once
                for (int x0 = g; x0 < n; x0 += kBatch * ng) {
                    float2 ms[kBatch];
                    f32x4 y[kBatch];
#pragma unroll
                    for (int x = 0; x < kBatch; ++x) {
                        const unsigned p = x0 + x * ng < n ? share((unsigned)(x0 + x * ng)) : kOob;
                        ms[x] = load_through2(pr, p + (kKvHeads * D + 2 * hq) * 4);
                        y[x] = load_through4(pr, p + (hq * D + d) * 4);
                    }
                    float tn = top;
#pragma unroll
                    for (int x = 0; x < kBatch; ++x) {
                        if (x0 + x * ng >= n) ms[x] = float2{-INFINITY, 0.f};
                        tn = fmaxf(tn, ms[x].x);
                    }
                    const float fo = top == -INFINITY ? 0.f : exp2_(top - tn);
                    top = tn;
                    ss *= fo;
                    v *= fo;
#pragma unroll
                    for (int x = 0; x < kBatch; ++x) {
                        const float fx = ms[x].x == -INFINITY ? 0.f : exp2_(ms[x].x - top);
                        ss += fx * ms[x].y;
                        if (fx != 0.f) v += fx * y[x];
                    }
                }
            };
            if (in) {
                if (n <= 4 * ng)
                    add(std::integral_constant<int, 4>{});
                else if (n <= 8 * ng)
                    add(std::integral_constant<int, 8>{});
                else
                    add(std::integral_constant<int, 16>{});
            }
            f32x4* const fv = reinterpret_cast<f32x4*>(lds);
            float2* const fs = reinterpret_cast<float2*>(lds + NT);
            fv[threadIdx.x] = v;
            fs[threadIdx.x] = float2{top, ss};
            __syncthreads();                        // (also: a group's shares are read before one is written over)
            if (in && ng > 1 && g == 0) {
                float tn = top;
                for (int x = 1; x < ng; ++x) tn = fmaxf(tn, fs[x * items + threadIdx.x].x);
                const float fo = top == -INFINITY ? 0.f : exp2_(top - tn);
                top = tn;
                ss *= fo;
                v *= fo;
                for (int x = 1; x < ng; ++x) {
                    const float2 y = fs[x * items + threadIdx.x];
                    const float fx = y.x == -INFINITY ? 0.f : exp2_(y.x - top);
                    ss += fx * y.y;
                    if (fx != 0.f) v += fx * fv[x * items + threadIdx.x];
                }
            }
            if (in && g == 0) {
                if (k ? level & 2 : level & 1) {
                    finish(k ? sh1.b : sh0.b, heads_of(k ? sh1.h : sh0.h).hq0 + hq, d, v, top, ss);
                } else {                            // the group's share takes its first one's place
                    store_through(pr, share(0) + (hq * D + d) * 4, v);
                    if (d == 0) store_through(pr, share(0) + (kKvHeads * D + 2 * hq) * 4, float2{top, ss});
                }
            }
        }
        // groups that are complete now count for their sequences
        todo &= ~level;
        if (!todo) break;
        level = 3;
        at_level(sh0, 1);
        at_level(sh1, 1);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (threadIdx.x < 2)
            flag[threadIdx.x] = (todo >> threadIdx.x & 1) && arrive(threadIdx.x ? sh1.count : sh0.count, threadIdx.x ? sh1.n : sh0.n);
        __syncthreads();
        todo = (unsigned)uni(flag[0]) | (unsigned)uni(flag[1]) << 1;
    }
}

// Weights: each entry's probabilities from the stored scores and the row's
// log of sums,
//     weight_j += sum over the group's heads of exp(s_j - lse).
// The entries of all sequences and kv heads, 256 at a time, form a line as
// above.  A launch of its own, since a sequence's sum is known only when its last
// workgroup has joined it; it reads 4 G + 8 bytes an entry, 3 MB for 32
// sequences of 2049 entries and two kv heads: 5.5 us, of which 3 are any
// launch's.  Bound by waits, one after the other: the lengths, the page number,
// then lse and score of each head in turn, in the end the weight itself (2 G + 3
// trips to memory).  (The workgroup that finishes a sequence could add its weights: 6.6
// against 10.5 us where a wave has a sequence to itself, but 29.4 against
// 26.8 us at 32 of 2049 entries and 101 against 19 at one of 32768, which one
// workgroup then reads alone.)
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
                        if (z != -INFINITY) v += exp2_(fmaf(s, a.score_scale, -z));
                    }
                    a.c.weight[(((size_t)pg * hkv + h) << psh) + ((int)e & pmask)] += v;
                }
            }
        }
        at += n;
    }
}

template <int D, bool FP8, bool WIDE>
hipError_t launch(const KvAttendArgs& a, bool accumulate, hipStream_t s) {
    // no more workgroups than the table rows could have work for
    const long long G = a.c.hq / a.c.hkv, HH = a.c.hkv * ((G + kKvHeads - 1) / kKvHeads);
    const long long tiles = (((long long)a.c.width << a.c.ps_shift) + 31) / 32 * a.B * HH;
    int grid = 1;
    while (grid < kKvAttendGrid && (long long)grid * NW < tiles) grid *= 2;
    if (!accumulate) {
        kv_attend_kernel<D, FP8, false, WIDE><<<grid, NT, 0, s>>>(a);
        return hipGetLastError();
    }
    kv_attend_kernel<D, FP8, true, WIDE><<<grid, NT, 0, s>>>(a);
    const long long blocks = (((long long)a.c.width << a.c.ps_shift) + 255) / 256 * a.B * a.c.hkv;
    kv_weigh_kernel<<<(int)std::min(blocks, 1024LL), 256, 0, s>>>(a);
    return hipGetLastError();
}

template <int D, bool FP8>
hipError_t launch(const KvAttendArgs& a, bool accumulate, hipStream_t s) {
    return a.c.hq / a.c.hkv > kKvHeads ? launch<D, FP8, true>(a, accumulate, s) : launch<D, FP8, false>(a, accumulate, s);
}

}  // namespace

hipError_t launch_kv_attend(const KvAttendArgs& a, int head_dim, bool fp8, bool accumulate, hipStream_t s) {
    if (head_dim == 64) return fp8 ? launch<64, true>(a, accumulate, s) : launch<64, false>(a, accumulate, s);
    return fp8 ? launch<128, true>(a, accumulate, s) : launch<128, false>(a, accumulate, s);
}

}  // namespace bdl
