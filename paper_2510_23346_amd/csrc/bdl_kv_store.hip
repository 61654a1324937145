// Key-value cache in 8-bit integers with a scale for each block of 16 entries
// of a head: append, and reading any cache back (gfx950, wave64).
#include "bdl_kv_device.h"

namespace bdl {

namespace {

// ------------------------------------------------------------------ append
// A block's scale is that of its largest magnitude so far:
//
//     m = max(|x| over the call's rows of the block, 2^-64),  s = m / 127,
//
// or max(s, the scale before) where the block's first entry is not among the
// call's; x is stored as rint(x / s).  Where the scale grows, the entries that
// were there are rounded again, rint(q s_before / s).  (m / 127 and x / s are
// products with the fp32 reciprocals.)  So a block has one owner: the wave of
// the first token of its run, tokens of one sequence that follow each other in
// the call and, with gaps or without, in the block.  It has all 16 rows of the block,
// those that are new in registers, four lanes a row; its other tokens' waves leave.
//
// Tokens of a block that do not stand so have owners that know nothing of each other,
// and what the block holds is anything.  That is found out: an owner leaves its token's
// number at the block's place in a.owners and takes the one it finds there, which is
// an earlier call's, anything at all, or another owner's.  So it looks whether that
// token, now, is of its block and not of its run.  (A cache of more blocks than there
// are places, 3.2 million at head size 128, shares them, and an owner may not be found.)
//
// Rotation and norm are those of the bf16 cache, and queries are dealt with by
// threads of the same launch as there.
//
// Bound by the trips to memory of an owner (which token, its run and page, then the
// block and the angles) and the waves that find they are none: 4288 tokens of 8 + 1 + 1
// heads of 128, 22 MB read and written, 11.3 to 12.6 us, where the bf16 cache's launch
// takes 8.5; 10240 tokens of 32 + 8 + 8 heads, 235 MB, 76 us, 3.1 TB/s.
template <int N>
struct Piece {
    float x[N];
};

// N numbers of a row
template <int N>
__device__ __forceinline__ Piece<N> load_piece(const uint16_t* p) {
    Piece<N> r;
#pragma unroll
    for (int k = 0; k < N; k += 8) {
        float y[8];
        unpack8(ld16(p + k), y);
#pragma unroll
        for (int i = 0; i < 8; ++i) r.x[k + i] = y[i];
    }
    return r;
}

template <int N>
__device__ __forceinline__ Piece<N> load_piece(const float* p) {
    Piece<N> r;
#pragma unroll
    for (int k = 0; k < N; k += 4) {
        const float4 v = *reinterpret_cast<const float4*>(p + k);
        r.x[k] = v.x, r.x[k + 1] = v.y, r.x[k + 2] = v.z, r.x[k + 3] = v.w;
    }
    return r;
}

// four numbers to the nearest integers, within +-127 (NaN: any of them)
__device__ __forceinline__ uint32_t pack4_int8(const float* x, float f) {
    uint32_t r = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        r |= ((uint32_t)(int)__builtin_amdgcn_fmed3f(rintf(x[k] * f), -127.f, 127.f) & 255u) << (8 * k);
    return r;
}

template <int N>
__device__ __forceinline__ void unpack_int8(const uint32_t (&w)[N / 4], Piece<N>& r) {
#pragma unroll
    for (int k = 0; k < N; ++k) r.x[k] = (float)(int8_t)(w[k / 4] >> (8 * (k % 4)));
}

constexpr float kLeast = 5.421010862427522e-20f;     // 2^-64

// One block: that of token t, entry i0 of row seq (which there is), and of the tokens
// of its run behind it
template <int D, bool NORM>
__device__ __forceinline__ void store_block(const KvAppendArgs& a, int t, int seq, int i0, int kh, bool value) {
#pragma clang fp contract(off)
    constexpr int N = D / 8;
    const int l = threadIdx.x & 63, r = l >> 2, c = l & 3;
    // (two trips to memory: the page, the run and its rows; what the block holds and
    // the angles)
    const int j = r - (i0 & (kKvBlock - 1)), d0 = N * c, d1 = D / 2 + N * c;
    int tok = min(t + max(j, 0), a.T - 1);
    const int page = a.c.table[(long long)seq * a.c.tstride + (i0 >> a.c.ps_shift)];
    const int seq_r = a.seqs[tok], index_r = a.index[tok];
    int pos_r = a.positions[tok];
    const uint16_t* const x = a.qkv + (a.c.hq + (value ? a.c.hkv : 0) + kh) * D;
    Piece<N> y0 = load_piece<N>(x + tok * a.qkv_stride + d0), y1 = load_piece<N>(x + tok * a.qkv_stride + d1);
    if ((unsigned)page >= (unsigned)a.c.n_pages) {
        kv_error(a.c);
        return;
    }
    const long long e0 = (((long long)page * a.c.hkv + kh) << a.c.ps_shift) + (i0 & ((1 << a.c.ps_shift) - 1) & ~(kKvBlock - 1));
    // the lane's token, if the run goes as far: it is the row's where there are no gaps
    const int index_1 = __shfl_up(index_r, 4);
    const bool follows = j >= 0 && j < a.T - t && seq_r == seq && (index_r >> 4) == (i0 >> 4) && (j == 0 || index_r > index_1);
    const unsigned long long breaks = __ballot(j >= 0 && !follows);
    bool has = follows && (breaks == 0 || l < (int)__builtin_ctzll(breaks));
    const unsigned long long run = __ballot(has);
    const int tokens = __popcll(run) >> 2;
    if (__any(has && index_r != i0 + j)) {
        // a run with gaps: each row looks for its token
        has = false;
#pragma unroll 1
        for (int k = i0 & (kKvBlock - 1); k < kKvBlock; ++k)
            if ((run >> (4 * k) & 1) && (__builtin_amdgcn_readlane(index_r, 4 * k) & (kKvBlock - 1)) == r) {
                has = true;
                tok = t + k - (i0 & (kKvBlock - 1));
            }
        pos_r = a.positions[tok];
        y0 = load_piece<N>(x + tok * a.qkv_stride + d0);
        y1 = load_piece<N>(x + tok * a.qkv_stride + d1);
    }
    const bool asks = kh == 0 && value && l == 0;
    int other = -1;
    if (asks)
        other = atomicExch(a.owners + (unsigned)((((unsigned long long)(unsigned)page << a.c.ps_shift) +
                                                  (unsigned)(i0 & ((1 << a.c.ps_shift) - 1))) >> 4) % a.n_owners, t);
    const bool mine = has && pos_r >= 0 && pos_r < a.n_positions;
    const int pos = mine ? pos_r : 0;
    const unsigned long long rows = __ballot(mine);
    if (rows == 0) return;
    const bool anew = rows & 1;
    float* const scale_at = a.c.scales + (e0 >> 4) * 2 + value;
    const float before = *scale_at;
    char* const base = (value ? a.c.V : a.c.K) + (e0 + r) * D;
    uint32_t q0[N / 4], q1[N / 4];
#pragma unroll
    for (int k = 0; k < N / 4; ++k) q0[k] = q1[k] = 0;
    if (!anew) {
#pragma unroll
        for (int k = 0; k < N / 4; ++k) {
            q0[k] = reinterpret_cast<const uint32_t*>(base + d0)[k];
            q1[k] = reinterpret_cast<const uint32_t*>(base + d1)[k];
        }
    }
    if (!value) {
        if constexpr (NORM) {
            float ss = 0.f;
#pragma unroll
            for (int k = 0; k < N; ++k) ss += y0.x[k] * y0.x[k] + y1.x[k] * y1.x[k];
            ss += __shfl_xor(ss, 1);
            ss += __shfl_xor(ss, 2);
            const float f = 1.f / sqrtf(ss * (1.f / D) + a.eps);
            const Piece<N> w0 = load_piece<N>(a.k_norm + d0), w1 = load_piece<N>(a.k_norm + d1);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                y0.x[k] = y0.x[k] * f * w0.x[k];
                y1.x[k] = y1.x[k] * f * w1.x[k];
            }
        }
        {
            const long long at = (long long)pos * (D / 2);
            if (a.interleaved) {
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    float* const y = part ? y1.x : y0.x;
                    const Piece<N / 2> cc = load_piece<N / 2>(a.cos + at + (part ? d1 : d0) / 2), ss = load_piece<N / 2>(a.sin + at + (part ? d1 : d0) / 2);
#pragma unroll
                    for (int k = 0; k < N / 2; ++k) {
                        const float u = y[2 * k], v = y[2 * k + 1];
                        y[2 * k] = u * cc.x[k] - v * ss.x[k];
                        y[2 * k + 1] = v * cc.x[k] + u * ss.x[k];
                    }
                }
            } else {
                const Piece<N> cc = load_piece<N>(a.cos + at + d0), ss = load_piece<N>(a.sin + at + d0);
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    const float u = y0.x[k], v = y1.x[k];
                    y0.x[k] = u * cc.x[k] - v * ss.x[k];
                    y1.x[k] = v * cc.x[k] + u * ss.x[k];
                }
            }
        }
    }
    // the largest magnitude, as an integer: infinities and NaN above all numbers
    unsigned top = 0;
    if (mine)
#pragma unroll
        for (int k = 0; k < N; ++k)
            top = max(top, max(__float_as_uint(y0.x[k]) & 0x7fffffffu, __float_as_uint(y1.x[k]) & 0x7fffffffu));
#pragma unroll
    for (int x = 32; x; x >>= 1) top = max(top, (unsigned)__shfl_xor((int)top, x));
    float s = top >= 0x7f800000u ? NAN : fmaxf(__uint_as_float(top), kLeast) * (1.f / 127.f);
    if (!anew) s = s != s || before != before ? NAN : fmaxf(s, before);
    if (mine) {
        const float f = 1.f / s;
#pragma unroll
        for (int k = 0; k < N / 4; ++k) {
            q0[k] = pack4_int8(y0.x + 4 * k, f);
            q1[k] = pack4_int8(y1.x + 4 * k, f);
        }
    } else if (!anew && s != before) {
        const float f = before / s;
        Piece<N> z;
        unpack_int8<N>(q0, z);
#pragma unroll
        for (int k = 0; k < N / 4; ++k) q0[k] = pack4_int8(z.x + 4 * k, f);
        unpack_int8<N>(q1, z);
#pragma unroll
        for (int k = 0; k < N / 4; ++k) q1[k] = pack4_int8(z.x + 4 * k, f);
    }
    if (mine || (!anew && s != before)) {
#pragma unroll
        for (int k = 0; k < N / 4; ++k) {
            reinterpret_cast<uint32_t*>(base + d0)[k] = q0[k];
            reinterpret_cast<uint32_t*>(base + d1)[k] = q1[k];
        }
    }
    if (l == 0) *scale_at = s;
    if (kh == 0 && value && a.lens) {
        const int last = (63 - __builtin_clzll(rows)) >> 2;
        if (l == 0) atomicMax(a.lens + seq, (i0 & ~(kKvBlock - 1)) + last + 1);
    }
    // (the run's tokens stand from t on)
    if (asks && other >= 0 && other < a.T && (other < t || other >= t + tokens) && a.seqs[other] == seq && (a.index[other] >> 4) == (i0 >> 4))
        kv_error(a.c);
}

// The first `q_groups` workgroups take `q_rows` tokens' queries each, as append does.
// A wave of the others has a head's keys or values of a token, and leaves if that is
// not the first of a block's run.  MANY: of 16 tokens, `step` (1 more than a multiple of
// 16) apart, so that runs that begin together have their firsts in different waves; each
// lane looks at one
template <int D, bool NORM, bool MANY>
__global__ __launch_bounds__(256) void kv_store_kernel(const KvAppendArgs a, int q_groups, int q_rows, int step) {
#pragma clang fp contract(off)
    if ((int)blockIdx.x >= q_groups) {
        const long long unit = (long long)(blockIdx.x - q_groups) * 4 + wave_id();
        const int per = 2 * a.c.hkv, t0 = (int)(unit / per), u = (int)(unit - (long long)t0 * per), cap = a.c.width << a.c.ps_shift;
        if (t0 >= step) return;
        const int l = threadIdx.x & 63, t = MANY ? t0 + min(l, kKvBlock - 1) * step : t0, at_t = min(t, a.T - 1), before = max(at_t - 1, 0);
        const int seq = a.seqs[at_t], at = a.index[at_t], seq1 = a.seqs[before], at1 = a.index[before];
        bool first = seq >= 0 && seq < a.n_seqs && at >= 0 && at < cap;
        if (t > 0 && seq1 == seq && (at1 >> 4) == (at >> 4) && at1 < at) first = false;
        if constexpr (MANY) {
#pragma unroll 1
            for (unsigned long long m = __ballot(first && l < kKvBlock && t < a.T); m; m &= m - 1) {
                const int x = (int)__builtin_ctzll(m);
                store_block<D, NORM>(a, t0 + x * step, __builtin_amdgcn_readlane(seq, x), __builtin_amdgcn_readlane(at, x), u >> 1, u & 1);
            }
        } else if (first) {
            store_block<D, NORM>(a, t0, seq, at, u >> 1, u & 1);
        }
        return;
    }
    constexpr int P = D / 16;
    const int units = a.c.hq * P;
    for (int i = threadIdx.x; i < units * q_rows; i += 256) {
        const int row = i / units, u = i - row * units, h = u / P, j = u % P;
        const int t = blockIdx.x * q_rows + row;
        if (t >= a.T) return;
        const int d0 = a.interleaved ? 16 * j : 8 * j, d1 = a.interleaved ? 16 * j + 8 : D / 2 + 8 * j;
        const uint16_t* x = a.qkv + t * a.qkv_stride + h * D;
        const int pos = a.positions[t];
        const bool pos_ok = pos >= 0 && pos < a.n_positions;
        float y0[8], y1[8];
        unpack8(ld16(x + d0), y0);
        unpack8(ld16(x + d1), y1);
        if (NORM) {
            const u32x4 w0 = ld16(a.q_norm + d0), w1 = ld16(a.q_norm + d1);
            head_norm<D>(y0, y1, w0, w1, a.eps);
        }
        rotate16(y0, y1, a.cos, a.sin, (long long)(pos_ok ? pos : 0) * (D / 2) + 8 * j, a.interleaved);
        if (!pos_ok)
#pragma unroll
            for (int k = 0; k < 8; ++k) y0[k] = y1[k] = 0.f;
        uint16_t* q = a.q_out + t * a.q_stride + h * D;
        *reinterpret_cast<u32x4*>(q + d0) = pack8(y0);
        *reinterpret_cast<u32x4*>(q + d1) = pack8(y1);
        if (u == 0) {
            const int seq = a.seqs[t], at = a.index[t], cap = a.c.width << a.c.ps_shift;
            if (!pos_ok || (seq != -1 && !(seq >= 0 && seq < a.n_seqs && at >= 0 && at < cap))) kv_error(a.c);
        }
    }
}

template <int D>
hipError_t store(const KvAppendArgs& a, hipStream_t s) {
    const int units = a.c.hq * (D / 16), rows = std::max(1, 256 / units);
    const long long q_groups = ((long long)a.T + rows - 1) / rows, waves = (long long)a.T * 2 * a.c.hkv;
    // 16 tokens a wave where waves for one each would wait for room, most of them to leave
    // again; not where many tokens may be the only ones of their sequences, whose blocks
    // such a wave stores one by one.  (Heads of 128, one token and 16 a wave: 8 prompts of
    // 512 of one kv head 13.4 and 10.6 us, of 1024 21.7 and 17.0; of 8 kv heads 4 of 512
    // 31 and 18, 4 of 1024 beside 192 single tokens 56 and 41, one of 10240 147 and 76, 2000
    // single tokens 60 and 83; the 4 of 1024 beside 192, of one kv head, 14.3 and 18.6)
    const bool many = (waves > 4096 && a.T >= 64LL * a.n_seqs) || (waves > 16384 && a.T >= 4LL * a.n_seqs);
    const int step = many ? ((a.T + kKvBlock - 1) / kKvBlock + kKvBlock - 2) / kKvBlock * kKvBlock + 1 : a.T;
    const long long blocks = ((long long)step * 2 * a.c.hkv + 3) / 4;
    if (q_groups + blocks >= 1 << 24) return hipErrorInvalidValue;
    auto run = [&](auto kernel) { kernel<<<(int)(q_groups + blocks), 256, 0, s>>>(a, (int)q_groups, rows, step); };
    if (a.q_norm)
        many ? run(kv_store_kernel<D, true, true>) : run(kv_store_kernel<D, true, false>);
    else
        many ? run(kv_store_kernel<D, false, true>) : run(kv_store_kernel<D, false, false>);
    return hipGetLastError();
}

// ------------------------------------------------------------------ read
// Entries as bf16: the stored number times its scale, rounded once.  A thread
// takes 8 numbers of a row (one 16-byte store, so that a wave's covers whole lines:
// 32 bytes a thread 99 us where these take 91), of R rows in turn, whose loads are
// in flight together.  Bound by its memory traffic: 293888 entries of two kv heads
// of 128, 454 MB read and written, 90 us, 5.0 TB/s (a large copy 5.2).
template <int D, int FMT, int R>
__global__ __launch_bounds__(256) void kv_read_kernel(const KvReadArgs a) {
#pragma clang fp contract(off)
    constexpr int SZ = FMT == kBf16 ? 2 : 1;
    const int u = blockIdx.y * blockDim.x + threadIdx.x, h2 = u / (D / 8), j = u % (D / 8);
    const long long t0 = (long long)blockIdx.x * blockDim.y * R + threadIdx.y;
    if (t0 >= a.T || h2 >= 2 * a.c.hkv) return;
    const bool v = h2 >= a.c.hkv;
    const int h = v ? h2 - a.c.hkv : h2, cap = a.c.width << a.c.ps_shift;
    // each step for all of the thread's rows (past the last: that one again)
    int t[R], seq[R], at[R], page[R];
    bool ok[R];
#pragma unroll
    for (int k = 0; k < R; ++k) {
        t[k] = (int)min(t0 + (long long)k * blockDim.y, (long long)a.T - 1);
        seq[k] = a.seqs[t[k]];
        at[k] = a.index[t[k]];
    }
#pragma unroll
    for (int k = 0; k < R; ++k) {
        ok[k] = seq[k] >= 0 && seq[k] < a.n_seqs && at[k] >= 0 && at[k] < cap;
        if (!ok[k] && seq[k] != -1) kv_error(a.c);
        page[k] = ok[k] ? a.c.table[(long long)seq[k] * a.c.tstride + (at[k] >> a.c.ps_shift)] : 0;
    }
    u32x4 x[R];
    float f[R];
#pragma unroll
    for (int k = 0; k < R; ++k) {
        if (ok[k] && (unsigned)page[k] >= (unsigned)a.c.n_pages) {
            kv_error(a.c);
            ok[k] = false;
        }
        const long long e = ok[k] ? (((long long)page[k] * a.c.hkv + h) << a.c.ps_shift) + (at[k] & ((1 << a.c.ps_shift) - 1)) : 0;
        const char* const p = (v ? a.c.V : a.c.K) + e * (D * SZ) + 8 * j * SZ;
        if constexpr (FMT == kBf16) {
            x[k] = *reinterpret_cast<const u32x4*>(p);
        } else {
            const uint2 w = *reinterpret_cast<const uint2*>(p);
            x[k][0] = w.x, x[k][1] = w.y;
        }
        f[k] = FMT == kInt8 ? a.c.scales[(e >> 4) * 2 + v] : v ? a.v_scale : a.k_scale;
    }
#pragma unroll
    for (int k = 0; k < R; ++k) {
        u32x4 o = x[k];
        if constexpr (FMT != kBf16) {
            float y[8];
#pragma unroll
            for (int i = 0; i < 8; i += 4) {
                const uint32_t w = x[k][i / 4];
                if constexpr (FMT == kInt8) {
#pragma unroll
                    for (int b = 0; b < 4; ++b) y[i + b] = (float)(int8_t)(w >> (8 * b));
                } else {
                    typedef float f32x2 __attribute__((ext_vector_type(2)));
                    const f32x2 p0 = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), p1 = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
                    y[i] = p0[0], y[i + 1] = p0[1], y[i + 2] = p1[0], y[i + 3] = p1[1];
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = pk_bf16(y[2 * i] * f[k], y[2 * i + 1] * f[k]);
        }
        if (!ok[k]) o = u32x4{0, 0, 0, 0};
        if (t0 + (long long)k * blockDim.y < a.T)
            *reinterpret_cast<u32x4*>((v ? a.v_out + t[k] * a.v_stride : a.k_out + t[k] * a.k_stride) + h * D + 8 * j) = o;
    }
}

template <int D, int FMT>
hipError_t read(const KvReadArgs& a, hipStream_t s) {
    const int units = 2 * a.c.hkv * (D / 8), x = std::min(units, 256), y = 256 / x;
    const dim3 block(x, y);
    auto grid = [&](int rows) { return dim3((unsigned)(((long long)a.T + y * rows - 1) / (y * rows)), (units + x - 1) / x); };
    // four rows a thread from where one each would take more than two rounds of the
    // chip's threads (2.2 million threads 14.4 against 17.4 us, 12 times as many 91 against 137)
    const bool many = (long long)a.T * units >= 256 * 2048 * 4;
    if (many)
        kv_read_kernel<D, FMT, 4><<<grid(4), block, 0, s>>>(a);
    else
        kv_read_kernel<D, FMT, 1><<<grid(1), block, 0, s>>>(a);
    return hipGetLastError();
}

template <int D>
hipError_t read(const KvReadArgs& a, bool fp8, hipStream_t s) {
    return a.c.scales ? read<D, kInt8>(a, s) : fp8 ? read<D, kFp8>(a, s) : read<D, kBf16>(a, s);
}

}  // namespace

hipError_t launch_kv_store(const KvAppendArgs& a, int head_dim, hipStream_t s) {
    return head_dim == 64 ? store<64>(a, s) : store<128>(a, s);
}

hipError_t launch_kv_read(const KvReadArgs& a, int head_dim, bool fp8, hipStream_t s) {
    return head_dim == 64 ? read<64>(a, fp8, s) : read<128>(a, fp8, s);
}

}  // namespace bdl
