// Internal interface between the C ABI's key-value cache calls and their
// kernels (gfx950).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <string>

namespace bdl {

// records the message for bdlora_last_error and returns the code
int api_fail(int code, const std::string& msg);

constexpr int kKvMaxHeads = 1024;      // query heads
constexpr int kKvMinPage = 16, kKvMaxPage = 65536;

// attend: the most workgroups of a launch, heads a workgroup takes at once,
// and what one leaves for a sequence that it shares with others: unnormalised
// sums [heads][D], then each head's maximum and sum
constexpr int kKvAttendGrid = 512, kKvHeads = 16;

// Counters lie a cache line apart (in numbers of 4 bytes): atomic operations on
// one line wait for each other, 512 of 16 sequences for 4 us.  Attention
// has one for each sequence that goes on behind the workgroup it begins in, and
// one for each group of a sequence's workgroups, of which two can begin at one.
constexpr int kKvCount = 32, kKvAttendCounts = 3 * kKvAttendGrid;
constexpr int kv_part_floats(int D) { return kKvHeads * (D + 2); }

// What every kernel knows of the cache and of the call's page table.  Pages
// are [n_pages][hkv][1 << ps_shift] entries: K and V of D elements each,
// weight and pos (null when the cache does not track weights) of one.
struct KvCache {
    char *K, *V;
    float* weight;
    int* pos;
    int hq, hkv, ps_shift, n_pages;
    const int* table;     // [rows][tstride], `width` pages of a row used
    int tstride, width;
    int* err;             // sticky error flag
};

struct KvAppendArgs {
    KvCache c;
    const uint16_t* qkv;
    long long qkv_stride, q_stride;
    uint16_t* q_out;
    const float *cos, *sin;
    int n_positions, interleaved;
    const int *seqs, *index, *positions;
    int* lens;            // may be null
    int T, n_seqs;
    float k_inv, v_inv;   // 8-bit cache: 1 / scale
};

struct KvAttendArgs {
    KvCache c;
    const uint16_t* q;
    uint16_t* out;
    long long q_stride, out_stride;
    const int *lens, *starts;
    int has_starts;             // 0: starts is there to be read, and means nothing
    float* lse;                 // may be null
    int B;
    float* part;                // [2 kKvAttendGrid][kv_part_floats(D)]
    unsigned* count;            // kKvAttendCounts counters: zero between calls
    float* logits;              // accumulating: [n_pages][hq][page], products <q, k>
    float* lse2;                // accumulating: [B][hq], lse in those units
    float score_scale;    // > 0, times the product of raw values: scores in units of log 2
    unsigned q_sign;      // a negative scale: flips the queries' signs (two bf16 each word)
    float v_scale;
};

struct KvEvictArgs {
    KvCache c;
    int* lens;
    int B, budget, recent, n_cu;
    int* scratch;         // [n_pages][hkv][page]: the places to fill and what fills them
    unsigned* count;      // B hkv counters, then B: zero between calls
};

hipError_t launch_kv_append(const KvAppendArgs& a, int head_dim, bool fp8, hipStream_t s);
hipError_t launch_kv_attend(const KvAttendArgs& a, int head_dim, bool fp8, bool accumulate, hipStream_t s);
hipError_t launch_kv_evict(const KvEvictArgs& a, int head_dim, bool fp8, hipStream_t s);

}  // namespace bdl
