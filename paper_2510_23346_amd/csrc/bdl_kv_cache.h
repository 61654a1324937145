// What the C ABI's key-value cache calls share: the cache, argument checks.
#pragma once

#include "bdlora.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <exception>
#include <string>

#include "bdl_kv.h"

struct bdlora_kv {
    int device = 0;
    bdlora_kv_desc d;
    char *k = nullptr, *v = nullptr;
    float* weight = nullptr;
    int* pos = nullptr;
    float* scales = nullptr;       // int8 caches
    char* ws = nullptr;            // the workspace, one allocation
    int* err = nullptr;
    int n_cu = 0;
    float* lse2 = nullptr;         // [max_seqs][n_q_heads]
    float* part = nullptr;         // attend's shares of sequences
    unsigned* count = nullptr;     // kKvAttendCounts counters
    float* logits = nullptr;       // [n_pages][n_q_heads][page_size]
    unsigned* evict_count = nullptr;   // [max_seqs][n_kv_heads + 1] counters
    int* scratch = nullptr;        // [n_pages][n_kv_heads][page_size], where logits lie too
};

namespace {

using bdl::api_fail;

// the thread's current device for the length of a call
struct Device {
    int old = -1;
    bool ok = false;
    explicit Device(int dev) { ok = hipGetDevice(&old) == hipSuccess && (old == dev || hipSetDevice(dev) == hipSuccess); dev_ = dev; }
    ~Device() {
        if (old >= 0 && old != dev_) (void)hipSetDevice(old);
    }
    int dev_;
};

inline int hip_fail(const char* what, hipError_t e) {
    (void)hipGetLastError();
    return api_fail(e == hipErrorOutOfMemory ? BDLORA_ERR_OOM : BDLORA_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

// no C++ exception (an allocation of a message's string) leaves the C ABI
template <class F>
int guarded(F f) noexcept {
    try {
        return f();
    } catch (...) {
        return BDLORA_ERR_OOM;
    }
}

inline bool aligned(const void* p, unsigned n) { return ((uintptr_t)p & (n - 1u)) == 0; }

inline int check_table(const bdlora_kv* c, const int32_t* table, int64_t stride, int32_t width) {
    if (!table || !aligned(table, 4)) return api_fail(BDLORA_ERR_INVALID_ARG, "null or misaligned page table");
    if (width < 1 || stride < width || stride > INT32_MAX) return api_fail(BDLORA_ERR_INVALID_ARG, "a page table row needs 1 <= width <= stride");
    if (((long long)width * c->d.page_size) > (1LL << 30))
        return api_fail(BDLORA_ERR_SHAPE, "a page table row may name at most 2^30 entries");
    return BDLORA_OK;
}

// rows of bf16 values that the kernels take in 16-byte pieces
inline int check_rows(const void* p, int64_t stride, long long row, const char* name) {
    if (!p || !aligned(p, 16)) return api_fail(BDLORA_ERR_INVALID_ARG, std::string(name) + " must be 16-byte aligned");
    if (stride < row || stride % 8 || stride > (1LL << 31))
        return api_fail(BDLORA_ERR_INVALID_ARG, std::string(name) + " needs a row stride of at least its row, a multiple of 8 elements");
    return BDLORA_OK;
}

inline bdl::KvCache view(const bdlora_kv* c, const int32_t* table, int64_t stride, int32_t width) {
    bdl::KvCache v;
    v.K = c->k;
    v.V = c->v;
    v.weight = c->weight;
    v.pos = c->pos;
    v.scales = c->scales;
    v.hq = c->d.n_q_heads;
    v.hkv = c->d.n_kv_heads;
    v.ps_shift = __builtin_ctz((unsigned)c->d.page_size);
    v.n_pages = c->d.n_pages;
    v.table = table;
    v.tstride = (int)stride;
    v.width = width;
    v.err = c->err;
    return v;
}

}  // namespace
