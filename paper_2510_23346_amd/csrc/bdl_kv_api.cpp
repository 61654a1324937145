// C ABI of the key-value cache: validation, workspace and launches.
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

int hip_fail(const char* what, hipError_t e) {
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

bool aligned(const void* p, unsigned n) { return ((uintptr_t)p & (n - 1u)) == 0; }

int check_desc(const bdlora_kv_desc* d) {
    if (!d) return api_fail(BDLORA_ERR_INVALID_ARG, "null description");
    if (d->n_kv_heads < 1 || d->n_q_heads < 1 || d->n_q_heads > bdl::kKvMaxHeads || d->n_q_heads % d->n_kv_heads)
        return api_fail(BDLORA_ERR_SHAPE, "n_q_heads must be 1..1024 and a multiple of n_kv_heads");
    if (d->head_dim != 64 && d->head_dim != 128) return api_fail(BDLORA_ERR_SHAPE, "head_dim must be 64 or 128");
    if (d->page_size < bdl::kKvMinPage || d->page_size > bdl::kKvMaxPage || (d->page_size & (d->page_size - 1)))
        return api_fail(BDLORA_ERR_SHAPE, "page_size must be a power of two, 16..65536");
    if (d->n_pages < 1) return api_fail(BDLORA_ERR_INVALID_ARG, "n_pages must be positive");
    if (d->max_seqs < 1 || d->max_seqs > 65535) return api_fail(BDLORA_ERR_INVALID_ARG, "max_seqs must be 1..65535");
    if (d->format != BDLORA_KV_BF16 && d->format != BDLORA_KV_FP8_E4M3)
        return api_fail(BDLORA_ERR_INVALID_ARG, "unknown cache format");
    if (!(d->k_scale > 0.f && d->v_scale > 0.f) || !std::isfinite(d->k_scale) || !std::isfinite(d->v_scale) ||
        !std::isfinite(1.f / d->k_scale) || !std::isfinite(1.f / d->v_scale))
        return api_fail(BDLORA_ERR_INVALID_ARG, "k_scale and v_scale must be positive and finite, and so their reciprocals");
    if (d->format == BDLORA_KV_BF16 && (d->k_scale != 1.f || d->v_scale != 1.f))
        return api_fail(BDLORA_ERR_INVALID_ARG, "a bf16 cache has scales of 1");
    return BDLORA_OK;
}

struct Parts {
    long long clear, err, count, evict_count, part, lse2, logits, total;   // (what starts at zero lies below clear)
};

Parts layout(const bdlora_kv_desc& d, bool weights) {
    Parts p;
    long long at = 0;
    auto take = [&](long long bytes) {
        const long long r = at;
        at += (bytes + 255) / 256 * 256;
        return r;
    };
    p.err = take(4);
    p.count = take(4LL * bdl::kKvCount * bdl::kKvAttendCounts);
    p.evict_count = take(weights ? 4LL * bdl::kKvCount * d.max_seqs * (d.n_kv_heads + 1) : 0);
    p.clear = at;
    p.part = take(2LL * bdl::kKvAttendGrid * bdl::kv_part_floats(d.head_dim) * 4);
    p.lse2 = take(weights ? 4LL * d.max_seqs * d.n_q_heads : 0);
    p.logits = take(weights ? 4LL * d.n_pages * d.n_q_heads * d.page_size : 0);
    p.total = at;
    return p;
}

int check_table(const bdlora_kv* c, const int32_t* table, int64_t stride, int32_t width) {
    if (!table || !aligned(table, 4)) return api_fail(BDLORA_ERR_INVALID_ARG, "null or misaligned page table");
    if (width < 1 || stride < width || stride > INT32_MAX) return api_fail(BDLORA_ERR_INVALID_ARG, "a page table row needs 1 <= width <= stride");
    if (((long long)width * c->d.page_size) > (1LL << 30))
        return api_fail(BDLORA_ERR_SHAPE, "a page table row may name at most 2^30 entries");
    return BDLORA_OK;
}

// rows of bf16 values that the kernels take in 16-byte pieces
int check_rows(const void* p, int64_t stride, long long row, const char* name) {
    if (!p || !aligned(p, 16)) return api_fail(BDLORA_ERR_INVALID_ARG, std::string(name) + " must be 16-byte aligned");
    if (stride < row || stride % 8 || stride > (1LL << 31))
        return api_fail(BDLORA_ERR_INVALID_ARG, std::string(name) + " needs a row stride of at least its row, a multiple of 8 elements");
    return BDLORA_OK;
}

bdl::KvCache view(const bdlora_kv* c, const int32_t* table, int64_t stride, int32_t width) {
    bdl::KvCache v;
    v.K = c->k;
    v.V = c->v;
    v.weight = c->weight;
    v.pos = c->pos;
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

extern "C" {

int bdlora_kv_create(const bdlora_kv_desc* desc, void* k, void* v, float* weight, int32_t* pos, int32_t device,
                     bdlora_kv_t* out) {
    return guarded([&]() -> int {
        if (!out) return api_fail(BDLORA_ERR_INVALID_ARG, "null output handle");
        *out = nullptr;
        if (int rc = check_desc(desc)) return rc;
        if (!k || !v || !aligned(k, 16) || !aligned(v, 16))
            return api_fail(BDLORA_ERR_INVALID_ARG, "k and v must be 16-byte aligned device memory");
        if ((weight == nullptr) != (pos == nullptr))
            return api_fail(BDLORA_ERR_INVALID_ARG, "weight and pos come together or not at all");
        if (!aligned(weight, 16) || !aligned(pos, 16))
            return api_fail(BDLORA_ERR_INVALID_ARG, "weight and pos must be 16-byte aligned");
        int ndev = 0;
        if (hipGetDeviceCount(&ndev) != hipSuccess || ndev <= 0) {
            (void)hipGetLastError();
            return api_fail(BDLORA_ERR_UNSUPPORTED, "no HIP device");
        }
        if (device < 0 || device >= ndev) return api_fail(BDLORA_ERR_INVALID_ARG, "bad device index");
        hipDeviceProp_t prop;
        if (hipError_t e = hipGetDeviceProperties(&prop, device)) return hip_fail("hipGetDeviceProperties", e);
        if (std::strncmp(prop.gcnArchName, "gfx950", 6) != 0)
            return api_fail(BDLORA_ERR_UNSUPPORTED, std::string("device is ") + prop.gcnArchName + ", need gfx950");
        Device guard(device);
        if (!guard.ok) return api_fail(BDLORA_ERR_HIP, "hipSetDevice failed");
        const Parts p = layout(*desc, weight != nullptr);
        char* ws = nullptr;
        if (hipError_t e = hipMalloc((void**)&ws, (size_t)p.total)) return hip_fail("hipMalloc of the cache's workspace", e);
        hipError_t e = hipMemset(ws, 0, (size_t)p.clear);
        if (!e) e = hipStreamSynchronize(nullptr);
        if (e) {
            (void)hipFree(ws);
            return hip_fail("clearing the cache's workspace", e);
        }
        bdlora_kv* c = new (std::nothrow) bdlora_kv();
        if (!c) {
            (void)hipFree(ws);
            return api_fail(BDLORA_ERR_OOM, "host allocation failed");
        }
        c->device = device;
        c->d = *desc;
        c->k = (char*)k;
        c->v = (char*)v;
        c->weight = weight;
        c->pos = pos;
        c->ws = ws;
        c->err = (int*)(ws + p.err);
        c->n_cu = std::max(1, prop.multiProcessorCount);
        c->count = (unsigned*)(ws + p.count);
        c->part = (float*)(ws + p.part);
        c->lse2 = (float*)(ws + p.lse2);
        c->logits = (float*)(ws + p.logits);
        c->evict_count = (unsigned*)(ws + p.evict_count);
        c->scratch = (int*)(ws + p.logits);
        *out = c;
        return BDLORA_OK;
    });
}

int bdlora_kv_destroy(bdlora_kv_t c) {
    return guarded([&]() -> int {
        if (!c) return api_fail(BDLORA_ERR_INVALID_ARG, "null cache");
        Device guard(c->device);
        (void)hipDeviceSynchronize();
        (void)hipFree(c->ws);
        delete c;
        return BDLORA_OK;
    });
}

int bdlora_kv_bytes(const bdlora_kv_desc* desc, int32_t weights, int64_t* page_bytes, int64_t* workspace_bytes) {
    return guarded([&]() -> int {
        if (int rc = check_desc(desc)) return rc;
        const long long size = desc->format == BDLORA_KV_BF16 ? 2 : 1;
        if (page_bytes)
            *page_bytes = (2LL * desc->head_dim * size + (weights ? 8 : 0)) * desc->n_kv_heads * desc->page_size;
        if (workspace_bytes) *workspace_bytes = layout(*desc, weights != 0).total;
        return BDLORA_OK;
    });
}

int bdlora_kv_append(bdlora_kv_t c, const void* qkv, int64_t qkv_stride, const float* cos, const float* sin,
                     int32_t n_positions, int32_t interleaved, const int32_t* seqs, const int32_t* index,
                     const int32_t* positions, int32_t T, const int32_t* table, int64_t table_stride, int32_t table_width,
                     int32_t n_seqs, int32_t* lens, void* q_out, int64_t q_stride, void* stream) {
    return guarded([&]() -> int {
        if (!c) return api_fail(BDLORA_ERR_INVALID_ARG, "null cache");
        if (T < 0) return api_fail(BDLORA_ERR_INVALID_ARG, "negative T");
        if (T == 0) return BDLORA_OK;
        const long long D = c->d.head_dim;
        if (int rc = check_rows(qkv, qkv_stride, (c->d.n_q_heads + 2 * c->d.n_kv_heads) * D, "qkv")) return rc;
        if (int rc = check_rows(q_out, q_stride, c->d.n_q_heads * D, "q_out")) return rc;
        if (!cos || !sin || !aligned(cos, 16) || !aligned(sin, 16) || n_positions < 1)
            return api_fail(BDLORA_ERR_INVALID_ARG, "cos and sin must be 16-byte aligned, of at least one position");
        if (!seqs || !index || !positions || !aligned(seqs, 4) || !aligned(index, 4) || !aligned(positions, 4) || !aligned(lens, 4))
            return api_fail(BDLORA_ERR_INVALID_ARG, "seqs, index and positions must be int32 device arrays");
        if (n_seqs < 1) return api_fail(BDLORA_ERR_INVALID_ARG, "n_seqs must be positive");
        if (int rc = check_table(c, table, table_stride, table_width)) return rc;
        Device guard(c->device);
        if (!guard.ok) return api_fail(BDLORA_ERR_HIP, "hipSetDevice failed");
        bdl::KvAppendArgs a;
        a.c = view(c, table, table_stride, table_width);
        a.qkv = (const uint16_t*)qkv;
        a.qkv_stride = qkv_stride;
        a.q_out = (uint16_t*)q_out;
        a.q_stride = q_stride;
        a.cos = cos;
        a.sin = sin;
        a.n_positions = n_positions;
        a.interleaved = interleaved != 0;
        a.seqs = seqs;
        a.index = index;
        a.positions = positions;
        a.lens = lens;
        a.T = T;
        a.n_seqs = n_seqs;
        a.k_inv = 1.f / c->d.k_scale;
        a.v_inv = 1.f / c->d.v_scale;
        if (hipError_t e = bdl::launch_kv_append(a, c->d.head_dim, c->d.format == BDLORA_KV_FP8_E4M3, (hipStream_t)stream))
            return hip_fail("append launch", e);
        return BDLORA_OK;
    });
}

int bdlora_kv_attend(bdlora_kv_t c, const void* q, int64_t q_stride, int32_t B, const int32_t* table, int64_t table_stride,
                     int32_t table_width, const int32_t* lens, const int32_t* starts, float scale, int32_t accumulate,
                     void* out, int64_t out_stride, float* lse, void* stream) {
    return guarded([&]() -> int {
        if (!c) return api_fail(BDLORA_ERR_INVALID_ARG, "null cache");
        if (B < 0 || B > c->d.max_seqs) return api_fail(BDLORA_ERR_INVALID_ARG, "B must be 0..max_seqs");
        if (accumulate && !c->weight) return api_fail(BDLORA_ERR_INVALID_ARG, "this cache tracks no weights");
        if (!std::isfinite(scale)) return api_fail(BDLORA_ERR_INVALID_ARG, "scale must be finite");
        if (B == 0) return BDLORA_OK;
        const long long row = (long long)c->d.n_q_heads * c->d.head_dim;
        if (int rc = check_rows(q, q_stride, row, "q")) return rc;
        if (int rc = check_rows(out, out_stride, row, "out")) return rc;
        if (!lens || !aligned(lens, 4) || !aligned(starts, 4) || !aligned(lse, 4))
            return api_fail(BDLORA_ERR_INVALID_ARG, "lens (and starts) must be int32, lse fp32 device arrays");
        if (int rc = check_table(c, table, table_stride, table_width)) return rc;
        // (the kernel counts tiles of 32 entries in 32 bits)
        const long long heads = (long long)c->d.n_kv_heads * ((c->d.n_q_heads / c->d.n_kv_heads + bdl::kKvHeads - 1) / bdl::kKvHeads);
        if (((long long)table_width * c->d.page_size + 63) / 32 * B * heads > INT32_MAX)
            return api_fail(BDLORA_ERR_SHAPE, "more than 2^31 tiles: B x kv heads x a row's entries / 32");
        Device guard(c->device);
        if (!guard.ok) return api_fail(BDLORA_ERR_HIP, "hipSetDevice failed");
        bdl::KvAttendArgs a;
        a.c = view(c, table, table_stride, table_width);
        a.q = (const uint16_t*)q;
        a.q_stride = q_stride;
        a.out = (uint16_t*)out;
        a.out_stride = out_stride;
        a.lens = lens;
        a.starts = starts ? starts : lens;
        a.has_starts = starts != nullptr;
        a.lse = lse;
        a.B = B;
        a.part = c->part;
        a.count = c->count;
        a.logits = c->logits;
        a.lse2 = c->lse2;
        // (the kernels mask with -infinity times the scale: it is kept above zero)
        a.score_scale = (float)std::max(std::fabs((double)scale * c->d.k_scale * 1.4426950408889634), 1e-37);
        a.q_sign = scale < 0.f ? 0x80008000u : 0u;
        a.v_scale = c->d.v_scale;
        if (hipError_t e = bdl::launch_kv_attend(a, c->d.head_dim, c->d.format == BDLORA_KV_FP8_E4M3, accumulate != 0, (hipStream_t)stream))
            return hip_fail("attend launch", e);
        return BDLORA_OK;
    });
}

int bdlora_kv_evict(bdlora_kv_t c, int32_t B, const int32_t* table, int64_t table_stride, int32_t table_width, int32_t* lens,
                    int32_t budget, int32_t recent, void* stream) {
    return guarded([&]() -> int {
        if (!c) return api_fail(BDLORA_ERR_INVALID_ARG, "null cache");
        if (!c->weight) return api_fail(BDLORA_ERR_INVALID_ARG, "this cache tracks no weights");
        if (B < 0 || B > c->d.max_seqs) return api_fail(BDLORA_ERR_INVALID_ARG, "B must be 0..max_seqs");
        if (budget < 1 || recent < 0 || recent > budget)
            return api_fail(BDLORA_ERR_INVALID_ARG, "evict needs budget >= 1 and 0 <= recent <= budget");
        if (B == 0) return BDLORA_OK;
        if (!lens || !aligned(lens, 4)) return api_fail(BDLORA_ERR_INVALID_ARG, "lens must be an int32 device array");
        if (int rc = check_table(c, table, table_stride, table_width)) return rc;
        Device guard(c->device);
        if (!guard.ok) return api_fail(BDLORA_ERR_HIP, "hipSetDevice failed");
        bdl::KvEvictArgs a;
        a.c = view(c, table, table_stride, table_width);
        a.lens = lens;
        a.B = B;
        a.budget = budget;
        a.recent = recent;
        a.scratch = c->scratch;
        a.count = c->evict_count;
        a.n_cu = c->n_cu;
        if (hipError_t e = bdl::launch_kv_evict(a, c->d.head_dim, c->d.format == BDLORA_KV_FP8_E4M3, (hipStream_t)stream))
            return hip_fail("evict launch", e);
        return BDLORA_OK;
    });
}

int bdlora_kv_get_device_error(bdlora_kv_t c, void* stream, int32_t* flag) {
    return guarded([&]() -> int {
        if (!c || !flag) return api_fail(BDLORA_ERR_INVALID_ARG, "null argument");
        Device guard(c->device);
        if (!guard.ok) return api_fail(BDLORA_ERR_HIP, "hipSetDevice failed");
        hipStream_t s = (hipStream_t)stream;
        int32_t v = 0;
        const int32_t zero = 0;
        if (hipError_t e = hipMemcpyAsync(&v, c->err, 4, hipMemcpyDeviceToHost, s)) return hip_fail("hipMemcpyAsync", e);
        if (hipError_t e = hipStreamSynchronize(s)) return hip_fail("hipStreamSynchronize", e);
        if (hipError_t e = hipMemcpyAsync(c->err, &zero, 4, hipMemcpyHostToDevice, s)) return hip_fail("hipMemcpyAsync", e);
        if (hipError_t e = hipStreamSynchronize(s)) return hip_fail("hipStreamSynchronize", e);
        *flag = v;
        return BDLORA_OK;
    });
}

}  // extern "C"
