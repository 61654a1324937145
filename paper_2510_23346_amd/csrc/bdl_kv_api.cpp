// C ABI of the key-value cache: validation, workspace and launches.
#include "bdl_kv_cache.h"

namespace {

int check_desc(const bdlora_kv_desc* d) {
    if (!d) return api_fail(BDLORA_ERR_INVALID_ARG, "null description");
    if (d->n_kv_heads < 1 || d->n_q_heads < 1 || d->n_q_heads > bdl::kKvMaxHeads || d->n_q_heads % d->n_kv_heads)
        return api_fail(BDLORA_ERR_SHAPE, "n_q_heads must be 1..1024 and a multiple of n_kv_heads");
    if (d->head_dim != 64 && d->head_dim != 128) return api_fail(BDLORA_ERR_SHAPE, "head_dim must be 64 or 128");
    if (d->page_size < bdl::kKvMinPage || d->page_size > bdl::kKvMaxPage || (d->page_size & (d->page_size - 1)))
        return api_fail(BDLORA_ERR_SHAPE, "page_size must be a power of two, 16..65536");
    if (d->n_pages < 1) return api_fail(BDLORA_ERR_INVALID_ARG, "n_pages must be positive");
    if (d->max_seqs < 1 || d->max_seqs > 65535) return api_fail(BDLORA_ERR_INVALID_ARG, "max_seqs must be 1..65535");
    if (d->format != BDLORA_KV_BF16 && d->format != BDLORA_KV_FP8_E4M3 && d->format != BDLORA_KV_INT8_BLOCK)
        return api_fail(BDLORA_ERR_INVALID_ARG, "unknown cache format");
    if (!(d->k_scale > 0.f && d->v_scale > 0.f) || !std::isfinite(d->k_scale) || !std::isfinite(d->v_scale) ||
        !std::isfinite(1.f / d->k_scale) || !std::isfinite(1.f / d->v_scale))
        return api_fail(BDLORA_ERR_INVALID_ARG, "k_scale and v_scale must be positive and finite, and so their reciprocals");
    if (d->format != BDLORA_KV_FP8_E4M3 && (d->k_scale != 1.f || d->v_scale != 1.f))
        return api_fail(BDLORA_ERR_INVALID_ARG, "a bf16 cache, and one with a scale for each block, has k_scale and v_scale of 1");
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
    p.part = take((long long)bdl::kKvSlots * bdl::kv_part_floats(d.head_dim) * 4);
    p.lse2 = take(weights ? 4LL * d.max_seqs * d.n_q_heads : 0);
    p.logits = take(weights ? 4LL * d.n_pages * d.n_q_heads * d.page_size : 0);
    p.total = at;
    return p;
}

int create(const bdlora_kv_desc* desc, void* k, void* v, float* scales, float* weight, int32_t* pos, int32_t device,
           bdlora_kv_t* out) {
    return guarded([&]() -> int {
        if (!out) return api_fail(BDLORA_ERR_INVALID_ARG, "null output handle");
        *out = nullptr;
        if (int rc = check_desc(desc)) return rc;
        if ((desc->format == BDLORA_KV_INT8_BLOCK) != (scales != nullptr))
            return api_fail(BDLORA_ERR_INVALID_ARG, "a cache with a scale for each block, and no other, is made with its array of scales");
        if (!aligned(scales, 8)) return api_fail(BDLORA_ERR_INVALID_ARG, "scales must be 8-byte aligned device memory");
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
        c->scales = scales;
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

int append(bdlora_kv_t c, const void* qkv, int64_t qkv_stride, const void* q_norm, const void* k_norm, float eps, const float* cos,
           const float* sin, int32_t n_positions, int32_t interleaved, const int32_t* seqs, const int32_t* index,
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
        if ((q_norm == nullptr) != (k_norm == nullptr))
            return api_fail(BDLORA_ERR_INVALID_ARG, "q_norm and k_norm come together or not at all");
        if (!aligned(q_norm, 16) || !aligned(k_norm, 16))
            return api_fail(BDLORA_ERR_INVALID_ARG, "q_norm and k_norm must be 16-byte aligned");
        if (q_norm && !(eps >= 0.f && std::isfinite(eps)))
            return api_fail(BDLORA_ERR_INVALID_ARG, "eps must be finite and not negative");
        if (n_seqs < 1) return api_fail(BDLORA_ERR_INVALID_ARG, "n_seqs must be positive");
        if (int rc = check_table(c, table, table_stride, table_width)) return rc;
        // (a grid holds less than 2^24 workgroups of 256: T for queries, T x kv heads / 2 for blocks at most)
        if (c->scales && (long long)T * (c->d.n_kv_heads + 2) > (1LL << 25) - 8)
            return api_fail(BDLORA_ERR_SHAPE, "more than 2^25 - 8: T x (kv heads + 2)");
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
        a.q_norm = (const uint16_t*)q_norm;
        a.k_norm = (const uint16_t*)k_norm;
        a.eps = eps;
        a.owners = (int*)c->part;
        a.n_owners = (unsigned)(bdl::kKvSlots * bdl::kv_part_floats(c->d.head_dim));
        a.k_inv = 1.f / c->d.k_scale;
        a.v_inv = 1.f / c->d.v_scale;
        if (hipError_t e = bdl::launch_kv_append(a, c->d.head_dim, c->d.format == BDLORA_KV_FP8_E4M3, (hipStream_t)stream))
            return hip_fail("append launch", e);
        return BDLORA_OK;
    });
}

int attend(bdlora_kv_t c, const void* q, int64_t q_stride, int32_t B, const int32_t* table, int64_t table_stride,
           int32_t table_width, const int32_t* lens, const int32_t* starts, int32_t sinks, float scale, int32_t accumulate,
           void* out, int64_t out_stride, float* lse, void* stream) {
    return guarded([&]() -> int {
        if (!c) return api_fail(BDLORA_ERR_INVALID_ARG, "null cache");
        if (B < 0 || B > c->d.max_seqs) return api_fail(BDLORA_ERR_INVALID_ARG, "B must be 0..max_seqs");
        if (accumulate && !c->weight) return api_fail(BDLORA_ERR_INVALID_ARG, "this cache tracks no weights");
        if (!std::isfinite(scale)) return api_fail(BDLORA_ERR_INVALID_ARG, "scale must be finite");
        if (sinks < 0) return api_fail(BDLORA_ERR_INVALID_ARG, "sinks must not be negative");
        if (B == 0) return BDLORA_OK;
        const long long row = (long long)c->d.n_q_heads * c->d.head_dim;
        if (int rc = check_rows(q, q_stride, row, "q")) return rc;
        if (int rc = check_rows(out, out_stride, row, "out")) return rc;
        if (!lens || !aligned(lens, 4) || !aligned(starts, 4) || !aligned(lse, 4))
            return api_fail(BDLORA_ERR_INVALID_ARG, "lens (and starts) must be int32, lse fp32 device arrays");
        if (int rc = check_table(c, table, table_stride, table_width)) return rc;
        // (the kernel counts tiles of 32 entries in 32 bits)
        const long long heads = (long long)c->d.n_kv_heads * ((c->d.n_q_heads / c->d.n_kv_heads + bdl::kKvHeads - 1) / bdl::kKvHeads);
        if (((long long)table_width * c->d.page_size + (sinks ? 127 : 63)) / 32 * B * heads > INT32_MAX)
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
        a.sinks = starts ? sinks : 0;         // (without a window every entry is attended to)
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

}  // namespace

extern "C" {

int bdlora_kv_create(const bdlora_kv_desc* desc, void* k, void* v, float* weight, int32_t* pos, int32_t device,
                     bdlora_kv_t* out) {
    return create(desc, k, v, nullptr, weight, pos, device, out);
}

int bdlora_kv_create_blocks(const bdlora_kv_desc* desc, void* k, void* v, float* scales, int32_t device, bdlora_kv_t* out) {
    return create(desc, k, v, scales, nullptr, nullptr, device, out);
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
        if (weights && desc->format == BDLORA_KV_INT8_BLOCK)
            return api_fail(BDLORA_ERR_INVALID_ARG, "a cache with a scale for each block tracks no weights");
        const long long size = desc->format == BDLORA_KV_BF16 ? 2 : 1;
        if (page_bytes)
            *page_bytes = (2LL * desc->head_dim * size + (weights ? 8 : 0)) * desc->n_kv_heads * desc->page_size +
                          (desc->format == BDLORA_KV_INT8_BLOCK ? 8LL * desc->n_kv_heads * (desc->page_size / bdl::kKvBlock) : 0);
        if (workspace_bytes) *workspace_bytes = layout(*desc, weights != 0).total;
        return BDLORA_OK;
    });
}

int bdlora_kv_append(bdlora_kv_t c, const void* qkv, int64_t qkv_stride, const float* cos, const float* sin,
                     int32_t n_positions, int32_t interleaved, const int32_t* seqs, const int32_t* index,
                     const int32_t* positions, int32_t T, const int32_t* table, int64_t table_stride, int32_t table_width,
                     int32_t n_seqs, int32_t* lens, void* q_out, int64_t q_stride, void* stream) {
    return append(c, qkv, qkv_stride, nullptr, nullptr, 0.f, cos, sin, n_positions, interleaved, seqs, index, positions, T, table,
                  table_stride, table_width, n_seqs, lens, q_out, q_stride, stream);
}

int bdlora_kv_append_norm(bdlora_kv_t c, const void* qkv, int64_t qkv_stride, const void* q_norm, const void* k_norm, float eps,
                          const float* cos, const float* sin, int32_t n_positions, int32_t interleaved, const int32_t* seqs,
                          const int32_t* index, const int32_t* positions, int32_t T, const int32_t* table, int64_t table_stride,
                          int32_t table_width, int32_t n_seqs, int32_t* lens, void* q_out, int64_t q_stride, void* stream) {
    if (!q_norm || !k_norm) return guarded([]() -> int { return api_fail(BDLORA_ERR_INVALID_ARG, "null q_norm or k_norm"); });
    return append(c, qkv, qkv_stride, q_norm, k_norm, eps, cos, sin, n_positions, interleaved, seqs, index, positions, T, table,
                  table_stride, table_width, n_seqs, lens, q_out, q_stride, stream);
}

int bdlora_kv_attend(bdlora_kv_t c, const void* q, int64_t q_stride, int32_t B, const int32_t* table, int64_t table_stride,
                     int32_t table_width, const int32_t* lens, const int32_t* starts, float scale, int32_t accumulate,
                     void* out, int64_t out_stride, float* lse, void* stream) {
    return attend(c, q, q_stride, B, table, table_stride, table_width, lens, starts, 0, scale, accumulate, out, out_stride, lse, stream);
}

int bdlora_kv_attend_sinks(bdlora_kv_t c, const void* q, int64_t q_stride, int32_t B, const int32_t* table, int64_t table_stride,
                           int32_t table_width, const int32_t* lens, const int32_t* starts, int32_t sinks, float scale,
                           int32_t accumulate, void* out, int64_t out_stride, float* lse, void* stream) {
    return attend(c, q, q_stride, B, table, table_stride, table_width, lens, starts, sinks, scale, accumulate, out, out_stride, lse,
                  stream);
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
