// C ABI of the key-value cache's calls over many rows: attention of many new
// tokens, reading entries back.
#include "bdl_kv_cache.h"

extern "C" {

int bdlora_kv_read(bdlora_kv_t c, const int32_t* seqs, const int32_t* index, int32_t T, const int32_t* table,
                   int64_t table_stride, int32_t table_width, int32_t n_seqs, void* k_out, int64_t k_stride, void* v_out,
                   int64_t v_stride, void* stream) {
    return guarded([&]() -> int {
        if (!c) return api_fail(BDLORA_ERR_INVALID_ARG, "null cache");
        if (T < 0) return api_fail(BDLORA_ERR_INVALID_ARG, "negative T");
        if (T == 0) return BDLORA_OK;
        const long long row = (long long)c->d.n_kv_heads * c->d.head_dim;
        if (int rc = check_rows(k_out, k_stride, row, "k_out")) return rc;
        if (int rc = check_rows(v_out, v_stride, row, "v_out")) return rc;
        if (k_out == v_out) return api_fail(BDLORA_ERR_INVALID_ARG, "k_out and v_out must not be the same memory");
        if (!seqs || !index || !aligned(seqs, 4) || !aligned(index, 4))
            return api_fail(BDLORA_ERR_INVALID_ARG, "seqs and index must be int32 device arrays");
        if (n_seqs < 1) return api_fail(BDLORA_ERR_INVALID_ARG, "n_seqs must be positive");
        if (int rc = check_table(c, table, table_stride, table_width)) return rc;
        Device guard(c->device);
        if (!guard.ok) return api_fail(BDLORA_ERR_HIP, "hipSetDevice failed");
        bdl::KvReadArgs a;
        a.c = view(c, table, table_stride, table_width);
        a.seqs = seqs;
        a.index = index;
        a.T = T;
        a.n_seqs = n_seqs;
        a.k_out = (uint16_t*)k_out;
        a.v_out = (uint16_t*)v_out;
        a.k_stride = k_stride;
        a.v_stride = v_stride;
        a.k_scale = c->d.k_scale;
        a.v_scale = c->d.v_scale;
        if (hipError_t e = bdl::launch_kv_read(a, c->d.head_dim, c->d.format == BDLORA_KV_FP8_E4M3, (hipStream_t)stream))
            return hip_fail("read launch", e);
        return BDLORA_OK;
    });
}

int bdlora_kv_attend_prompt(bdlora_kv_t c, const void* q, int64_t q_stride, int32_t T, const int32_t* q_starts, int32_t B,
                            const int32_t* table, int64_t table_stride, int32_t table_width, const int32_t* lens, int32_t window,
                            int32_t sinks, float scale, void* out, int64_t out_stride, float* lse, void* stream) {
    return guarded([&]() -> int {
        if (!c) return api_fail(BDLORA_ERR_INVALID_ARG, "null cache");
        if (B < 0 || B > c->d.max_seqs) return api_fail(BDLORA_ERR_INVALID_ARG, "B must be 0..max_seqs");
        if (T < 0) return api_fail(BDLORA_ERR_INVALID_ARG, "negative T");
        if (window < 0 || sinks < 0) return api_fail(BDLORA_ERR_INVALID_ARG, "window and sinks must not be negative");
        if (!std::isfinite(scale)) return api_fail(BDLORA_ERR_INVALID_ARG, "scale must be finite");
        if (T == 0 || B == 0) return BDLORA_OK;
        const long long row = (long long)c->d.n_q_heads * c->d.head_dim;
        if (int rc = check_rows(q, q_stride, row, "q")) return rc;
        if (int rc = check_rows(out, out_stride, row, "out")) return rc;
        if (!lens || !aligned(lens, 4) || !q_starts || !aligned(q_starts, 4) || !aligned(lse, 4))
            return api_fail(BDLORA_ERR_INVALID_ARG, "lens and q_starts must be int32, lse fp32 device arrays");
        if (int rc = check_table(c, table, table_stride, table_width)) return rc;
        // (rows of a kv head, one for each token and query head, are counted in 32 bits)
        if ((long long)T * c->d.n_q_heads > 1LL << 30)
            return api_fail(BDLORA_ERR_SHAPE, "more than 2^30 rows: T x query heads");
        // (and a grid holds less than 2^24 workgroups of 256)
        if ((long long)B * c->d.n_kv_heads >= 1LL << 23)
            return api_fail(BDLORA_ERR_SHAPE, "2^23 sequences' heads or more: B x kv heads");
        Device guard(c->device);
        if (!guard.ok) return api_fail(BDLORA_ERR_HIP, "hipSetDevice failed");
        bdl::KvPromptArgs a;
        a.c = view(c, table, table_stride, table_width);
        a.q = (const uint16_t*)q;
        a.q_stride = q_stride;
        a.out = (uint16_t*)out;
        a.out_stride = out_stride;
        a.q_starts = q_starts;
        a.lens = lens;
        a.lse = lse;
        a.T = T;
        a.B = B;
        a.part = c->part;
        a.count = c->count;
        a.split = 0;
        a.window = std::min(window, 1 << 30);         // (no row sees more, and an entry's number less it fits 32 bits)
        a.sinks = window ? sinks : 0;         // (without a window every entry is attended to)
        // (kept above zero: masked scores are -infinity, times the scale too)
        a.score_scale = (float)std::max(std::fabs((double)scale * c->d.k_scale * 1.4426950408889634), 1e-37);
        a.q_sign = scale < 0.f ? 0x80008000u : 0u;
        a.v_scale = c->d.v_scale;
        if (hipError_t e = bdl::launch_kv_prompt(a, c->d.head_dim, c->d.format == BDLORA_KV_FP8_E4M3, (hipStream_t)stream))
            return hip_fail("prompt attention launch", e);
        return BDLORA_OK;
    });
}

}  // extern "C"
