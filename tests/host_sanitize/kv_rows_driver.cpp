// The argument checks of the key-value cache's calls over many rows, of its
// format with a scale for each block, of norms and sinks, under AddressSanitizer
// and UndefinedBehaviorSanitizer.  As in kv_driver.cpp, caches are made by hand
// and the launchers are stubs: a call whose arguments are right fails at the
// device or the stub (HIP), one whose arguments are wrong must not get that far.
#include "../../paper_2510_23346_amd/csrc/bdl_kv_api.cpp"
#include "../../paper_2510_23346_amd/csrc/bdl_kv_rows_api.cpp"

#include <cstdio>
#include <cstdlib>

namespace bdl {
hipError_t launch_kv_append(const KvAppendArgs&, int, bool, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_kv_attend(const KvAttendArgs&, int, bool, bool, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_kv_evict(const KvEvictArgs&, int, bool, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_kv_read(const KvReadArgs&, int, bool, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_kv_prompt(const KvPromptArgs&, int, bool, hipStream_t) { return hipErrorNotSupported; }
}  // namespace bdl

static int failed = 0, checks = 0;

static void expect(int got, int want, const char* what) {
    ++checks;
    if (got != want) {
        ++failed;
        std::printf("%s: got %d, want %d (%s)\n", what, got, want, bdlora_last_error());
    }
}

int main() {
    const int INV = BDLORA_ERR_INVALID_ARG, SH = BDLORA_ERR_SHAPE, HIP = BDLORA_ERR_HIP;
    alignas(16) static char mem[4096];
    void* const p = mem;
    int* const i = (int*)mem;
    float* const f = (float*)mem;

    // the format
    const bdlora_kv_desc bf16{8, 2, 128, 64, 100, 16, BDLORA_KV_BF16, 1.f, 1.f};
    bdlora_kv_desc int8 = bf16;
    int8.format = BDLORA_KV_INT8_BLOCK;
    int64_t page = 0, ws = 0, ws0 = 0;
    expect(bdlora_kv_bytes(&int8, 0, &page, &ws), BDLORA_OK, "bytes");
    expect(bdlora_kv_bytes(&bf16, 0, nullptr, &ws0), BDLORA_OK, "bytes");
    expect(page == 2LL * 2 * 64 * 128 + 2 * 4 * 8 && ws == ws0, 1, "a page's bytes and its scales'");
    expect(bdlora_kv_bytes(&int8, 1, &page, &ws), INV, "block scales and weights");
    bdlora_kv_desc scaled = int8;
    scaled.k_scale = 0.5f;
    expect(bdlora_kv_bytes(&scaled, 0, &page, &ws), INV, "block scales and k_scale");
    bdlora_kv_t out = (bdlora_kv_t)p;
    expect(bdlora_kv_create(&int8, p, p, nullptr, nullptr, 0, &out), INV, "block scales without their array");
    expect(out == nullptr, 1, "handle cleared");
    expect(bdlora_kv_create_blocks(&bf16, p, p, f, 0, &out), INV, "scales of a bf16 cache");
    expect(bdlora_kv_create_blocks(&int8, p, p, nullptr, 0, &out), INV, "null scales");
    expect(bdlora_kv_create_blocks(&int8, p, p, (float*)(mem + 4), 0, &out), INV, "misaligned scales");
    expect(bdlora_kv_create_blocks(&int8, p, p, f, 0, nullptr), INV, "null handle");

    bdlora_kv c;
    c.device = 0;
    c.d = int8;
    c.k = c.v = mem;
    c.scales = f;
    bdlora_kv plain = c;
    plain.d = bf16;
    plain.scales = nullptr;

    // append with norms
    struct A {
        bdlora_kv_t c;
        const void *qkv, *qn, *kn;
        float eps;
        int T;
        void* q;
    };
    const A a0{&c, p, p, p, 1e-6f, 3, p};
    auto app = [&](auto change, int want, const char* what) {
        A a = a0;
        change(a);
        expect(bdlora_kv_append_norm(a.c, a.qkv, 12 * 128, a.qn, a.kn, a.eps, f, f, 10, 0, i, i, i, a.T, i, 4, 4, 2, i, a.q, 8 * 128, nullptr),
               want, what);
    };
    app([](A&) {}, HIP, "append with norms");
    app([&](A& a) { a.c = &plain; }, HIP, "append with norms to bf16");
    app([](A& a) { a.T = 0; }, BDLORA_OK, "append nothing");
    app([](A& a) { a.eps = 0.f; }, HIP, "eps 0");
    app([](A& a) { a.qn = nullptr; }, INV, "null q_norm");
    app([](A& a) { a.kn = nullptr; }, INV, "null k_norm");
    app([&](A& a) { a.qn = mem + 8; }, INV, "misaligned q_norm");
    app([&](A& a) { a.kn = mem + 2; }, INV, "misaligned k_norm");
    app([](A& a) { a.eps = -1e-6f; }, INV, "negative eps");
    app([](A& a) { a.eps = NAN; }, INV, "eps NaN");
    app([](A& a) { a.eps = INFINITY; }, INV, "eps infinite");
    app([](A& a) { a.c = nullptr; }, INV, "null cache");
    app([&](A& a) { a.qkv = mem + 8; }, INV, "misaligned qkv");
    app([](A& a) { a.T = (1 << 23) - 1; }, SH, "more tokens than a grid is for");
    app([](A& a) { a.T = (1 << 23) - 2; }, HIP, "as many");
    app([&](A& a) { a.c = &plain, a.T = 1 << 23; }, HIP, "to bf16");

    // sinks
    auto att = [&](bdlora_kv_t cc, int B, const int* starts, int sinks, int acc, int want, const char* what) {
        expect(bdlora_kv_attend_sinks(cc, p, 8 * 128, B, i, 4, 4, i, starts, sinks, 0.1f, acc, p, 8 * 128, f, nullptr), want, what);
    };
    att(&c, 3, i, 4, 0, HIP, "attend with sinks");
    att(&c, 3, nullptr, 4, 0, HIP, "sinks without starts");
    att(&c, 3, i, INT32_MAX, 0, HIP, "many sinks");
    att(&c, 0, i, 4, 0, BDLORA_OK, "attend nothing");
    att(&c, 3, i, -1, 0, INV, "negative sinks");
    att(&c, 3, i, 4, 1, INV, "accumulate without weights");
    att(nullptr, 3, i, 4, 0, INV, "null cache");
    expect(bdlora_kv_evict(&c, 3, i, 4, 4, i, 5, 5, nullptr), INV, "evict from a cache with block scales");

    // attention of many tokens
    struct P {
        bdlora_kv_t c;
        const void* q; int64_t qs; int T; const int* qb; int B; const int* t; int64_t ts; int tw; const int* l; int w, s; float sc; void* o;
        int64_t os; float* e;
    };
    const P p0{&c, p, 8 * 128, 7, i, 3, i, 4, 4, i, 5, 2, 0.1f, p, 8 * 128, f};
    auto pro = [&](auto change, int want, const char* what) {
        P x = p0;
        change(x);
        expect(bdlora_kv_attend_prompt(x.c, x.q, x.qs, x.T, x.qb, x.B, x.t, x.ts, x.tw, x.l, x.w, x.s, x.sc, x.o, x.os, x.e, nullptr), want, what);
    };
    pro([](P&) {}, HIP, "prompt");
    pro([&](P& x) { x.c = &plain, x.e = nullptr, x.w = x.s = 0; }, HIP, "prompt without the optional ones");
    pro([](P& x) { x.w = x.s = INT32_MAX; }, HIP, "largest window and sinks");
    pro([](P& x) { x.T = 0, x.q = nullptr; }, BDLORA_OK, "no tokens");
    pro([](P& x) { x.B = 0, x.l = nullptr; }, BDLORA_OK, "no sequences");
    pro([](P& x) { x.c = nullptr; }, INV, "null cache");
    pro([](P& x) { x.T = -1; }, INV, "negative T");
    pro([](P& x) { x.B = -1; }, INV, "negative B");
    pro([](P& x) { x.B = 17; }, INV, "more than max_seqs");
    pro([](P& x) { x.w = -1; }, INV, "negative window");
    pro([](P& x) { x.s = -1; }, INV, "negative sinks");
    pro([](P& x) { x.sc = NAN; }, INV, "scale NaN");
    pro([](P& x) { x.q = nullptr; }, INV, "null q");
    pro([&](P& x) { x.q = mem + 8; }, INV, "misaligned q");
    pro([](P& x) { x.qs = 8 * 128 - 8; }, INV, "q stride");
    pro([](P& x) { x.o = nullptr; }, INV, "null out");
    pro([](P& x) { x.os = 8 * 128 + 4; }, INV, "out stride");
    pro([](P& x) { x.qb = nullptr; }, INV, "null q_starts");
    pro([&](P& x) { x.qb = (int*)(mem + 2); }, INV, "misaligned q_starts");
    pro([](P& x) { x.l = nullptr; }, INV, "null lens");
    pro([&](P& x) { x.e = (float*)(mem + 1); }, INV, "misaligned lse");
    pro([](P& x) { x.t = nullptr; }, INV, "null table");
    pro([](P& x) { x.tw = 5; }, INV, "width beyond the stride");
    pro([](P& x) { x.ts = x.tw = 1 << 25; }, SH, "more than 2^30 entries");
    pro([](P& x) { x.T = (1 << 27) + 1; }, SH, "more than 2^30 rows");
    pro([](P& x) { x.T = 1 << 27; }, HIP, "2^30 rows");
    bdlora_kv many = c;
    many.d.n_q_heads = many.d.n_kv_heads = 256;
    many.d.max_seqs = 65535;
    pro([&](P& x) { x.c = &many, x.qs = x.os = 256 * 128, x.B = 1 << 15; }, SH, "2^23 sequences' heads");
    pro([&](P& x) { x.c = &many, x.qs = x.os = 256 * 128, x.B = (1 << 15) - 1; }, HIP, "fewer");

    // read
    struct R {
        bdlora_kv_t c;
        const int *s, *ix; int T; const int* t; int64_t ts; int tw, ns; void* k; int64_t ks; void* v; int64_t vs;
    };
    const R r0{&c, i, i, 3, i, 4, 4, 2, p, 2 * 128, mem + 2048, 2 * 128};
    auto rd = [&](auto change, int want, const char* what) {
        R r = r0;
        change(r);
        expect(bdlora_kv_read(r.c, r.s, r.ix, r.T, r.t, r.ts, r.tw, r.ns, r.k, r.ks, r.v, r.vs, nullptr), want, what);
    };
    rd([](R&) {}, HIP, "read");
    rd([](R& r) { r.T = 0, r.k = nullptr; }, BDLORA_OK, "read nothing");
    rd([](R& r) { r.c = nullptr; }, INV, "null cache");
    rd([](R& r) { r.T = -1; }, INV, "negative T");
    rd([](R& r) { r.s = nullptr; }, INV, "null seqs");
    rd([&](R& r) { r.ix = (int*)(mem + 1); }, INV, "misaligned index");
    rd([](R& r) { r.k = nullptr; }, INV, "null k_out");
    rd([&](R& r) { r.v = mem + 8; }, INV, "misaligned v_out");
    rd([](R& r) { r.ks = 2 * 128 - 8; }, INV, "k stride");
    rd([](R& r) { r.vs = 2 * 128 + 1; }, INV, "v stride");
    rd([](R& r) { r.ns = 0; }, INV, "no sequences");
    rd([](R& r) { r.v = r.k; }, INV, "one memory for both");
    rd([](R& r) { r.tw = 0; }, INV, "no width");
    std::printf("%d checks, %d failed checks\n", checks, failed);
    return failed != 0;
}
