// The key-value cache's host code (argument checks, sizing) on random and on
// wrong arguments, under AddressSanitizer and UndefinedBehaviorSanitizer.  The
// launchers are stubs; a cache is made here by hand, since creating one asks
// for a device.  A call whose arguments are right gets past the checks and
// fails at the device or at the stub (HIP); one whose arguments are wrong must
// not get that far.
#include "../../paper_2510_23346_amd/csrc/bdl_kv_api.cpp"

#include <cstdio>
#include <cstdlib>

namespace bdl {
hipError_t launch_kv_append(const KvAppendArgs&, int, bool, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_kv_attend(const KvAttendArgs&, int, bool, bool, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_kv_evict(const KvEvictArgs&, int, bool, hipStream_t) { return hipErrorNotSupported; }
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
    // sizes against the plain formula, and wrong descriptions
    std::srand(1);
    for (int k = 0; k < 2000; ++k) {
        bdlora_kv_desc d{};
        d.n_kv_heads = 1 + std::rand() % 16;
        d.n_q_heads = d.n_kv_heads * (1 + std::rand() % 64);
        d.head_dim = std::rand() % 2 ? 64 : 128;
        d.page_size = 16 << std::rand() % 13;
        d.n_pages = 1 + std::rand();
        d.max_seqs = 1 + std::rand() % 65535;
        d.format = std::rand() % 2;
        d.k_scale = d.v_scale = d.format ? 0.25f : 1.f;
        const bool fits = d.n_q_heads <= 1024;
        int64_t page = -1, ws = -1, ws0 = -1;
        const int rc = bdlora_kv_bytes(&d, 1, &page, &ws);
        expect(rc, fits ? BDLORA_OK : SH, "kv_bytes");
        if (rc) continue;
        expect(bdlora_kv_bytes(&d, 0, nullptr, &ws0), BDLORA_OK, "kv_bytes without weights");
        const long long entries = (long long)d.n_kv_heads * d.page_size;
        expect(page == entries * (2LL * d.head_dim * (d.format ? 1 : 2) + 8), 1, "page bytes");
        expect(ws - ws0 >= 4LL * d.n_pages * d.page_size * d.n_q_heads, 1, "workspace holds the scores");
        expect(ws0 > 0 && ws0 < (64LL << 20) + 8LL * d.max_seqs * d.n_q_heads, 1, "workspace without weights");
    }
    const bdlora_kv_desc good{8, 2, 128, 64, 100, 16, BDLORA_KV_BF16, 1.f, 1.f};
    auto desc = [&](auto change, int want, const char* what) {
        bdlora_kv_desc d = good;
        change(d);
        expect(bdlora_kv_bytes(&d, 1, nullptr, nullptr), want, what);
        bdlora_kv_t c = nullptr;
        alignas(16) static char mem[16];
        if (want) expect(bdlora_kv_create(&d, mem, mem, nullptr, nullptr, 0, &c), want, what);
    };
    desc([](auto&) {}, BDLORA_OK, "good");
    desc([](auto& d) { d.n_q_heads = 9; }, SH, "heads");
    desc([](auto& d) { d.n_q_heads = 0; }, SH, "no heads");
    desc([](auto& d) { d.n_kv_heads = -1; }, SH, "negative heads");
    desc([](auto& d) { d.head_dim = 96; }, SH, "head size");
    for (int p : {0, -16, 8, 24, 100, 131072}) desc([p](auto& d) { d.page_size = p; }, SH, "page size");
    desc([](auto& d) { d.n_pages = 0; }, INV, "pages");
    desc([](auto& d) { d.max_seqs = 65536; }, INV, "sequences");
    desc([](auto& d) { d.format = 2; }, INV, "format");
    desc([](auto& d) { d.format = 1, d.k_scale = 0.f; }, INV, "scale 0");
    desc([](auto& d) { d.format = 1, d.v_scale = -1.f; }, INV, "negative scale");
    desc([](auto& d) { d.format = 1, d.v_scale = NAN; }, INV, "scale NaN");
    desc([](auto& d) { d.format = 1, d.k_scale = 1e-44f; }, INV, "scale without reciprocal");
    desc([](auto& d) { d.k_scale = 2.f; }, INV, "bf16 with a scale");
    expect(bdlora_kv_bytes(nullptr, 0, nullptr, nullptr), INV, "null description");

    alignas(16) static char mem[4096];
    void* const p = mem;
    int* const i = (int*)mem;
    float* const f = (float*)mem;
    bdlora_kv_t out = (bdlora_kv_t)p;
    expect(bdlora_kv_create(&good, p, p, f, nullptr, 0, &out), INV, "weight without pos");
    expect(out == nullptr, 1, "handle cleared");
    expect(bdlora_kv_create(&good, nullptr, p, nullptr, nullptr, 0, &out), INV, "null k");
    expect(bdlora_kv_create(&good, mem + 8, p, nullptr, nullptr, 0, &out), INV, "misaligned k");
    expect(bdlora_kv_create(&good, p, p, nullptr, nullptr, 0, nullptr), INV, "null handle");
    expect(bdlora_kv_destroy(nullptr), INV, "destroy null");

    bdlora_kv c;
    c.device = 0;
    c.d = good;
    c.k = c.v = mem;
    bdlora_kv w = c;
    w.weight = f;
    w.pos = i;

    // append: one argument wrong at a time
    struct A {
        bdlora_kv_t c;
        const void* qkv; int64_t qs; const float *cos, *sin; int n; const int *s, *ix, *po; int T; const int* t; int64_t ts; int tw, ns;
        int* l; void* q; int64_t os;
    };
    const A a0{&c, p, 12 * 128, f, f, 10, i, i, i, 3, i, 4, 4, 2, i, p, 8 * 128};
    auto app = [&](auto change, int want, const char* what) {
        A a = a0;
        change(a);
        expect(bdlora_kv_append(a.c, a.qkv, a.qs, a.cos, a.sin, a.n, 0, a.s, a.ix, a.po, a.T, a.t, a.ts, a.tw, a.ns, a.l, a.q, a.os, nullptr),
               want, what);
    };
    app([](A&) {}, HIP, "append");
    app([](A& a) { a.T = 0, a.qkv = nullptr; }, BDLORA_OK, "append nothing");
    app([](A& a) { a.l = nullptr; }, HIP, "append without lens");
    app([](A& a) { a.c = nullptr; }, INV, "null cache");
    app([](A& a) { a.T = -1; }, INV, "negative T");
    app([](A& a) { a.qkv = nullptr; }, INV, "null qkv");
    app([&](A& a) { a.qkv = mem + 2; }, INV, "misaligned qkv");
    app([](A& a) { a.qs = 12 * 128 - 8; }, INV, "qkv stride below a row");
    app([](A& a) { a.qs = 12 * 128 + 4; }, INV, "qkv stride");
    app([](A& a) { a.qs = INT64_MAX / 2 * 2; }, INV, "huge stride");
    app([](A& a) { a.os = 8; }, INV, "q_out stride");
    app([&](A& a) { a.q = mem + 8; }, INV, "misaligned q_out");
    app([&](A& a) { a.cos = (float*)(mem + 4); }, INV, "misaligned cos");
    app([](A& a) { a.sin = nullptr; }, INV, "null sin");
    app([](A& a) { a.n = 0; }, INV, "no positions");
    app([](A& a) { a.s = nullptr; }, INV, "null seqs");
    app([&](A& a) { a.ix = (int*)(mem + 2); }, INV, "misaligned index");
    app([](A& a) { a.po = nullptr; }, INV, "null positions");
    app([](A& a) { a.t = nullptr; }, INV, "null table");
    app([](A& a) { a.tw = 0; }, INV, "no width");
    app([](A& a) { a.ts = 3; }, INV, "table stride");
    app([](A& a) { a.ts = a.tw = 1 << 25; }, SH, "more than 2^30 entries");
    app([](A& a) { a.ns = 0; }, INV, "no sequences");

    struct B {
        bdlora_kv_t c;
        const void* q; int64_t qs; int B; const int* t; int64_t ts; int tw; const int *l, *s; float sc; int acc; void* o; int64_t os; float* e;
    };
    const B b0{&w, p, 8 * 128, 3, i, 4, 4, i, i, 0.1f, 1, p, 8 * 128, f};
    auto att = [&](auto change, int want, const char* what) {
        B b = b0;
        change(b);
        expect(bdlora_kv_attend(b.c, b.q, b.qs, b.B, b.t, b.ts, b.tw, b.l, b.s, b.sc, b.acc, b.o, b.os, b.e, nullptr), want, what);
    };
    att([](B&) {}, HIP, "attend");
    att([](B& b) { b.s = nullptr, b.e = nullptr, b.acc = 0; }, HIP, "attend without the optional ones");
    att([](B& b) { b.sc = -1.f; }, HIP, "negative scale");
    att([](B& b) { b.B = 0, b.q = nullptr; }, BDLORA_OK, "attend nothing");
    att([](B& b) { b.c = nullptr; }, INV, "null cache");
    att([&](B& b) { b.c = &c; }, INV, "accumulate without weights");
    att([](B& b) { b.B = 17; }, INV, "more than max_seqs");
    att([](B& b) { b.B = -1; }, INV, "negative B");
    att([](B& b) { b.sc = INFINITY; }, INV, "infinite scale");
    att([](B& b) { b.l = nullptr; }, INV, "null lens");
    att([&](B& b) { b.s = (int*)(mem + 1); }, INV, "misaligned starts");
    att([&](B& b) { b.e = (float*)(mem + 2); }, INV, "misaligned lse");
    att([](B& b) { b.o = nullptr; }, INV, "null out");
    att([](B& b) { b.os = 1000; }, INV, "out stride");
    att([](B& b) { b.qs = 8 * 128 + 1; }, INV, "q stride");
    att([](B& b) { b.tw = 5; }, INV, "width beyond the stride");
    bdlora_kv wide = w;
    wide.d = bdlora_kv_desc{1024, 1024, 64, 65536, 1, 65535, 0, 1.f, 1.f};
    att([&](B& b) { b.c = &wide, b.qs = b.os = 1024 * 64, b.B = 65535; b.ts = b.tw = 16384; }, SH, "more than 2^31 tiles");

    auto ev = [&](bdlora_kv_t cc, int B_, const int* t, int64_t ts, int tw, int* l, int budget, int recent, int want, const char* what) {
        expect(bdlora_kv_evict(cc, B_, t, ts, tw, l, budget, recent, nullptr), want, what);
    };
    ev(&w, 3, i, 4, 4, i, 5, 5, HIP, "evict");
    ev(&w, 0, i, 4, 4, nullptr, 5, 2, BDLORA_OK, "evict nothing");
    ev(&c, 3, i, 4, 4, i, 5, 2, INV, "evict without weights");
    ev(nullptr, 3, i, 4, 4, i, 5, 2, INV, "null cache");
    ev(&w, 17, i, 4, 4, i, 5, 2, INV, "more than max_seqs");
    ev(&w, 3, i, 4, 4, i, 0, 0, INV, "budget 0");
    ev(&w, 3, i, 4, 4, i, 5, 6, INV, "recent beyond the budget");
    ev(&w, 3, i, 4, 4, i, 5, -1, INV, "negative recent");
    ev(&w, 3, nullptr, 4, 4, i, 5, 2, INV, "null table");
    ev(&w, 3, i, 4, 4, nullptr, 5, 2, INV, "null lens");
    int32_t flag = 0;
    expect(bdlora_kv_get_device_error(nullptr, nullptr, &flag), INV, "error of null");
    expect(bdlora_kv_get_device_error(&w, nullptr, nullptr), INV, "null flag");
    std::printf("%d checks, %d failed checks\n", checks, failed);
    return failed != 0;
}
