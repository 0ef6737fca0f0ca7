// Host-side sanitizer run of adapters and the cache of 4 bits: their argument checks at the ends of their types, and how the context's workspaces grow, are kept
// and go.  Built like lifecycle.cpp: this program and api.hip's host code under AddressSanitizer and UndefinedBehaviorSanitizer.
// Exit status 0 = every call as include/gelo.h promises and no report.
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <vector>
#include <dlfcn.h>
#include <hip/hip_runtime.h>
#include "gelo.h"

// The library's device allocations come through here: none of more than `malloc_most` bytes succeeds.
static size_t malloc_most = SIZE_MAX;
static int mallocs = 0, frees = 0;
extern "C" hipError_t hipMalloc(void** ptr, size_t size) {
    static const auto real = reinterpret_cast<hipError_t (*)(void**, size_t)>(dlsym(RTLD_NEXT, "hipMalloc"));
    if (size > malloc_most) { *ptr = nullptr; return hipErrorOutOfMemory; }
    ++mallocs;
    return real(ptr, size);
}
extern "C" hipError_t hipFree(void* ptr) {
    static const auto real = reinterpret_cast<hipError_t (*)(void*)>(dlsym(RTLD_NEXT, "hipFree"));
    ++frees;
    return real(ptr);
}

static int failures = 0;
#define EXPECT(call, want) do { gelo_status got_ = (call); if (got_ != (want)) { \
    std::printf("line %d: %s -> %s, expected %s\n", __LINE__, #call, gelo_status_string(got_), gelo_status_string(want)); ++failures; } } while (0)
#define REFUSED(call) do { gelo_status got_ = (call); if (got_ == GELO_OK) { std::printf("line %d: %s accepted\n", __LINE__, #call); ++failures; } } while (0)
#define HOLDS(what) do { if (!(what)) { std::printf("line %d: not so: %s\n", __LINE__, #what); ++failures; } } while (0)
#define HIP_OK(call) do { hipError_t e_ = (call); if (e_ != hipSuccess) { std::printf("line %d: %s\n", __LINE__, hipGetErrorString(e_)); return 2; } } while (0)

static const int kPages = 512, kPageRows = 16, kWidth = 64, kPiece = 17 * kPageRows * kWidth / 32;
static const int kD = 1024, kP = 512, kRank = 16, kRows = 4096, kAdapters = 3;

int main() {
    gelo_ctx* ctx = nullptr;
    EXPECT(gelo_create(&ctx, 0, 1, 0), GELO_OK);
    if (!ctx) { std::printf("no context\n"); return 2; }
    uint8_t *K, *V;
    float *H, *Z, *A, *B, *Q, *O;
    int32_t *ints, *which;                                        // kv_len at 0, row_start at 16, page numbers at 64
    HIP_OK(hipMalloc(reinterpret_cast<void**>(&K), (size_t)kPages * kPiece));
    HIP_OK(hipMalloc(reinterpret_cast<void**>(&V), (size_t)kPages * kPiece));
    HIP_OK(hipMalloc(reinterpret_cast<void**>(&H), sizeof(float) * kRows * kD));
    HIP_OK(hipMalloc(reinterpret_cast<void**>(&Z), sizeof(float) * kRows * kP));
    HIP_OK(hipMalloc(reinterpret_cast<void**>(&A), sizeof(float) * kAdapters * kRank * kD));
    HIP_OK(hipMalloc(reinterpret_cast<void**>(&B), sizeof(float) * kAdapters * kP * kRank));
    HIP_OK(hipMalloc(reinterpret_cast<void**>(&Q), sizeof(float) * 64 * 4 * kWidth));
    HIP_OK(hipMalloc(reinterpret_cast<void**>(&O), sizeof(float) * 64 * 4 * kWidth));
    HIP_OK(hipMalloc(reinterpret_cast<void**>(&ints), sizeof(int32_t) * (64 + kPages)));
    HIP_OK(hipMalloc(reinterpret_cast<void**>(&which), sizeof(int32_t) * kRows));
    HIP_OK(hipMemset(K, 0, (size_t)kPages * kPiece));
    HIP_OK(hipMemset(V, 0, (size_t)kPages * kPiece));
    HIP_OK(hipMemset(H, 0, sizeof(float) * kRows * kD));
    HIP_OK(hipMemset(Z, 0, sizeof(float) * kRows * kP));
    HIP_OK(hipMemset(A, 0, sizeof(float) * kAdapters * kRank * kD));
    HIP_OK(hipMemset(B, 0, sizeof(float) * kAdapters * kP * kRank));
    HIP_OK(hipMemset(Q, 0, sizeof(float) * 64 * 4 * kWidth));
    std::vector<int32_t> host(64 + kPages, 0);
    host[0] = 2000; host[1] = 1500; host[17] = 1; host[18] = 2;
    for (int i = 0; i < kPages; ++i) host[64 + i] = i;
    HIP_OK(hipMemcpy(ints, host.data(), sizeof(int32_t) * host.size(), hipMemcpyHostToDevice));
    std::vector<int32_t> numbers(kRows);
    for (int i = 0; i < kRows; ++i) numbers[i] = i % 5 - 1;       // none's and beyond the last among them
    HIP_OK(hipMemcpy(which, numbers.data(), sizeof(int32_t) * kRows, hipMemcpyHostToDevice));
    const int before = mallocs, gone = frees;

    // ------------------------------------------------------------------------------------------------ the cache
    const gelo_kv_cache_fp4 cache{K, V, kPages, 1, kPageRows, kWidth, kPiece, kPiece};
    const gelo_seq_batch two{2, 2, 1, 2048, ints + 16, ints, ints + 64, kPages / 2}, longer{2, 2, 1, 4096, ints + 16, ints, ints + 64, kPages / 2};
    size_t bytes = 1;
    EXPECT(gelo_fp4_page_bytes(kPageRows, kWidth, &bytes), GELO_OK);
    HOLDS(bytes == (size_t)kPiece);
    EXPECT(gelo_fp4_page_bytes(kPageRows, kWidth, nullptr), GELO_EINVAL);
    for (int bad : {0, -16, INT32_MIN, 8, 17, 24, INT32_MAX, 1 << 30}) REFUSED(gelo_fp4_page_bytes(bad, kWidth, &bytes));
    for (int bad : {0, -32, INT32_MIN, 16, 33, INT32_MAX, 1 << 30}) REFUSED(gelo_fp4_page_bytes(kPageRows, bad, &bytes));
    auto attend = [&](const gelo_kv_cache_fp4* c, const gelo_seq_batch* b, int heads = 2, int64_t ld = 128, float scale = 1.f, void* to = nullptr) {
        return gelo_attention_fp4(ctx, GELO_F32, heads, Q, ld, c, b, scale, 1, to ? to : O, ld, nullptr);
    };
    auto append = [&](const gelo_kv_cache_fp4* c, const gelo_seq_batch* b, int heads = 2, int64_t ld = 256) {
        return gelo_rope_append_fp4(ctx, GELO_F32, heads, Q, ld, c, b, GELO_ROPE_HALF, 0, nullptr, 0, O, 128, nullptr);
    };
    auto read = [&](const gelo_kv_cache_fp4* c, const gelo_seq_batch* b, void* k, void* v, int64_t ld = 64) {
        return gelo_cache_rows_fp4(ctx, GELO_F32, c, b, k, ld, v, ld, nullptr);
    };
    EXPECT(gelo_attention_fp4(nullptr, GELO_F32, 2, Q, 128, &cache, &two, 1.f, 1, O, 128, nullptr), GELO_EINVAL);
    EXPECT(gelo_rope_append_fp4(nullptr, GELO_F32, 2, Q, 256, &cache, &two, GELO_ROPE_HALF, 0, nullptr, 0, O, 128, nullptr), GELO_EINVAL);
    EXPECT(gelo_cache_rows_fp4(nullptr, GELO_F32, &cache, &two, Q, 64, nullptr, 0, nullptr), GELO_EINVAL);
    EXPECT(read(&cache, &two, nullptr, nullptr), GELO_EINVAL);
    EXPECT(read(&cache, &two, O, O), GELO_EINVAL);
    EXPECT(attend(&cache, &two, 2, 128, 1.f, Q), GELO_EINVAL);
    EXPECT(attend(&cache, &two, 2, 128, __builtin_inff()), GELO_EINVAL);
    for (int i = 0; i < 12; ++i) {
        gelo_kv_cache_fp4 c = cache;
        switch (i) {
            case 0: c.k = nullptr; break;
            case 1: c.v = nullptr; break;
            case 2: c.v = V + 8; break;
            case 3: c.n_pages = 0; break;
            case 4: c.n_kv_heads = INT32_MAX; break;
            case 5: c.page_rows = 24; break;
            case 6: c.page_rows = INT32_MIN; break;
            case 7: c.head_dim = INT32_MAX; break;
            case 8: c.page_stride = kPiece - 16; break;
            case 9: c.page_stride = INT64_MAX - 15; break;
            case 10: c.page_stride = INT64_MIN; break;
            case 11: c.page_stride = kPiece + 8; break;
        }
        REFUSED(attend(&c, &two));
        REFUSED(append(&c, &two));
        REFUSED(read(&c, &two, O, nullptr));
    }
    for (int i = 0; i < 8; ++i) {
        gelo_seq_batch b = two;
        switch (i) {
            case 0: b.n_seqs = 0; break;
            case 1: b.n_rows = 0; break;
            case 2: b.max_kv_len = 0; break;
            case 3: b.max_kv_len = INT32_MAX; break;
            case 4: b.table_ld = 1; break;
            case 5: b.kv_len = nullptr; break;
            case 6: b.page_table = nullptr; break;
            case 7: b.n_rows = INT32_MIN; break;
        }
        REFUSED(attend(&cache, &b));
        REFUSED(append(&cache, &b));
        REFUSED(read(&cache, &b, O, nullptr));
    }
    REFUSED(attend(nullptr, &two));
    REFUSED(attend(&cache, nullptr));
    for (int bad : {0, -1, INT32_MIN, INT32_MAX}) REFUSED(attend(&cache, &two, bad));
    for (int bad : {-1, INT32_MIN, INT32_MAX}) REFUSED(append(&cache, &two, bad));
    for (int64_t bad : {(int64_t)0, (int64_t)-128, (int64_t)INT64_MIN, (int64_t)INT64_MAX}) { REFUSED(attend(&cache, &two, 2, bad)); REFUSED(append(&cache, &two, 2, bad)); REFUSED(read(&cache, &two, O, nullptr, bad)); }
    HOLDS(mallocs == before && frees == gone);

    // ------------------------------------------------------------------------------------------------ adapters
    gelo_adapters adapters{A, B, nullptr, kAdapters, kRank, 1, {kP}, (int64_t)kRank * kD, kD, (int64_t)kP * kRank, kRank};
    auto adapt = [&](const gelo_adapters& a, int n = 4, int d = kD, int p = kP, int64_t ldh = kD, int64_t ldz = kP, float* to = nullptr) {
        return gelo_adapt(ctx, GELO_F32, n, d, p, H, ldh, &a, which, Z, kP, to ? to : Z, ldz, nullptr);
    };
    EXPECT(gelo_adapt(nullptr, GELO_F32, 4, kD, kP, H, kD, &adapters, which, Z, kP, Z, kP, nullptr), GELO_EINVAL);
    EXPECT(gelo_adapt(ctx, GELO_F32, 4, kD, kP, H, kD, nullptr, which, Z, kP, Z, kP, nullptr), GELO_EINVAL);
    EXPECT(gelo_adapt(ctx, GELO_F32, 4, kD, kP, H, kD, &adapters, nullptr, Z, kP, Z, kP, nullptr), GELO_EINVAL);
    EXPECT(adapt(adapters, 4, kD, kP, kD, kP, H), GELO_EINVAL);
    EXPECT(adapt(adapters, 4, kD, kP, kD, kP, Z + 16), GELO_EINVAL);
    for (int i = 0; i < 17; ++i) {
        gelo_adapters a = adapters;
        switch (i) {
            case 0: a.a = nullptr; break;
            case 1: a.b = nullptr; break;
            case 2: a.n_adapters = 0; break;
            case 3: a.n_adapters = INT32_MIN; break;
            case 4: a.rank = 12; break;
            case 5: a.rank = INT32_MAX; break;
            case 6: a.rank = 136; break;
            case 7: a.n_parts = 0; break;
            case 8: a.n_parts = INT32_MAX; break;
            case 9: a.part_end[0] = kP - 16; break;
            case 10: a.n_parts = 2; a.part_end[0] = 8; a.part_end[1] = kP; break;
            case 11: a.n_parts = 2; a.part_end[0] = kP; a.part_end[1] = kP; break;
            case 12: a.a_stride = -8; break;
            case 13: a.b_stride = INT64_MAX; break;
            case 14: a.lda = kD - 8; break;
            case 15: a.ldb = INT64_MAX - 7; break;
            case 16: a.a = A + 1; break;
        }
        REFUSED(adapt(a));
    }
    for (int bad : {0, -1, INT32_MIN}) { REFUSED(adapt(adapters, bad)); REFUSED(adapt(adapters, 4, bad)); REFUSED(adapt(adapters, 4, kD, bad)); }
    for (int bad : {INT32_MAX, INT32_MAX - 7, kD + 4}) { REFUSED(adapt(adapters, 4, bad)); REFUSED(adapt(adapters, 4, kD, bad)); }
    for (int64_t bad : {(int64_t)0, (int64_t)-8, (int64_t)INT64_MIN, (int64_t)INT64_MAX, (int64_t)kP - 8}) { REFUSED(adapt(adapters, 4, kD, kP, bad)); REFUSED(adapt(adapters, 4, kD, kP, kD, bad)); }
    for (int bad : {0, -8, 4, 136, INT32_MAX, INT32_MIN}) REFUSED(gelo_reserve_adapt(ctx, 4, bad, 1, 1));
    for (int bad : {0, -1, 5, INT32_MAX}) REFUSED(gelo_reserve_adapt(ctx, 4, 16, bad, 1));
    for (int bad : {0, -1, INT32_MIN}) { REFUSED(gelo_reserve_adapt(ctx, bad, 16, 1, 1)); REFUSED(gelo_reserve_adapt(ctx, 4, 16, 1, bad)); }
    EXPECT(gelo_reserve_adapt(nullptr, 4, 16, 1, 1), GELO_EINVAL);
    HOLDS(mallocs == before && frees == gone);
    malloc_most = 64;                                             // not enough: no call, and no harm
    EXPECT(adapt(adapters), GELO_ENOMEM);
    EXPECT(gelo_reserve_adapt(ctx, INT32_MAX, 128, 4, INT32_MAX), GELO_ENOMEM);
    malloc_most = SIZE_MAX;
    HOLDS(mallocs == before && frees == gone);

    // ------------------------------------------------------------------------------------------------ workspaces
    EXPECT(adapt(adapters), GELO_OK);
    HOLDS(mallocs == before + 1 && frees == gone);
    EXPECT(adapt(adapters, kRows), GELO_OK);                      // more: what was there stays
    HOLDS(mallocs == before + 2 && frees == gone);
    EXPECT(adapt(adapters), GELO_OK);
    EXPECT(attend(&cache, &two), GELO_OK);
    HOLDS(mallocs == before + 3 && frees == gone);
    EXPECT(attend(&cache, &longer), GELO_OK);
    HOLDS(mallocs == before + 4 && frees == gone);
    EXPECT(gelo_reserve_attention(ctx, 256), GELO_OK);
    HOLDS(mallocs == before + 5 && frees == gone);
    EXPECT(attend(&cache, &longer), GELO_OK);
    EXPECT(append(&cache, &two), GELO_OK);
    EXPECT(read(&cache, &two, O, O + 128), GELO_OK);
    HOLDS(mallocs == before + 5 && frees == gone);
    HIP_OK(hipDeviceSynchronize());
    EXPECT(gelo_reserve_adapt(ctx, 64, 128, 4, 64), GELO_OK);
    const int made = mallocs;
    gelo_adapters wide = adapters;
    wide.rank = 8;
    for (int n : {1, 2, 3, 16, 17, 63, 64}) EXPECT(adapt(wide, n), GELO_OK);
    HOLDS(mallocs == made);
    HIP_OK(hipDeviceSynchronize());
    const int left = frees;
    EXPECT(gelo_destroy(ctx), GELO_OK);
    HOLDS(frees >= left + 5);                                     // two of adapters', three of attention's at least

    for (void* p : {(void*)K, (void*)V, (void*)H, (void*)Z, (void*)A, (void*)B, (void*)Q, (void*)O, (void*)ints, (void*)which}) HIP_OK(hipFree(p));
    if (failures) { std::printf("%d expectation(s) failed\n", failures); return 1; }
    std::printf("all calls as promised\n");
    return 0;
}
