// Host-side sanitizer run of the operators between two projections: their argument checks, and how the context's attention workspace
// grows and goes.  Built like lifecycle.cpp: this program and api.hip's host code under AddressSanitizer and UndefinedBehaviorSanitizer.
// Exit status 0 = every call as include/gelo.h promises and no report.
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
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
#define HOLDS(what) do { if (!(what)) { std::printf("line %d: not so: %s\n", __LINE__, #what); ++failures; } } while (0)
#define HIP_OK(call) do { hipError_t e_ = (call); if (e_ != hipSuccess) { std::printf("line %d: %s\n", __LINE__, hipGetErrorString(e_)); return 2; } } while (0)

static const int kPages = 512, kPageRows = 16, kWidth = 64, kMostRows = 4096;

struct Buffers {
    float *K, *V, *Q, *O, *QKV, *table;
    int32_t *ints;                                                // kv_len at 0, row_start at 16, page numbers at 64
};

static gelo_kv_cache cache_of(const Buffers& b) {
    return gelo_kv_cache{b.K, b.V, kPages, 1, kPageRows, kWidth, (int64_t)kPageRows * kWidth, (int64_t)kPageRows * kWidth, kWidth};
}
static gelo_seq_batch batch_of(const Buffers& b, int n_seqs, int n_rows, int max_rows, int max_kv_len) {
    return gelo_seq_batch{n_seqs, n_rows, max_rows, max_kv_len, b.ints + 16, b.ints, b.ints + 64, kPages / 2};
}

int main() {
    gelo_ctx* ctx = nullptr;
    EXPECT(gelo_create(&ctx, 0, 1, 0), GELO_OK);
    if (!ctx) { std::printf("no context\n"); return 2; }
    Buffers b;
    HIP_OK(hipMalloc(reinterpret_cast<void**>(&b.K), sizeof(float) * kPages * kPageRows * kWidth));
    HIP_OK(hipMalloc(reinterpret_cast<void**>(&b.V), sizeof(float) * kPages * kPageRows * kWidth));
    HIP_OK(hipMalloc(reinterpret_cast<void**>(&b.Q), sizeof(float) * kMostRows * 2 * kWidth));
    HIP_OK(hipMalloc(reinterpret_cast<void**>(&b.O), sizeof(float) * kMostRows * 2 * kWidth));
    HIP_OK(hipMalloc(reinterpret_cast<void**>(&b.QKV), sizeof(float) * 64 * 4 * kWidth));
    HIP_OK(hipMalloc(reinterpret_cast<void**>(&b.table), sizeof(float) * 64 * kWidth));
    HIP_OK(hipMalloc(reinterpret_cast<void**>(&b.ints), sizeof(int32_t) * (64 + kPages)));
    HIP_OK(hipMemset(b.K, 0, sizeof(float) * kPages * kPageRows * kWidth));
    HIP_OK(hipMemset(b.Q, 0, sizeof(float) * kMostRows * 2 * kWidth));
    HIP_OK(hipMemset(b.QKV, 0, sizeof(float) * 64 * 4 * kWidth));
    std::vector<float> three((size_t)kPages * kPageRows * kWidth, 3.f), out(2 * kWidth);
    HIP_OK(hipMemcpy(b.V, three.data(), sizeof(float) * three.size(), hipMemcpyHostToDevice));
    // two sequences of one row each, 2000 and 5 rows in the cache; sequence s has the pages 256 s ...
    std::vector<int32_t> ints(64 + kPages, 0);
    ints[0] = 2000; ints[1] = 5;
    ints[16] = 0; ints[17] = 1; ints[18] = 2;
    for (int i = 0; i < kPages; ++i) ints[64 + i] = i;
    HIP_OK(hipMemcpy(b.ints, ints.data(), sizeof(int32_t) * ints.size(), hipMemcpyHostToDevice));
    const gelo_kv_cache cache = cache_of(b);
    const gelo_seq_batch two = batch_of(b, 2, 2, 1, 2000), longer = batch_of(b, 2, 2, 1, 4000), padded = batch_of(b, 2, kMostRows, 1, 4000);

    // nothing is enqueued or allocated by a call that is refused
    const int before = mallocs;
    gelo_kv_cache bad_cache = cache;
    gelo_seq_batch bad_batch = two;
    EXPECT(gelo_attention(nullptr, GELO_F32, 2, b.Q, 128, &cache, &two, 1.f, 1, b.O, 128, nullptr), GELO_EINVAL);
    EXPECT(gelo_attention(ctx, GELO_F32, 2, b.Q, 128, nullptr, &two, 1.f, 1, b.O, 128, nullptr), GELO_EINVAL);
    EXPECT(gelo_attention(ctx, GELO_F32, 2, b.Q, 128, &cache, nullptr, 1.f, 1, b.O, 128, nullptr), GELO_EINVAL);
    EXPECT(gelo_attention(ctx, GELO_F32, 2, b.Q, 128, &cache, &two, 1.f, 1, b.Q, 128, nullptr), GELO_EINVAL);      // O over Q
    EXPECT(gelo_attention(ctx, GELO_F32, 0, b.Q, 128, &cache, &two, 1.f, 1, b.O, 128, nullptr), GELO_EINVAL);
    bad_cache.page_rows = 24;
    EXPECT(gelo_attention(ctx, GELO_F32, 2, b.Q, 128, &bad_cache, &two, 1.f, 1, b.O, 128, nullptr), GELO_ESHAPE);
    bad_cache = cache; bad_cache.head_dim = 80; bad_cache.row_stride = 80;
    EXPECT(gelo_attention(ctx, GELO_F32, 2, b.Q, 160, &bad_cache, &two, 1.f, 1, b.O, 160, nullptr), GELO_ESHAPE);
    bad_batch.max_kv_len = INT32_MAX; bad_batch.table_ld = INT32_MAX;
    EXPECT(gelo_attention(ctx, GELO_F32, 2, b.Q, 128, &cache, &bad_batch, 1.f, 1, b.O, 128, nullptr), GELO_ESHAPE);
    bad_batch = two; bad_batch.max_rows = INT32_MAX;
    EXPECT(gelo_attention(ctx, GELO_F32, 2, b.Q, 128, &cache, &bad_batch, 1.f, 1, b.O, 128, nullptr), GELO_ESHAPE);
    EXPECT(gelo_reserve_attention(nullptr, 64), GELO_EINVAL);
    EXPECT(gelo_reserve_attention(ctx, 65), GELO_ESHAPE);
    EXPECT(gelo_rope_append(ctx, GELO_F32, 2, b.QKV, 256, &cache, nullptr, GELO_ROPE_HALF, 0, nullptr, 0, b.Q, 128, nullptr), GELO_EINVAL);
    EXPECT(gelo_rope_append(ctx, GELO_F32, 2, b.QKV, 256, &cache, &two, GELO_ROPE_HALF, 64, b.table, 1999, b.Q, 128, nullptr), GELO_ESHAPE);
    EXPECT(gelo_rope_append(ctx, GELO_F32, INT32_MAX, b.QKV, 256, &cache, &two, GELO_ROPE_HALF, 0, nullptr, 0, b.Q, 128, nullptr), GELO_ESHAPE);
    EXPECT(gelo_rope_append(ctx, GELO_F32, 2, b.QKV, 256, &cache, &two, GELO_ROPE_HALF, 0, nullptr, 0, b.QKV + 64, 256, nullptr), GELO_EINVAL);
    EXPECT(gelo_rope_table(ctx, 64, 0, INT32_MAX, 1e4, 1.0, 0.0, 1.0, 4.0, b.table, nullptr), GELO_ESHAPE);
    EXPECT(gelo_rope_table(ctx, 64, INT32_MAX, 1, 1e4, 1.0, 0.0, 1.0, 4.0, b.table, nullptr), GELO_EINVAL);
    EXPECT(gelo_rms_norm(ctx, GELO_F32, INT32_MAX, 64, b.Q, 64, nullptr, 0, b.table, 1e-5f, nullptr, 0, b.O, 64, nullptr, 0, nullptr, nullptr), GELO_ESHAPE);
    EXPECT(gelo_rms_norm(ctx, GELO_F32, (1 << 21) + 1, 8200, b.Q, 8200, nullptr, 0, b.table, 1e-5f, nullptr, 0, b.O, 8200, nullptr, 0, nullptr, nullptr), GELO_ESHAPE);
    EXPECT(gelo_rms_norm(ctx, GELO_F32, 4, 64, b.Q, 64, nullptr, 0, b.table, 1e-5f, b.O, 64, b.O, 64, nullptr, 0, nullptr, nullptr), GELO_EINVAL);
    EXPECT(gelo_project_fp8_codes(ctx, 4, 128, 8, nullptr, 128, b.table, b.QKV, b.O, 8, nullptr), GELO_EINVAL);
    EXPECT(gelo_project_fp8_codes(ctx, 4, 100, 8, reinterpret_cast<uint8_t*>(b.QKV), 128, b.table, b.QKV, b.O, 8, nullptr), GELO_ESHAPE);
    HOLDS(mallocs == before && frees == 0);

    // the first call that cuts its cache allocates, a larger one grows what there is, and a smaller one uses it
    auto attend = [&](gelo_ctx* c, const gelo_seq_batch& batch) { return gelo_attention(c, GELO_F32, 2, b.Q, 128, &cache, &batch, 1.f, 1, b.O, 128, nullptr); };
    const gelo_seq_batch whole = batch_of(b, 2, 2, 1, 64);
    EXPECT(attend(ctx, whole), GELO_OK);
    HOLDS(mallocs == before);
    malloc_most = 256;                                             // not enough: no call, and no harm
    EXPECT(attend(ctx, two), GELO_ENOMEM);
    malloc_most = SIZE_MAX;
    HOLDS(mallocs == before);
    EXPECT(attend(ctx, two), GELO_OK);
    HOLDS(mallocs == before + 1 && frees == 0);
    EXPECT(attend(ctx, longer), GELO_OK);
    HOLDS(mallocs == before + 2 && frees == 1);
    EXPECT(attend(ctx, two), GELO_OK);
    EXPECT(attend(ctx, padded), GELO_OK);                          // rows of no sequence take none of it
    HOLDS(mallocs == before + 2 && frees == 1);
    HIP_OK(hipDeviceSynchronize());
    for (int row = 0; row < 2; ++row) {                            // equal weights of equal values
        HIP_OK(hipMemcpy(out.data(), b.O + row * 2 * kWidth, sizeof(float) * out.size(), hipMemcpyDeviceToHost));
        for (float x : out) HOLDS(x > 2.999f && x < 3.001f);
    }
    // what was reserved is enough for every width up to its own and every batch, and stays where it is
    EXPECT(gelo_reserve_attention(ctx, 256), GELO_OK);
    HOLDS(mallocs == before + 3 && frees == 2);
    EXPECT(gelo_reserve_attention(ctx, 64), GELO_OK);
    EXPECT(attend(ctx, two), GELO_OK);
    EXPECT(attend(ctx, longer), GELO_OK);
    EXPECT(attend(ctx, padded), GELO_OK);
    EXPECT(gelo_rope_append(ctx, GELO_F32, 2, b.QKV, 256, &cache, &two, GELO_ROPE_HALF, 0, nullptr, 0, b.Q, 128, nullptr), GELO_OK);
    EXPECT(gelo_rope_append(ctx, GELO_F32, 2, b.QKV, 256, &cache, &two, GELO_ROPE_HALF, 0, nullptr, 0, b.QKV, 256, nullptr), GELO_OK);
    EXPECT(gelo_rope_table(ctx, 64, 0, 64, 1e4, 1.0, 0.0, 1.0, 4.0, b.table, nullptr), GELO_OK);
    EXPECT(gelo_rms_norm(ctx, GELO_F32, 4, 64, b.Q, 64, nullptr, 0, b.table, 1e-5f, nullptr, 0, b.O, 64, nullptr, 0, nullptr, nullptr), GELO_OK);
    HOLDS(mallocs == before + 3 && frees == 2);
    HIP_OK(hipDeviceSynchronize());
    // a context of its own holds a workspace of its own, and both go with their contexts
    gelo_ctx* other = nullptr;
    EXPECT(gelo_create(&other, 0, 2, 0), GELO_OK);
    const int made = mallocs, gone = frees;
    EXPECT(attend(other, two), GELO_OK);
    HOLDS(mallocs == made + 1);
    EXPECT(gelo_destroy(other), GELO_OK);
    HOLDS(frees > gone);
    EXPECT(attend(ctx, two), GELO_OK);
    HIP_OK(hipDeviceSynchronize());
    const int left = frees;
    EXPECT(gelo_destroy(ctx), GELO_OK);
    HOLDS(frees > left);
    HIP_OK(hipFree(b.K)); HIP_OK(hipFree(b.V)); HIP_OK(hipFree(b.Q)); HIP_OK(hipFree(b.O));
    HIP_OK(hipFree(b.QKV)); HIP_OK(hipFree(b.table)); HIP_OK(hipFree(b.ints));
    std::printf(failures ? "%d expectation(s) failed\n" : "layer: all calls as promised\n", failures);
    return failures ? 1 : 0;
}
