// Host-side sanitizer run of adapters at the ends of what a call may say, numbers of rows that leave 32 bits once anything is added to them, and of what a device has, memory
// for the workspace that a call needs and not for more.  Built like lifecycle.cpp: this program and api.hip's host code under AddressSanitizer and UndefinedBehaviorSanitizer.
// Exit status 0 = every call as include/gelo.h promises and no report.
#include <cstdint>
#include <cstdio>
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

static const int kD = 1024, kP = 1024, kRank = 16, kRows = 64;

int main() {
    gelo_ctx* ctx = nullptr;
    EXPECT(gelo_create(&ctx, 0, 1, 0), GELO_OK);
    if (!ctx) { std::printf("no context\n"); return 2; }
    float *X, *A, *B;                                             // H and Z side by side in the rows of X
    int32_t* which;
    HIP_OK(hipMalloc(reinterpret_cast<void**>(&X), sizeof(float) * kRows * (kD + kP)));
    HIP_OK(hipMalloc(reinterpret_cast<void**>(&A), sizeof(float) * kRank * kD));
    HIP_OK(hipMalloc(reinterpret_cast<void**>(&B), sizeof(float) * kP * kRank));
    HIP_OK(hipMalloc(reinterpret_cast<void**>(&which), sizeof(int32_t) * kRows));
    HIP_OK(hipMemset(X, 0, sizeof(float) * kRows * (kD + kP)));
    HIP_OK(hipMemset(A, 0, sizeof(float) * kRank * kD));
    HIP_OK(hipMemset(B, 0, sizeof(float) * kP * kRank));
    HIP_OK(hipMemset(which, 0, sizeof(int32_t) * kRows));
    gelo_adapters adapters{A, B, nullptr, 1, kRank, 1, {kP}, 0, kD, 0, kRank};
    auto adapt = [&](gelo_dtype type, int n, int count) {
        adapters.n_adapters = count;                              // (a stride of 0: all of them are the one)
        float* Z = X + (type == GELO_F32 ? kD : kD / 2);
        return gelo_adapt(ctx, type, n, kD, kP, X, kD + kP, &adapters, which, Z, kD + kP, Z, kD + kP, nullptr);
    };
    for (gelo_dtype type : {GELO_F32, GELO_BF16})
        for (int count : {1, 20, 12287, 12288, INT32_MAX})
            for (int under : {0, 14, 15, 30, 31, 61, 62, 63, 64, 1 << 30}) EXPECT(adapt(type, INT32_MAX - under, count), GELO_ESHAPE);
    EXPECT(adapt(GELO_F32, kRows, 1), GELO_OK);

    // -------------------------------------------------------------------------------- workspaces on a device that is nearly full
    const int first_rows = 20000, more = 64, times = 200;
    EXPECT(gelo_reserve_adapt(ctx, first_rows, kRank, 1, 1), GELO_OK);
    HIP_OK(hipDeviceSynchronize());
    int made = mallocs, gone = frees;
    malloc_most = (size_t)2 << 20;                                // (20000 rows take 1.4 MB, 26400 1.8: never room for twice what there is)
    for (int i = 1; i <= times / 2; ++i) {
        EXPECT(gelo_reserve_adapt(ctx, first_rows + i * more, kRank, 1, 1), GELO_OK);
        HOLDS(mallocs == made + i && frees == gone);              // what was there stays
    }
    EXPECT(gelo_reserve_adapt(ctx, first_rows, kRank, 1, 1), GELO_OK);
    EXPECT(adapt(GELO_F32, kRows, 1), GELO_OK);
    HOLDS(mallocs == made + times / 2);
    EXPECT(gelo_reserve_adapt(ctx, 2 * first_rows, kRank, 1, 1), GELO_ENOMEM);
    EXPECT(adapt(GELO_F32, kRows, 1), GELO_OK);                   // and no harm
    malloc_most = SIZE_MAX;
    EXPECT(gelo_reserve_adapt(ctx, first_rows + (times / 2 + 1) * more, kRank, 1, 1), GELO_OK);
    made = mallocs;
    EXPECT(gelo_reserve_adapt(ctx, 2 * (first_rows + times / 2 * more), kRank, 1, 1), GELO_OK);      // (twice as much, where there is room)
    HOLDS(mallocs == made && frees == gone);
    HIP_OK(hipDeviceSynchronize());
    EXPECT(gelo_destroy(ctx), GELO_OK);
    HOLDS(frees >= gone + times / 2 + 2);
    for (void* p : {(void*)X, (void*)A, (void*)B, (void*)which}) HIP_OK(hipFree(p));
    if (failures) { std::printf("%d expectation(s) failed\n", failures); return 1; }
    std::printf("all calls as promised\n");
    return 0;
}
