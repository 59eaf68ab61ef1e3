// Drives the norm, clipping and embedding entry points over a stand-in for the runtime's launch: nothing runs, launches are counted, and one of
// them can be made to fail.  The error of a launch is held until the next launch only, which is all that the library may rely on.  The argument
// names the checks: failures, empty.  Prints what went wrong, or "ok".  Host only: the addresses are invented, and no launch reaches a GPU.
#include <hip/hip_runtime_api.h>

#include <cstdint>
#include <cstdio>
#include <cstring>
#include <functional>
#include <vector>

#include "../include/mqgrad.h"

static int g_launches, g_fail;   // g_fail: the launch that fails, -1 for none
static hipError_t g_last;

extern "C" hipError_t hipLaunchKernel(const void*, dim3, dim3, void**, size_t, hipStream_t) {
    return g_last = g_launches++ == g_fail ? hipErrorLaunchFailure : hipSuccess;
}
extern "C" hipError_t __hipPushCallConfiguration(dim3, dim3, size_t, hipStream_t) { return hipSuccess; }
extern "C" hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* lds, hipStream_t* stream) {
    *grid = *block = dim3(1);
    *lds = 0;
    *stream = nullptr;
    return hipSuccess;
}
extern "C" hipError_t hipGetLastError() {
    const hipError_t e = g_last;
    g_last = hipSuccess;
    return e;
}

static int g_wrong;
static mqg_status with_failure(int at, const std::function<mqg_status()>& call) {
    g_launches = 0;
    g_fail = at;
    g_last = hipSuccess;
    return call();
}
// the call launches `launches` kernels; when one of them fails it says so and launches no more, since what follows reads what that one writes
static void check(const char* what, int launches, const std::function<mqg_status()>& call) {
    const mqg_status st = with_failure(-1, call);
    if (st != MQG_OK || g_launches != launches) {
        std::printf("%s: status %d, %d launches instead of %d\n", what, st, g_launches, launches);
        ++g_wrong;
    }
    for (int k = 0; k < launches; ++k) {
        const mqg_status bad = with_failure(k, call);
        if (bad != MQG_ELAUNCH || g_launches != k + 1) {
            std::printf("%s: launch %d of %d fails: status %d after %d launches\n", what, k, launches, bad, g_launches);
            ++g_wrong;
        }
    }
}

static void* at(uint64_t gigabyte) { return reinterpret_cast<void*>((gigabyte + 1) << 30); }

static mqg_status gradient(uint64_t tokens, uint32_t dim, uint64_t rows, int accumulate) {
    const mqg_rows g = {at(0), tokens, dim, MQG_BFLOAT16}, out = {at(64), rows, dim, MQG_FLOAT32};
    const mqg_tokens ids = {at(128), tokens, MQG_INDEX64, 0, INT64_MIN};
    return mqg_embedding_grad(&g, &ids, dim, 1.0f, &out, accumulate, at(192), nullptr);
}

static void failures() {
    for (int accumulate = 0; accumulate < 2; ++accumulate) {
        check("gradient, no positions", 1 - accumulate, [&] { return gradient(0, 64, 1000, accumulate); });
        check("gradient, direct", 1, [&] { return gradient(100, 64, 1000, accumulate); });
        check("gradient, one-launch sort", 3, [&] { return gradient(9000, 64, 1000, accumulate); });
        check("gradient, one digit", 4, [&] { return gradient(40000, 64, 1000, accumulate); });
        check("gradient, two digits", 6, [&] { return gradient(40000, 64, 100000, accumulate); });
        check("gradient, three digits", 8, [&] { return gradient(40000, 64, 2000000, accumulate); });
    }
    check("lookup", 1, [] {
        const mqg_rows table = {at(0), 1000, 64, MQG_FLOAT32}, out = {at(64), 50, 64, MQG_FLOAT16};
        const mqg_tokens ids = {at(128), 50, MQG_INDEX32, 0, 0};
        return mqg_embedding(&table, &ids, 64, 1.0f, &out, nullptr);
    });
    for (uint32_t count : {10u, 300u}) {
        for (uint64_t n : {1000ull, 10000000ull}) {
            std::vector<mqg_clip_item> items;
            for (uint32_t k = 0; k < count; ++k) items.push_back({at(2 * k), at(2 * k + 1), n, MQG_FLOAT32, MQG_BFLOAT16});
            const int norms = count == 10u ? 1 : 2, clips = count == 10u ? 1 : 3, finish = n == 1000u ? 0 : 1;   // few values: clipping adds the partial sums up
            double* norm = static_cast<double*>(at(1000));
            check("norm", norms + 1, [&] { return mqg_global_norm(items.data(), count, at(1001), norm, nullptr); });
            check("clip by a norm", clips, [&] { return mqg_clip_by_norm(items.data(), count, norm, 1.0, nullptr); });
            check("norm and clip", norms + finish + clips, [&] { return mqg_clip_global_norm(items.data(), count, 1.0, at(1001), norm, nullptr); });
        }
    }
}

// tensors, rows and tokens of which there are none lie over nothing, wherever their addresses point
static void empty() {
    char *scratch = static_cast<char*>(at(10)), *norm = static_cast<char*>(at(11)), *values = static_cast<char*>(at(12)), *out = static_cast<char*>(at(13));
    for (char* inside : {scratch + 64, norm + 4, values + 8, out + 8}) {
        std::vector<mqg_clip_item> items = {{values, out, 1000, MQG_FLOAT32, MQG_FLOAT32}, {inside, inside, 0, MQG_FLOAT32, MQG_BFLOAT16}};
        check("norm with an empty tensor", 2, [&] { return mqg_global_norm(items.data(), 2, scratch, (double*)norm, nullptr); });
        check("clip by a norm with an empty tensor", 1, [&] { return mqg_clip_by_norm(items.data(), 2, (double*)norm, 1.0, nullptr); });
        check("norm and clip with an empty tensor", 2, [&] { return mqg_clip_global_norm(items.data(), 2, 1.0, scratch, (double*)norm, nullptr); });
    }
    check("norm and clip of nothing", 1, [&] { return mqg_clip_global_norm(nullptr, 0, 1.0, norm, (double*)norm, nullptr); });
    check("norm of nothing", 1, [&] { return mqg_global_norm(nullptr, 0, norm, (double*)norm, nullptr); });
    const mqg_rows table = {values, 1000, 64, MQG_FLOAT32};
    for (char* inside : {values + 64, values}) {
        const mqg_rows none = {inside, 0, 64, MQG_FLOAT32};
        const mqg_tokens ids = {inside, 0, MQG_INDEX32, 0, INT64_MIN};
        check("lookup of no tokens", 0, [&] { return mqg_embedding(&table, &ids, 64, 1.0f, &none, nullptr); });
        check("gradient of no positions", 1, [&] { return mqg_embedding_grad(&none, &ids, 64, 1.0f, &table, 0, inside, nullptr); });
        const mqg_rows few = {out, 10, 64, MQG_FLOAT32};   // whose sums take no workspace
        const mqg_tokens tokens = {scratch, 10, MQG_INDEX32, 0, INT64_MIN};
        check("gradient without scratch memory", 1, [&] { return mqg_embedding_grad(&few, &tokens, 64, 1.0f, &table, 0, inside, nullptr); });
    }
}

int main(int argc, char** argv) {
    if (argc == 2 && std::strcmp(argv[1], "failures") == 0) failures();
    else if (argc == 2 && std::strcmp(argv[1], "empty") == 0) empty();
    else return 2;
    if (g_wrong == 0) std::printf("ok\n");
    return g_wrong == 0 ? 0 : 1;
}
