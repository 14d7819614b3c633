// Host-only driver of the operators on a routed batch (tests/test_ops_host_cpu.py
// builds and runs it).  The HIP runtime functions that they call are defined here, in
// the executable, and so take the place of the runtime's: memory is an address without
// anything behind it, kernels are recorded by name and grid and not run.
//
//   ops_path <scenario>        prints "ok", or the failed checks (exit 1)
#include <hip/hip_runtime_api.h>

#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <string>
#include <vector>

#include "hwr_ops.h"

namespace {

struct Launch {
    std::string kernel;
    dim3 grid, block;
    int device;
};
std::vector<Launch> g_log;
std::map<const void *, std::string> &kernels() {      // registered before main
    static std::map<const void *, std::string> m;
    return m;
}
std::map<uintptr_t, size_t> g_mem;
uintptr_t g_next = uintptr_t(1) << 40;
int g_mallocs = 0;
size_t g_fail = SIZE_MAX;         // allocations of this many bytes or more fail
bool g_capturing = false;
hipError_t g_error = hipSuccess;  // the last error: stays until it is asked for
int g_device = 0, g_wrong_device = 0;     // current; calls made on another than the context's
int g_context_device = 0;
dim3 g_grid, g_block;
size_t g_shm;
hipStream_t g_stream;

hipError_t launch(const void *f, dim3 grid, dim3 block) {
    g_log.push_back({kernels()[f], grid, block, g_device});
    g_wrong_device += g_device != g_context_device;
    return hipSuccess;
}

}  // namespace

extern "C" {
void **__hipRegisterFatBinary(const void *) {
    static void *h;
    return &h;
}
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *host, char *, const char *name, unsigned, void *, void *, void *, void *, int *) {
    kernels()[host] = name;
}
void __hipRegisterVar(void **, void *, char *, char *, int, size_t, int, int) {}
hipError_t __hipPushCallConfiguration(dim3 g, dim3 b, size_t shm, hipStream_t s) {
    g_grid = g, g_block = b, g_shm = shm, g_stream = s;
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3 *g, dim3 *b, size_t *shm, hipStream_t *s) {
    *g = g_grid, *b = g_block, *shm = g_shm, *s = g_stream;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void *f, dim3 grid, dim3 block, void **, size_t, hipStream_t) { return launch(f, grid, block); }
hipError_t hipExtLaunchKernel(const void *f, dim3 grid, dim3 block, void **, size_t, hipStream_t, hipEvent_t, hipEvent_t, int) {
    return launch(f, grid, block);
}
hipError_t hipMalloc(void **p, size_t n) {
    ++g_mallocs;
    g_wrong_device += g_device != g_context_device;
    if (n >= g_fail) return g_error = hipErrorOutOfMemory;
    g_mem[g_next] = n;
    *p = reinterpret_cast<void *>(g_next);
    g_next += (n + 4095) / 4096 * 4096 + 4096;
    return hipSuccess;
}
hipError_t hipFree(void *p) {
    g_mem.erase(reinterpret_cast<uintptr_t>(p));
    g_wrong_device += g_device != g_context_device;
    return hipSuccess;
}
hipError_t hipMemset(void *, int, size_t) { return hipSuccess; }
hipError_t hipDeviceSynchronize() { return hipSuccess; }
hipError_t hipGetDeviceCount(int *n) { return *n = 2, hipSuccess; }
hipError_t hipGetDevice(int *d) { return *d = g_device, hipSuccess; }
hipError_t hipSetDevice(int d) { return g_device = d, hipSuccess; }
hipError_t hipGetDevicePropertiesR0600(hipDeviceProp_tR0600 *p, int) {
    *p = {};
    std::strcpy(p->gcnArchName, "gfx950");
    p->multiProcessorCount = 256;
    return hipSuccess;
}
const char *hipGetErrorName(hipError_t) { return "error"; }
const char *hipGetErrorString(hipError_t) { return "injected"; }
hipError_t hipGetLastError() {
    const hipError_t e = g_error;
    g_error = hipSuccess;
    return e;
}
hipError_t hipStreamSynchronize(hipStream_t) { return hipSuccess; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus *c) {
    *c = g_capturing ? hipStreamCaptureStatusActive : hipStreamCaptureStatusNone;
    return hipSuccess;
}
}

namespace {

int g_bad = 0;
void check(bool ok, const std::string &what) {
    if (!ok) {
        std::printf("FAIL %s\n", what.c_str());
        ++g_bad;
    }
}

// Addresses that stand for matrices far apart
template <class T>
T *at(int i) {
    return reinterpret_cast<T *>((uintptr_t(2) << 44) + (uintptr_t(i) << 40));
}

// A context, and the five operators on matrices of given sizes.
struct Rig {
    hwr_ops *ops = nullptr;
    int dtype = HWR_BF16, n = 0, G = 1, k = 8, m = 8, rank = 4;

    explicit Rig(int device = 0) { check(hwr_ops_init(device, reinterpret_cast<void *>(0x1000), &ops) == HWR_OK, "init"); }
    ~Rig() { hwr_ops_free(ops); }
    hwr_groups groups() const { return {n, G, at<int32_t>(0), at<int32_t>(1)}; }
    hwr_status group() { return hwr_group_rows(ops, n, at<int32_t>(2), nullptr, 0, G, at<int32_t>(0), at<int32_t>(1)); }
    hwr_status matmul() {
        const hwr_groups g = groups();
        const hwr_matmul_args a{dtype, k, m, at<char>(3), 0, at<char>(4), at<char>(5), 0};
        return hwr_grouped_matmul(ops, &g, &a);
    }
    hwr_status matmul_grad(bool dx = true, bool dw = true) {
        const hwr_groups g = groups();
        const hwr_matmul_grad_args a{dtype, k, m, at<char>(5), 0, at<char>(3), 0, at<char>(4), dx ? at<char>(6) : nullptr, 0,
                                     dw ? at<char>(7) : nullptr};
        return hwr_grouped_matmul_grad(ops, &g, &a);
    }
    hwr_status adapter() {
        const hwr_groups g = groups();
        const hwr_adapter_args a{dtype, k, m, rank, at<char>(3), 0, at<char>(4), at<char>(8), at<char>(9), nullptr, at<char>(5), 0};
        return hwr_adapter_matmul(ops, &g, &a);
    }
    hwr_status adapter_grad(bool dx = true, bool da = true, bool db = true) {
        const hwr_groups g = groups();
        const hwr_adapter_grad_args a{dtype, k, m, rank, at<char>(5), 0, at<char>(3), 0, at<char>(4), at<char>(8), at<char>(9), nullptr,
                                      dx ? at<char>(6) : nullptr, 0, da ? at<char>(10) : nullptr, db ? at<char>(11) : nullptr};
        return hwr_adapter_matmul_grad(ops, &g, &a);
    }
};

constexpr int kMaxRows = INT32_MAX - 511;

// Places are counted in 32 bits, up to a few tiles past the last: a batch with fewer
// than 512 rows to 2^31 is refused, and nothing is launched.
void row_limit() {
    Rig r;
    r.k = r.m = 1, r.rank = 1;
    for (int n : {kMaxRows + 1, INT32_MAX}) {
        r.n = n;
        g_log.clear();
        check(r.matmul() == HWR_ERR_INVALID_ARG, "matmul of " + std::to_string(n) + " rows");
        check(r.matmul_grad() == HWR_ERR_INVALID_ARG, "matmul_grad of " + std::to_string(n) + " rows");
        check(r.adapter() == HWR_ERR_INVALID_ARG, "adapter of " + std::to_string(n) + " rows");
        check(r.adapter_grad() == HWR_ERR_INVALID_ARG, "adapter_grad of " + std::to_string(n) + " rows");
        check(g_log.empty(), "nothing launched");
        check(std::strstr(hwr_ops_last_error(r.ops), "rows") != nullptr, "the message says why");
    }
    r.n = kMaxRows;
    check(r.matmul() == HWR_OK && r.matmul_grad() == HWR_OK, "the largest batch");
    r.n = INT32_MAX;
    check(r.group() == HWR_OK, "rows by group take any number");
}

// The runtime takes no grid of 2^32 threads or more in a dimension (hip_runtime_api.h says so
// of hipModuleLaunchKernel): the largest batches that memory can hold stay below.
void largest_grids() {
    struct Batch {
        int n, k, m, rank, G;
    };
    Rig r;
    for (const Batch &b : {Batch{1 << 27, 8, 8, 128, 4}, Batch{(1 << 28) + 5, 8, 8, 16, 1}, Batch{kMaxRows, 1, 1, 1, 1},
                           Batch{kMaxRows, 1, 1, 33, 1024}, Batch{(1 << 29) + 3, 8, 72, 8, 2}, Batch{1 << 30, 8, 64, 8, 1024}})
        for (int dtype : {HWR_BF16, HWR_F32}) {
            r.n = b.n, r.k = b.k, r.m = b.m, r.rank = b.rank, r.G = b.G, r.dtype = dtype;
            g_log.clear();
            check(r.group() == HWR_OK && r.matmul() == HWR_OK && r.matmul_grad() == HWR_OK && r.adapter() == HWR_OK &&
                      r.adapter_grad() == HWR_OK && r.adapter_grad(true, false, false) == HWR_OK, "queued");
            for (const Launch &l : g_log)
                check(static_cast<uint64_t>(l.grid.x) * l.block.x < uint64_t(1) << 32 && l.grid.y <= 65535 && l.grid.z == 1,
                      std::to_string(b.n) + " rows: " + std::to_string(l.grid.x) + " x " + std::to_string(l.block.x) + " of " + l.kernel);
        }
}

// A call has all of its work space before it queues anything: where it cannot, nothing is
// queued, and reserving what the refusal asks for is enough.
void work_space() {
    struct Batch {
        int n, k, m, rank, G;
    };
    struct Call {
        const char *name;
        hwr_status (*make)(Rig &);
    };
    const Call calls[] = {{"group", [](Rig &r) { return r.group(); }},
                          {"matmul", [](Rig &r) { return r.matmul(); }},
                          {"matmul_grad", [](Rig &r) { return r.matmul_grad(); }},
                          {"matmul_grad dw", [](Rig &r) { return r.matmul_grad(false, true); }},
                          {"adapter", [](Rig &r) { return r.adapter(); }},
                          {"adapter_grad", [](Rig &r) { return r.adapter_grad(); }},
                          {"adapter_grad dx", [](Rig &r) { return r.adapter_grad(true, false, false); }},
                          {"adapter_grad db", [](Rig &r) { return r.adapter_grad(false, false, true); }}};
    int needed = 0;
    for (const Batch &b : {Batch{16000, 1001, 1003, 16, 3}, Batch{400, 4104, 4096, 16, 2}, Batch{300, 1601, 523, 100, 1},
                           Batch{40, 4096, 4096, 16, 32}, Batch{9000, 1024, 2048, 32, 4}, Batch{100000, 40, 24, 4, 1000}})
        for (int dtype : {HWR_BF16, HWR_F32})
            for (const Call &c : calls) {
                const std::string what = std::string(c.name) + " of " + std::to_string(b.n) + (dtype == HWR_BF16 ? " bf16" : " fp32");
                Rig r;
                r.n = b.n, r.k = b.k, r.m = b.m, r.rank = b.rank, r.G = b.G, r.dtype = dtype;
                g_log.clear();
                g_capturing = true;
                const hwr_status first = c.make(r);
                if (first == HWR_OK) {
                    g_capturing = false;
                    continue;                                  // takes none
                }
                ++needed;
                check(first == HWR_ERR_STATE && g_log.empty(), what + ": " + std::to_string(g_log.size()) + " launches recorded, then refused");
                const char *ask = std::strstr(hwr_ops_last_error(r.ops), "hwr_ops_reserve ");
                const unsigned long long bytes = ask ? std::strtoull(ask + 16, nullptr, 10) : 0;
                g_capturing = false;
                check(bytes > 0 && hwr_ops_reserve(r.ops, bytes) == HWR_OK, what + ": reserve");
                g_capturing = true;
                check(c.make(r) == HWR_OK, what + ": what was asked for is enough");
                g_capturing = false;
                // a context of its own: one allocation; and none to be had
                Rig s;
                s.n = b.n, s.k = b.k, s.m = b.m, s.rank = b.rank, s.G = b.G, s.dtype = dtype;
                g_log.clear();
                g_fail = 1;
                check(c.make(s) == HWR_ERR_OOM && g_log.empty(), what + ": no memory, nothing queued");
                g_fail = SIZE_MAX;
                g_mallocs = 0;
                check(c.make(s) == HWR_OK && g_mallocs == 1, what + ": " + std::to_string(g_mallocs) + " allocations");
                g_mallocs = 0;
                check(c.make(s) == HWR_OK && g_mallocs == 0, what + ": once");
            }
    check(needed > 50, std::to_string(needed) + " calls took work space");
}

// Whatever device is current when a call is made, the call works on its context's and
// leaves the current one as it was, also where it is refused or fails.
void current_device() {
    for (int device : {0, 1})
        for (int current : {0, 1}) {
            const std::string what = "context on " + std::to_string(device) + ", current " + std::to_string(current);
            g_context_device = device, g_device = current, g_wrong_device = 0;
            {
                Rig r(device);
                check(g_device == current, what + ": init");
                r.n = 300, r.k = 264, r.m = 392, r.rank = 16, r.G = 3;
                check(r.group() == HWR_OK && r.matmul() == HWR_OK && r.matmul_grad() == HWR_OK && r.adapter() == HWR_OK &&
                          r.adapter_grad() == HWR_OK, what + ": queued");
                check(g_device == current, what + ": calls");
                check(hwr_ops_reserve(r.ops, 1 << 24) == HWR_OK && g_device == current, what + ": reserve");
                g_fail = 1;
                r.n = 200000;
                check(r.adapter() == HWR_ERR_OOM && g_device == current, what + ": no memory");
                g_fail = SIZE_MAX;
                r.k = 0;
                check(r.matmul() == HWR_ERR_INVALID_ARG && g_device == current, what + ": refused");
            }
            check(g_device == current, what + ": free");
            check(g_wrong_device == 0, what + ": " + std::to_string(g_wrong_device) + " on the wrong device");
        }
    hwr_ops *none = nullptr;
    g_device = 1, g_fail = 1;
    check(hwr_ops_init(0, nullptr, &none) == HWR_ERR_OOM && g_device == 1, "init without memory");
    g_device = 0, g_fail = SIZE_MAX;
}

// An error that was reported once is not reported again by the next launch.
void errors_are_reported_once() {
    Rig r;
    r.n = 300, r.k = 264, r.m = 392, r.rank = 16, r.G = 3;
    hwr_ops *none = nullptr;
    g_fail = 1;
    check(hwr_ops_init(0, nullptr, &none) == HWR_ERR_OOM && !none, "init without memory");
    g_fail = SIZE_MAX;
    check(r.matmul() == HWR_OK, "a launch after it");
    g_fail = 1;
    r.n = 200000;
    check(r.adapter() == HWR_ERR_OOM, "no memory");
    g_fail = SIZE_MAX;
    r.n = 300;
    check(r.matmul() == HWR_OK, "a launch after it");
    // the rounded size is not to be had, the size itself is
    Rig s;
    s.n = 200000, s.k = s.m = 40;
    g_fail = size_t(1) << 25;      // 200,000 rows of 128 bytes: 24.4 MB
    check(s.adapter() == HWR_OK, "no room to round up");
    g_fail = SIZE_MAX;
}

// Every pointer has to be aligned to its elements.
void alignment() {
    Rig r;
    r.n = 300, r.k = 264, r.m = 392, r.rank = 16, r.G = 3;
    g_log.clear();
    for (int which = 0; which < 2; ++which)
        for (int by = 1; by < 4; ++by) {
            hwr_groups g = r.groups();
            const int32_t *&p = which ? g.order : g.offsets;
            p = reinterpret_cast<const int32_t *>(reinterpret_cast<uintptr_t>(p) + by);
            const hwr_matmul_args m{HWR_BF16, 264, 392, at<char>(3), 0, at<char>(4), at<char>(5), 0};
            const hwr_matmul_grad_args mg{HWR_BF16, 264, 392, at<char>(5), 0, at<char>(3), 0, at<char>(4), at<char>(6), 0, at<char>(7)};
            const hwr_adapter_args a{HWR_BF16, 264, 392, 16, at<char>(3), 0, at<char>(4), at<char>(8), at<char>(9), nullptr, at<char>(5), 0};
            const hwr_adapter_grad_args ag{HWR_BF16, 264, 392, 16, at<char>(5), 0, at<char>(3), 0, at<char>(4), at<char>(8), at<char>(9),
                                           nullptr, at<char>(6), 0, at<char>(10), at<char>(11)};
            const std::string what = std::string(which ? "order" : "offsets") + " off by " + std::to_string(by);
            check(hwr_grouped_matmul(r.ops, &g, &m) == HWR_ERR_INVALID_ARG, what + ": matmul");
            check(hwr_grouped_matmul_grad(r.ops, &g, &mg) == HWR_ERR_INVALID_ARG, what + ": matmul_grad");
            check(hwr_adapter_matmul(r.ops, &g, &a) == HWR_ERR_INVALID_ARG, what + ": adapter");
            check(hwr_adapter_matmul_grad(r.ops, &g, &ag) == HWR_ERR_INVALID_ARG, what + ": adapter_grad");
            check(std::strstr(hwr_ops_last_error(r.ops), "aligned") != nullptr, what + ": the message says why");
        }
    check(g_log.empty(), "nothing launched");
}

// The input gradient of few rows of many groups: n rows make n tiles at most, however many
// groups there are, so small tiles and parts of the contraction occupy the device.
void few_rows_of_many_groups() {
    struct Batch {
        int n, G, k;
    };
    for (const Batch &b : {Batch{1, 32, 4096}, Batch{4, 1024, 2048}, Batch{7, 9, 2048}}) {
        Rig r;
        r.n = b.n, r.G = b.G, r.k = r.m = b.k;
        g_log.clear();
        check(r.matmul_grad(true, false) == HWR_OK && g_log.size() == 2, "dx: parts and their sum");
        const uint64_t tiles = uint64_t(b.n) * ((b.k + 63) / 64);
        check(g_log[0].kernel.find("Li64ELi64E") != std::string::npos, "tiles of 64: " + g_log[0].kernel);
        check(g_log[0].grid.x >= 256 || g_log[0].grid.x >= 4 * tiles, std::to_string(g_log[0].grid.x) + " workgroups");
    }
}

struct Scenario {
    const char *name;
    void (*run)();
};
const Scenario kScenarios[] = {{"row_limit", row_limit}, {"largest_grids", largest_grids}, {"work_space", work_space}, {"current_device", current_device},
                               {"errors_are_reported_once", errors_are_reported_once}, {"alignment", alignment},
                               {"few_rows_of_many_groups", few_rows_of_many_groups}};

}  // namespace

int main(int argc, char **argv) {
    if (argc != 2) return 2;
    for (const Scenario &s : kScenarios)
        if (std::strcmp(argv[1], s.name) == 0) {
            s.run();
            std::printf(g_bad ? "%d failed\n" : "ok\n", g_bad);
            return g_bad ? 1 : 0;
        }
    return 2;
}
