// Calls under stream capture on the stand-in runtime of ops_path.cpp (tests/test_capture_host_cpu.py
// builds and runs it).
//
//   capture_path <scenario>      prints "ok", or the failed checks (exit 1)
#define main ops_path_main
#include "ops_path.cpp"
#undef main

#include <algorithm>

int g_copies = 0;
extern "C" hipError_t hipMemcpy(void *, const void *, size_t, hipMemcpyKind) {
    ++g_copies;
    return hipSuccess;
}

namespace {

// What allocates, copies and waits is refused before it does.
void adamw_init() {
    Rig r;
    const hwr_adamw_tensor t{600, at<char>(10), at<char>(11), nullptr, at<char>(12), at<char>(13), nullptr, nullptr};
    const hwr_adamw_config c{HWR_F32, 32, 1, &t}, none{HWR_F32, 32, 0, nullptr};
    for (const hwr_adamw_config *f : {&c, &none}) {
        hwr_adamw *w = reinterpret_cast<hwr_adamw *>(8);
        g_mallocs = g_copies = 0;
        g_capturing = true;
        check(hwr_adamw_init(r.ops, f, &w) == HWR_ERR_STATE && !w, "refused");
        check(g_mallocs == 0 && g_copies == 0 && g_log.empty(), "nothing recorded");
        check(std::strstr(hwr_ops_last_error(r.ops), "captured") != nullptr, hwr_ops_last_error(r.ops));
        g_capturing = false;
        check(hwr_adamw_init(r.ops, f, &w) == HWR_OK && w, "before it, it is made");
        hwr_adamw_free(w);
    }
}

// Both gradients of a product run in the space that they need one after the other, in which they
// cannot share a launch: a graph that was captured with so much can be captured again.
void gradients_one_after_the_other() {
    auto asked = [](Rig &r, bool dx, bool dw) -> uint64_t {
        g_capturing = true;
        const hwr_status st = r.matmul_grad(dx, dw);
        g_capturing = false;
        const char *ask = std::strstr(hwr_ops_last_error(r.ops), "hwr_ops_reserve ");
        return st == HWR_ERR_STATE && ask ? std::strtoull(ask + 16, nullptr, 10) : 0;
    };
    auto launched = [](const char *kernel) {
        for (const Launch &l : g_log)
            if (l.kernel.find(kernel) != std::string::npos) return true;
        return false;
    };
    int found = 0;
    for (int n = 100; n < 3000; n += n / 8)
        for (int dtype : {HWR_BF16, HWR_F32}) {
            const std::string what = std::to_string(n) + (dtype == HWR_BF16 ? " rows, bf16" : " rows, fp32");
            auto set = [&](Rig &r) { r.n = n, r.k = r.m = 512, r.dtype = dtype; };
            Rig r, more;
            set(r), set(more);
            const uint64_t both = asked(r, true, true), least = std::max(asked(r, true, false), asked(r, false, true));
            if (!least) continue;
            check(hwr_ops_reserve(r.ops, least) == HWR_OK && hwr_ops_reserve(more.ops, both) == HWR_OK, what + ": reserve");
            g_log.clear();
            g_capturing = true;
            check(r.matmul_grad() == HWR_OK, what + ": " + std::to_string(least) + " bytes, " + hwr_ops_last_error(r.ops));
            found += !launched("k_grad");
            g_log.clear();
            check(more.matmul_grad() == HWR_OK && launched("k_grad"), what + ": one launch in what is asked for");
            g_capturing = false;
            // and where memory is short
            Rig s;
            set(s);
            g_fail = least + 1;
            g_log.clear();
            check(s.matmul_grad() == HWR_OK && launched("k_grad") == (both <= least), what + ": short of memory");
            g_fail = SIZE_MAX;
        }
    check(found > 2, std::to_string(found) + " in two launches");
}

const Scenario kCapture[] = {{"adamw_init", adamw_init}, {"gradients_one_after_the_other", gradients_one_after_the_other}};

}  // namespace

int main(int argc, char **argv) {
    if (argc != 2) return 2;
    for (const Scenario &s : kCapture)
        if (std::strcmp(argv[1], s.name) == 0) {
            s.run();
            std::printf(g_bad ? "%d failed\n" : "ok\n", g_bad);
            return g_bad ? 1 : 0;
        }
    return 2;
}
