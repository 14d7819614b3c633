// Calls under stream capture on the stand-in runtime of ops_path.cpp (tests/test_capture_host_cpu.py
// builds and runs it).
//
//   capture_path <scenario>      prints "ok", or the failed checks (exit 1)
#define main ops_path_main
#include "ops_path.cpp"
#undef main

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

const Scenario kCapture[] = {{"adamw_init", adamw_init}};

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
