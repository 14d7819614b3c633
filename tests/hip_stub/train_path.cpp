// The host side of a training step's operators on the stand-in runtime of ops_path.cpp
// (tests/test_train_host_cpu.py builds and runs it).
//
//   train_path <scenario>        prints "ok", or the failed checks (exit 1)
#define main ops_path_main
#include "ops_path.cpp"
#undef main

#include <functional>

size_t g_copied = 0;
extern "C" hipError_t hipMemcpy(void *, const void *, size_t n, hipMemcpyKind) {
    g_wrong_device += g_device != g_context_device;
    g_copied += n;
    return hipSuccess;
}

namespace {

struct Train : Rig {
    using Rig::Rig;
    hwr_status linear(int act = HWR_ACT_GELU) {
        const hwr_groups g = groups();
        const hwr_linear_args a{dtype, k, m, act, at<char>(3), 0, at<char>(4), at<char>(8), at<char>(9), 0, at<char>(5), 0, at<char>(6), 0};
        return hwr_grouped_linear(ops, &g, &a);
    }
    hwr_status linear_grad(bool dx = true, bool dw = true, bool db = true, int act = HWR_ACT_SILU) {
        const hwr_groups g = groups();
        const hwr_linear_grad_args a{dtype, k, m, act, at<char>(5), 0, at<char>(6), 0, at<char>(3), 0, at<char>(4), dx ? at<char>(7) : nullptr, 0,
                                     dw ? at<char>(8) : nullptr, db ? at<char>(9) : nullptr};
        return hwr_grouped_linear_grad(ops, &g, &a);
    }
    hwr_log_probs_args probs_args(int top) const {
        return {dtype, n, m, top, 1.0f, at<char>(3), 0, at<int32_t>(0), at<float>(4), at<float>(5), at<float>(6),
                top ? at<float>(7) : nullptr, top ? at<int32_t>(8) : nullptr};
    }
    hwr_status probs(int top = 0) {
        const hwr_log_probs_args a = probs_args(top);
        return hwr_log_probs(ops, &a);
    }
    hwr_status probs_grad() {
        const hwr_log_probs_grad_args a{dtype, n, m, 1.0f, at<char>(3), 0, at<int32_t>(0), at<float>(4), at<float>(5), at<float>(6), at<float>(7),
                                        at<char>(9), 0};
        return hwr_log_probs_grad(ops, &a);
    }
    hwr_adamw_tensor tensor(int64_t count, int bits, bool master, int first) const {
        const bool scales = bits == 8;
        return {count, at<char>(first), at<char>(first + 1), master ? at<float>(first + 2) : nullptr, at<char>(first + 3), at<char>(first + 4),
                scales ? at<float>(first + 5) : nullptr, scales ? at<float>(first + 6) : nullptr};
    }
    hwr_status adamw(const std::vector<hwr_adamw_tensor> &t, int bits, hwr_adamw **out) {
        const hwr_adamw_config c{dtype, bits, static_cast<int32_t>(t.size()), t.data()};
        return hwr_adamw_init(ops, &c, out);
    }
    hwr_status step(hwr_adamw *w, bool counted = false) {
        hwr_adamw_args a{1e-3, 0.9, 0.999, 1e-8, 0.1, 7, 3, nullptr, nullptr};
        if (counted) a.steps = at<int64_t>(40);
        return hwr_adamw_step(ops, w, &a);
    }
};

using Call = std::pair<const char *, std::function<hwr_status(Train &)>>;
const std::vector<Call> &calls() {
    static const std::vector<Call> c = {
        {"linear", [](Train &r) { return r.linear(); }},
        {"linear bare", [](Train &r) { return r.linear(HWR_ACT_NONE); }},
        {"linear_grad", [](Train &r) { return r.linear_grad(); }},
        {"linear_grad none", [](Train &r) { return r.linear_grad(true, true, true, HWR_ACT_NONE); }},
        {"linear_grad dx", [](Train &r) { return r.linear_grad(true, false, false); }},
        {"linear_grad dw", [](Train &r) { return r.linear_grad(false, true, false); }},
        {"linear_grad dbias", [](Train &r) { return r.linear_grad(false, false, true); }},
        {"log_probs", [](Train &r) { return r.probs(); }},
        {"log_probs top", [](Train &r) { return r.probs(std::min(r.m, 20)); }},
        {"log_probs_grad", [](Train &r) { return r.probs_grad(); }}};
    return c;
}
struct Batch {
    int n, k, m, G;
};

// A call has all of its work space before it queues anything; what a refusal asks for is enough.
void train_work_space() {
    int needed = 0;
    for (const Batch &b : {Batch{16000, 1001, 1003, 3}, Batch{400, 4104, 4096, 2}, Batch{300, 1601, 523, 1}, Batch{40, 4096, 4096, 32},
                           Batch{9000, 1024, 2048, 4}, Batch{2000, 40, 24, 1000}, Batch{3, 64, 65536, 1}, Batch{5, 512, 512, 2}})
        for (int dtype : {HWR_BF16, HWR_F32})
            for (const Call &c : calls()) {
                const std::string what = std::string(c.first) + " of " + std::to_string(b.n) + (dtype == HWR_BF16 ? " bf16" : " fp32");
                auto set = [&](Train &r) { r.n = b.n, r.k = b.k, r.m = b.m, r.G = b.G, r.dtype = dtype; };
                Train r;
                set(r);
                g_log.clear();
                g_capturing = true;
                const hwr_status first = c.second(r);
                g_capturing = false;
                if (first == HWR_OK) continue;                 // takes none
                ++needed;
                check(first == HWR_ERR_STATE && g_log.empty(), what + ": " + std::to_string(g_log.size()) + " launches recorded, then refused");
                const char *ask = std::strstr(hwr_ops_last_error(r.ops), "hwr_ops_reserve ");
                const unsigned long long bytes = ask ? std::strtoull(ask + 16, nullptr, 10) : 0;
                check(bytes > 0 && hwr_ops_reserve(r.ops, bytes) == HWR_OK, what + ": reserve");
                g_capturing = true;
                check(c.second(r) == HWR_OK, what + ": what was asked for is enough");
                g_capturing = false;
                Train s;
                set(s);
                g_log.clear();
                g_fail = 1;
                check(c.second(s) == HWR_ERR_OOM && g_log.empty(), what + ": no memory, nothing queued");
                g_fail = SIZE_MAX;
                g_mallocs = 0;
                check(c.second(s) == HWR_OK && g_mallocs == 1, what + ": " + std::to_string(g_mallocs) + " allocations");
                g_mallocs = 0;
                check(c.second(s) == HWR_OK && g_mallocs == 0, what + ": once");
            }
    check(needed > 40, std::to_string(needed) + " calls took work space");
}

void train_largest_grids() {
    auto grids = [](const std::string &what) {
        check(!g_log.empty(), what + ": queued");
        for (const Launch &l : g_log)
            check(l.grid.x > 0 && static_cast<uint64_t>(l.grid.x) * l.block.x < uint64_t(1) << 32 && l.grid.y <= 65535 && l.grid.z == 1,
                  what + ": " + std::to_string(l.grid.x) + " x " + std::to_string(l.block.x) + " of " + l.kernel);
    };
    Train r;
    for (const Batch &b : {Batch{1 << 27, 8, 8, 4}, Batch{kMaxRows, 1, 1, 1}, Batch{kMaxRows, 1, 1, 1024}, Batch{(1 << 28) + 3, 8, 264, 2}})
        for (int dtype : {HWR_BF16, HWR_F32}) {
            r.n = b.n, r.k = b.k, r.m = b.m, r.G = b.G, r.dtype = dtype;
            g_log.clear();
            check(r.linear() == HWR_OK && r.linear_grad() == HWR_OK && r.probs(1) == HWR_OK && r.probs() == HWR_OK && r.probs_grad() == HWR_OK,
                  "queued: " + std::string(hwr_ops_last_error(r.ops)));
            grids(std::to_string(b.n) + " rows");
        }
    r.n = INT32_MAX, r.m = 2048;
    g_log.clear();
    check(r.probs(32) == HWR_OK && r.probs_grad() == HWR_OK, "2^31 - 1 rows of logits");
    grids("2^31 - 1 rows of logits");
    r.n = 1, r.m = 1 << 24;
    g_log.clear();
    check(r.probs(32) == HWR_OK && r.probs_grad() == HWR_OK, "the longest row");
    grids("the longest row");
    hwr_adamw *w = nullptr;
    r.dtype = HWR_BF16;
    check(r.adamw({r.tensor(int64_t{1} << 36, 8, false, 10)}, 8, &w) == HWR_OK && w, "2^36 values");
    g_log.clear();
    check(r.step(w) == HWR_OK && r.step(w, true) == HWR_OK, "2^36 values");
    grids("2^36 values");
    hwr_adamw_free(w);
}

// Whatever device is current, the context's is used and the current one stays.
void train_current_device() {
    for (int device : {0, 1})
        for (int current : {0, 1}) {
            const std::string what = "context on " + std::to_string(device) + ", current " + std::to_string(current);
            g_context_device = device, g_device = current, g_wrong_device = 0;
            {
                Train r(device);
                r.n = 300, r.k = 264, r.m = 392, r.G = 3;
                for (const Call &c : calls()) check(c.second(r) == HWR_OK && g_device == current, what + ": " + c.first);
                hwr_adamw *w = nullptr;
                check(r.adamw({r.tensor(1000, 32, true, 10)}, 32, &w) == HWR_OK && g_device == current, what + ": init");
                check(r.step(w) == HWR_OK && r.step(w, true) == HWR_OK && g_device == current, what + ": step");
                if (device == 0) {                             // a context of another device refuses it
                    g_context_device = 1;
                    Train other(1);
                    check(other.step(w) == HWR_ERR_INVALID_ARG && std::strstr(hwr_ops_last_error(other.ops), "device"), what + ": another's");
                }
                g_context_device = device;
                hwr_adamw_free(w);
                check(g_device == current, what + ": free");
            }
            check(g_wrong_device == 0, what + ": " + std::to_string(g_wrong_device) + " on the wrong device");
        }
    g_device = g_context_device = 0;
}

void train_refusals() {
    Train r;
    r.n = 4, r.k = 8, r.m = 16, r.G = 2;
    g_log.clear();
    auto refused = [&](hwr_status s, const char *why, const std::string &what) {
        check(s == HWR_ERR_INVALID_ARG && std::strstr(hwr_ops_last_error(r.ops), why), what + ": " + hwr_ops_last_error(r.ops));
    };
    auto off = [](auto *p, int by) { return reinterpret_cast<decltype(p)>(reinterpret_cast<uintptr_t>(p) + by); };
    // log probabilities
    auto probs = [&](auto change) {
        hwr_log_probs_args a = r.probs_args(3);
        change(a);
        return hwr_log_probs(r.ops, &a);
    };
    refused(probs([](auto &a) { a.dtype = 7; }), "dtype", "dtype");
    refused(probs([](auto &a) { a.n = -1; }), "n < 0", "n");
    refused(probs([](auto &a) { a.m = 0; }), "m outside", "m");
    refused(probs([](auto &a) { a.m = (1 << 24) + 1; }), "m outside", "m");
    refused(probs([](auto &a) { a.top = -1; }), "top", "top");
    refused(probs([](auto &a) { a.top = 33; }), "top", "top");
    refused(probs([](auto &a) { a.m = 2, a.top = 3; }), "top", "top");
    refused(probs([](auto &a) { a.top = 0; }), "top", "top tokens without a number");
    refused(probs([](auto &a) { a.top_logp = nullptr, a.top_token = nullptr; }), "top", "a number without top tokens");
    refused(probs([](auto &a) { a.ldx = 15; }), "stride", "ldx");
    refused(probs([](auto &a) { a.x = nullptr; }), "x is required", "x");
    refused(probs([](auto &a) { a.token = nullptr; }), "token", "token");
    for (int by = 1; by < 4; ++by) {
        refused(probs([&](auto &a) { a.token = off(a.token, by); }), "aligned", "token");
        refused(probs([&](auto &a) { a.top_token = off(a.top_token, by); }), "aligned", "top_token");
        refused(probs([&](auto &a) { a.lse = off(a.lse, by); }), "aligned", "lse");
    }
    refused(probs([&](auto &a) { a.x = off(const_cast<char *>(static_cast<const char *>(a.x)), 1); }), "aligned", "x");
    // layers
    const hwr_groups g = r.groups();
    const hwr_linear_args good{HWR_F32, 8, 16, HWR_ACT_RELU, at<char>(3), 0, at<char>(4), at<char>(8), at<char>(9), 0, at<char>(5), 0, at<char>(6), 0};
    auto linear = [&](auto change) {
        hwr_linear_args a = good;
        change(a);
        return hwr_grouped_linear(r.ops, &g, &a);
    };
    refused(linear([](auto &a) { a.act = 4; }), "activation", "act");
    refused(linear([](auto &a) { a.y = const_cast<void *>(a.residual); }), "may not", "y in place of the residual");
    refused(linear([](auto &a) { a.z = a.y; }), "may not", "z in place of y");
    refused(linear([](auto &a) { a.z = const_cast<void *>(a.x); }), "may not", "z in place of x");
    for (int by = 1; by < 4; ++by)
        refused(linear([&](auto &a) { a.bias = off(const_cast<char *>(static_cast<const char *>(a.bias)), by); }), "aligned", "bias");
    // weights' steps
    hwr_adamw *w = reinterpret_cast<hwr_adamw *>(8);
    const hwr_adamw_tensor t = r.tensor(600, 8, false, 10);
    auto init = [&](int bits, auto change) {
        std::vector<hwr_adamw_tensor> v = {t, r.tensor(100, 8, false, 20)};
        change(v);
        return r.adamw(v, bits, &w);
    };
    refused(init(16, [](auto &) {}), "bits", "bits");
    refused(init(32, [](auto &) {}), "m_scale", "scales without 8 bits");
    refused(init(8, [](auto &v) { v[0].v_scale = nullptr; }), "m_scale", "no scale");
    refused(init(8, [](auto &v) { v[1].count = -1; }), "tensor 1: count", "count");
    refused(init(8, [](auto &v) { v[1].g = nullptr; }), "tensor 1: p, g", "g");
    refused(init(8, [](auto &v) { v[1].master = at<float>(30); }), "for some tensors", "master");
    refused(init(8, [&](auto &v) { v[0].p = off(static_cast<char *>(v[0].p), 1); }), "aligned", "p");
    refused(init(8, [&](auto &v) { v[0].m_scale = off(v[0].m_scale, 2); }), "aligned", "scale");
    refused(init(8, [&](auto &v) { v[1].p = static_cast<char *>(v[0].p) + 1198; }), "overlap", "weights");
    refused(init(8, [&](auto &v) { v[1].g = static_cast<char *>(v[0].m) + 598; }), "overlap", "a gradient and a state");
    refused(init(8, [&](auto &v) { v[1].m = v[1].v; }), "overlap", "states");
    refused(init(8, [&](auto &v) { v[1].m_scale = v[0].m_scale + 2; }), "overlap", "scales");
    check(w == nullptr, "no handle after a refusal");
    check(init(8, [&](auto &v) { v[1].p = static_cast<char *>(v[0].p) + 1200, v[1].g = v[0].g, v[1].m_scale = v[0].m_scale + 3; }) == HWR_OK && w,
          "side by side, and a gradient for two");
    check(g_log.empty(), "nothing launched");
    // steps
    g_capturing = true;
    check(r.step(w) == HWR_ERR_STATE && g_log.empty(), "a numbered step is not captured");
    check(r.step(w, true) == HWR_OK && g_log.size() == 2, "a counted one is");
    g_capturing = false;
    g_log.clear();
    check(r.step(w) == HWR_OK && g_log.size() == 1, "one launch");
    refused(hwr_adamw_step(r.ops, nullptr, nullptr), "adamw is NULL", "NULL");
    refused(hwr_adamw_step(r.ops, w, nullptr), "arguments", "NULL");
    hwr_adamw_free(w);
    // memory that is not to be had is reported, and freed
    const size_t blocks = g_mem.size();
    g_fail = 1;
    check(init(8, [](auto &) {}) == HWR_ERR_OOM && !w && g_mem.size() == blocks, "no memory");
    g_fail = SIZE_MAX;
    check(init(8, [](auto &) {}) == HWR_OK, "then");
    hwr_adamw_free(w);
    check(g_mem.size() == blocks, "freed");
}

const Scenario kTrain[] = {{"work_space", train_work_space}, {"largest_grids", train_largest_grids}, {"current_device", train_current_device},
                           {"refusals", train_refusals}};

}  // namespace

int main(int argc, char **argv) {
    if (argc != 2) return 2;
    for (const Scenario &s : kTrain)
        if (std::strcmp(argv[1], s.name) == 0) {
            s.run();
            std::printf(g_bad ? "%d failed\n" : "ok\n", g_bad);
            return g_bad ? 1 : 0;
        }
    return 2;
}
