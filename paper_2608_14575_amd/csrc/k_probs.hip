// Log probabilities from rows of logits: of a given token, with the entropy of the
// distribution and its most likely tokens, and the gradient of the logits.
//
// With z = scale x, M = max z, S = sum exp(z - M) and T = sum exp(z - M) (z - M):
//   lse = M + ln S,  log p[t] = z[t] - M - ln S,  H = ln S - T / S.
// One pass: a thread keeps M, S and T of the elements that it has seen and rescales S and T
// when M grows.  Exponents are taken of scale (x - M), which cannot overflow, so that masks of the
// type's lowest value are as good as infinities.  A row of nothing but masks (below kMasked) is
// empty: lse -inf.  (Its lse could not tell ln S from 0, and a gradient from it would be m times too large.)
//
// Bound by memory where rows are many: 8,192 x 32,000 bf16 95 us (5.5 TB/s), the gradient, which reads and writes them,
// 184 us (5.7 TB/s); 1,003 x 10,007 fp32 17 us.  About 11 instructions a logit, 4 of them the exponential (a quarter of the others' rate), take
// 70 us of the first.  Few rows wait for the steps after each other: 1 x 32,000 with five tokens 7 us, of which the logits
// 2 to 4 us, sums over 16 waves 1, the tokens 2; 48 x 128,000 with twenty 13.8 us.
#include <algorithm>

#include "ops_device.hpp"

namespace hwr {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.693147180559945309417f;
// the lowest finite values of bf16 and fp32 are below (-3.30e38)
constexpr float kMasked = -0x1.Fp127f;
// exp2 of less is 0 in fp32; products of it with a difference of logits stay finite
constexpr float kFar = -200.0f;

template <class E>
constexpr int kEpc = Elem<E>::kEpc;

template <class E>
__device__ inline void unpack(u32x4 v, float (&f)[kEpc<E>]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(E) == 2) {
            f[2 * i] = __uint_as_float(v[i] << 16);
            f[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
        } else {
            f[i] = __uint_as_float(v[i]);
        }
    }
}

// Elements [0, n) of a row from p on: single ones up to an address of whole chunks, chunks,
// and single ones after them.
template <class E>
struct Span {
    const E *p;
    int n, head, chunks;
    __device__ Span(const E *at, int len) : p(at), n(len) {
        head = min(len, static_cast<int>((16 - (reinterpret_cast<uintptr_t>(at) & 15)) & 15) / static_cast<int>(sizeof(E)));
        chunks = (len - head) / kEpc<E>;
    }
    // the i-th single element, or -1 (there are fewer than 2 kEpc)
    __device__ int single(int i) const {
        const int e = i < head ? i : i + chunks * kEpc<E>;
        return e < n && i < 2 * kEpc<E> ? e : -1;
    }
    __device__ int first(int chunk) const { return head + chunk * kEpc<E>; }
    __device__ u32x4 load(int chunk) const { return *reinterpret_cast<const u32x4 *>(p + first(chunk)); }
};

// M, S and T of some elements; M at least kMasked, so that S = 0 tells that there is no
// element, or that all are masks.
struct Sums {
    float m = kMasked, s = 0.0f, t = 0.0f;
    // elements of which m is at least the maximum, after rescale
    __device__ void add(float x, float c2) {
        const float d = (x - m) * c2, e = __builtin_amdgcn_exp2f(d);
        s += e;
        t = fmaf(e, fmaxf(d, kFar), t);
    }
    // sums relative to a maximum that is no smaller
    __device__ void rescale(float to, float c2) {
        const float d = fmaxf((m - to) * c2, kFar), f = __builtin_amdgcn_exp2f(d);
        t = f * fmaf(s, d, t);
        s *= f;
        m = to;
    }
    template <int LANES = 64>
    __device__ void join_lanes(float c2);
};

// (of all lanes of a wave, or of LANES neighbours, in every lane: the largest maximum first, then one rescale and sums)
template <int LANES>
__device__ inline void Sums::join_lanes(float c2) {
    float to = m;
#pragma unroll
    for (int d = 1; d < LANES; d <<= 1) to = fmaxf(to, __shfl_xor(to, d));
    rescale(to, c2);
#pragma unroll
    for (int d = 1; d < LANES; d <<= 1) s += __shfl_xor(s, d), t += __shfl_xor(t, d);
}

// Order of the most likely tokens: larger logits first, of equal ones the lower token.  Both
// zeros are equal, and all masks.  (A NaN has a place in the order too, so that there are always enough.)
__device__ inline uint32_t order_key(float x) {
    if (x != x) return 0xFFFFFFFFu;
    const uint32_t b = __float_as_uint(x < kMasked ? -INFINITY : x + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ inline float key_value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }
__device__ inline uint64_t rank_key(uint32_t key, int token) { return static_cast<uint64_t>(key) << 32 | ~static_cast<uint32_t>(token); }

// Candidates of a team, and what its threads exchange.
constexpr int kCandidates = 512;
constexpr int kShares = 64;       // maxima that the candidates' bound is found from
struct TeamSpace {
    float m[16], s[16], t[16];
    float most[kShares];
    uint64_t best[16];
    uint64_t candidate[kCandidates];
    int count;
};

template <int T>
__device__ inline void team_sync() {
    if constexpr (T == 64) wave_lds();
    else __syncthreads();
}

// How many of keys[0, count) are larger.
__device__ inline int larger(const uint64_t *keys, int count, uint64_t than) {
    int n = 0, j = 0;
    for (; j + 8 <= count; j += 8)
#pragma unroll
        for (int u = 0; u < 8; ++u) n += keys[j + u] > than;
    for (; j < count; ++j) n += keys[j] > than;
    return n;
}

// Chunks of a row that a thread loads at a time.
constexpr int kLoad = 4;

// Rows up to kShortElements, which 16 threads load at a time, have those, up to kWaveElements a wave; longer ones
// 256 threads, or 1024 where workgroups are few and long.  us, 16 threads / a wave: bf16 16,384 x 128 5.7 / 12.7, 16,384 x 512 5.8 / 12.8,
// 1,000 x 300 5.7 / 5.1 (the call's host time); the gradient 5.6 / 7.0, 7.9 / 8.5, 5.5 / 5.1.
// A wave / 256 threads, with 20 tokens: bf16 16,384 x 1,000 29.5 / 67.6, 4,000 x 2,000 11.2 / 19.9.  Many rows fill the card with a wave
// each, without joins between waves: kManyRows of up to kManyElements have one too (with tokens, whose search is the longer part of a
// wave's time, kManyTops): 16,384 x 4,000 25.5 / 47.9 and 45.0 / 70.4 with 20 tokens, 2,000 x 4,000 5.7 / 8.8 and 12.2 / 13.3; but 300 x 6,000
// 5.4 / 5.1 and 13.3 / 8.4, 2,000 x 6,000 with tokens 17.1 / 14.2; fp32 8,192 x 8,000 40.3 / 39.7 and 76.0 / 64.8.
// 1024 threads / 256, with 20 tokens: bf16 2 x 32,000 9.4 / 12.5, 100 x 32,000 10.0 / 14.1, but 512 x 16,384 16.5 / 11.8, 1,000 x 9,000
// 28.7 / 11.8.
template <class E>
constexpr int kShortElements = 16 * kLoad * kEpc<E>;
constexpr int kWaveElements = 2048, kManyElements = 6144, kManyRows = 1024, kManyTops = 4096, kFewTeams = 256, kTeamElements = 8192;
// out(rank, key, token) of the `top` first of the row, ranks in any order; T threads, `threads` of which have chunks, whose largest
// elements are `most`, and whose chunks, where the row has kLoad a thread at most, are `in` (KEPT; else they
// are loaded again: to keep them takes registers that many workgroups want).
//
// The threads' maxima are joined to kShares.  The top-th largest of those bounds the top-th largest element
// from below, and is reached by at least `top` elements: those at or above it are the candidates (a
// few more than `top` unless values are equal: 24 for the 20th of 64, 44 for the 32nd), and only threads whose maximum reaches
// it look for them.  Each candidate's rank is the number of candidates before it.  Where there are more
// than kCandidates (long runs of equal logits), they are found one by one instead.
template <class E, int T, bool KEPT, class Out>
__device__ inline void select_top(const Span<E> &row, const u32x4 (&in)[kLoad], int threads, int offset, int top, float most,
                                  TeamSpace &ts, int tid, Out out) {
    constexpr int kShare = T / kShares;    // threads that share a maximum
    float shared = most;
#pragma unroll
    for (int d = 1; d < kShare; d <<= 1) shared = fmaxf(shared, __shfl_xor(shared, d));
    if (tid % kShare == 0) ts.most[tid / kShare] = shared;
    if (tid == 0) ts.count = 0;
    team_sync<T>();
    // (each wave for itself, bit by bit from the top: the largest key that `top` shares reach.  The low half of a bf16
    // value's key tells nothing: without it the bound is at most the value.)
    const uint32_t key = order_key(ts.most[tid & 63]);
    uint32_t floor = 0;
#pragma unroll
    for (int bit = 31; bit >= (sizeof(E) == 2 ? 16 : 0); --bit) {
        const uint32_t at = floor | 1u << bit;
        if (__popcll(__ballot(key >= at)) >= top) floor = at;
    }
    // (kMasked: threads without elements, or with masks alone: all elements are candidates)
    if (floor <= order_key(kMasked)) floor = 0;
    const float bound = floor ? key_value(floor) : -INFINITY;
    // chunks of the row: the thread's
    auto chunks = [&](bool kept, auto visit) {
        if (KEPT && kept && row.chunks <= kLoad * T) {
#pragma unroll
            for (int u = 0; u < kLoad; ++u)
                if (tid + u * T < row.chunks) visit(in[u], tid + u * T);
        } else {
#pragma unroll 1
            for (int c = tid < threads ? tid : row.chunks; c < row.chunks; c += threads) visit(row.load(c), c);
        }
    };
    auto elements = [&](u32x4 v, int c, auto visit) {
        float f[kEpc<E>];
        unpack<E>(v, f);
#pragma unroll
        for (int i = 0; i < kEpc<E>; ++i) visit(f[i], offset + row.first(c) + i);
    };
    if (floor == 0 || most >= bound) {
        auto add = [&](float x, int token) {
            if (floor && !(x >= bound)) return;
            const int at = atomicAdd(&ts.count, 1);
            if (at < kCandidates) ts.candidate[at] = rank_key(order_key(x), token);
        };
        const int e = row.single(tid);
        if (e >= 0) add(static_cast<float>(row.p[e]), offset + e);
        chunks(true, [&](u32x4 v, int c) {
            // (a wave goes through the elements of a chunk where one of its lanes has a candidate in it)
            float f[kEpc<E>], largest = -INFINITY;
            unpack<E>(v, f);
#pragma unroll
            for (int i = 0; i < kEpc<E>; ++i) largest = fmaxf(largest, f[i]);
            if (floor == 0 || largest >= bound) elements(v, c, add);
        });
    }
    team_sync<T>();
    const int count = ts.count;
    if (count <= kCandidates) {
        for (int i = tid; i < count; i += T) {
            const uint64_t mine = ts.candidate[i];
            const int before = larger(ts.candidate, count, mine);
            if (before < top) out(before, static_cast<uint32_t>(mine >> 32), static_cast<int>(~static_cast<uint32_t>(mine)));
        }
        return;
    }
    uint64_t last = ~uint64_t{0};
    for (int r = 0; r < top; ++r) {
        uint64_t best = 0;
        auto next = [&](float x, int token) {
            const uint64_t k = rank_key(order_key(x), token);
            if (k < last && k > best) best = k;
        };
        const int e = row.single(tid);
        if (e >= 0) next(static_cast<float>(row.p[e]), offset + e);
        chunks(false, [&](u32x4 v, int c) { elements(v, c, next); });
#pragma unroll
        for (int d = 32; d; d >>= 1) best = max(best, static_cast<uint64_t>(__shfl_xor(static_cast<unsigned long long>(best), d)));
        if constexpr (T > 64) {
            if ((tid & 63) == 0) ts.best[tid >> 6] = best;
            __syncthreads();
            for (int w = 0; w < T / 64; ++w) best = max(best, ts.best[w]);
            __syncthreads();
        }
        if (tid == 0) out(r, static_cast<uint32_t>(best >> 32), static_cast<int>(~static_cast<uint32_t>(best)));
        last = best;
    }
}

// Log probability of a logit.
__device__ inline float log_prob(const ProbsArgs &a, const Sums &v, float log_s, float x) {
    return v.s == 0.0f || x < kMasked ? v.s == v.s ? -INFINITY : NAN : (x - v.m) * a.scale - log_s;
}

// The results of a row but the most likely tokens, from its sums.
template <class E>
__device__ inline void store_sums(const ProbsArgs &a, int64_t r, const Sums &v, float log_s) {
    const bool empty = v.s == 0.0f;
    if (a.lse) a.lse[r] = empty ? -INFINITY : fmaf(v.m, a.scale, log_s);
    if (a.entropy) a.entropy[r] = empty ? 0.0f : fmaxf(log_s - kLn2 * (v.t / v.s), v.s == v.s ? 0.0f : NAN);
    if (a.logp) {
        const int t = a.token[r];
        float lp = 0.0f;
        if (static_cast<unsigned>(t) < static_cast<unsigned>(a.m)) {
            const float x = static_cast<float>(static_cast<const E *>(a.x)[r * a.ldx + t]);
            lp = log_prob(a, v, log_s, x);
        }
        a.logp[r] = lp;
    }
}

// Partial results of a row: [n][parts] sums, then [n][parts][top] keys.  They are written and read past the caches that
// compute units do not share.
__device__ inline float *part_sums(const ProbsArgs &a, int64_t r, int part) { return static_cast<float *>(a.partial) + (r * a.parts + part) * 4; }
__device__ inline uint64_t *part_top(const ProbsArgs &a, int64_t r, int part) {
    return reinterpret_cast<uint64_t *>(part_sums(a, a.n, 0)) + (r * a.parts + part) * a.top;
}
template <class V>
__device__ inline void put_shared(V *at, V v) { __hip_atomic_store(at, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
template <class V>
__device__ inline V get_shared(V *at) { return __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

constexpr int kMaxParts = 16;
constexpr int kPartElements = 16384;
static_assert(kPartElements >= kMaxTop && kMaxParts * kMaxTop <= kCandidates && kMaxParts <= 64);

// Whether this workgroup is the last of the row's parts; what the others have put is then there to be got.  No one waits for
// another: whoever comes last goes on, and the count is zero again.  What is shared goes through put_shared and get_shared
// alone, past the L2s (an XCD's each), so that it is enough that a part's stores are done (vmcnt, every wave before the barrier)
// before it is counted.  (Fences of the whole device, which write back an L2 in every wave: 48 x 128,000 with
// twenty tokens 58 us; a second launch instead 14.6.)
__device__ inline bool last_part(const ProbsArgs &a, int64_t r, TeamSpace &ts, int tid) {
    wait_vm<0>();
    __syncthreads();
    // (counts up to the last part, and from there to zero again)
    if (tid == 0) ts.count = static_cast<int>(atomicInc(a.arrived + r, static_cast<unsigned>(a.parts - 1)));
    __syncthreads();
    return ts.count == a.parts - 1;
}

// A row's results from those of its parts.
template <class E, int T, bool TOP>
__device__ inline void join_parts(const ProbsArgs &a, int64_t r, TeamSpace &ts, int tid, float c2) {
    Sums v;
    const int lane = tid & 63;
    if (lane < a.parts) {
        float *o = part_sums(a, r, lane);
        v.m = get_shared(o), v.s = get_shared(o + 1), v.t = get_shared(o + 2);
    }
    const int count = a.parts * a.top;
    if constexpr (TOP) {
        uint64_t *top = part_top(a, r, 0);
        for (int i = tid; i < count; i += T) ts.candidate[i] = get_shared(top + i);
    }
    v.join_lanes(c2);
    const float log_s = logf(v.s);
    if (tid == 0) store_sums<E>(a, r, v, log_s);
    if constexpr (TOP) {
        __syncthreads();
        for (int i = tid; i < count; i += T) {
            const uint64_t mine = ts.candidate[i];
            const int before = larger(ts.candidate, count, mine);
            if (before >= a.top) continue;
            if (a.top_logp) a.top_logp[r * a.top + before] = log_prob(a, v, log_s, key_value(static_cast<uint32_t>(mine >> 32)));
            if (a.top_token) a.top_token[r * a.top + before] = static_cast<int>(~static_cast<uint32_t>(mine));
        }
    }
}

// T threads to a row, or to a part of it; 256 / T rows to a workgroup where T is less (less than a wave without tokens alone).
template <class E, int T, bool TOP>
__global__ void __launch_bounds__(T < 256 ? 256 : T, T == 64 ? 8 : 1) k_probs(ProbsArgs a) {
    constexpr int NT = T < 256 ? 256 : T, kRows = NT / T, U = kLoad;
    static_assert(T == 64 || kRows == 1 || !TOP);
    __shared__ TeamSpace space[T >= 64 ? kRows : 1];
    constexpr bool kKept = T == 1024;
    const int tid = threadIdx.x % T, lane = tid & 63;
    TeamSpace &ts = space[T >= 64 ? threadIdx.x / T : 0];
    const int64_t item = static_cast<int64_t>(block_id<NT>()) * kRows + threadIdx.x / T;
    const int64_t r = kRows > 1 ? item : item / a.parts;
    const int part = kRows > 1 ? 0 : static_cast<int>(item % a.parts);
    if (r >= a.n) return;
    const int first = static_cast<int>(static_cast<int64_t>(a.m) * part / a.parts);
    const int last = static_cast<int>(static_cast<int64_t>(a.m) * (part + 1) / a.parts);
    const Span<E> row(static_cast<const E *>(a.x) + r * a.ldx + first, last - first);
    const float c2 = a.scale * kLog2e;

    Sums v;
    if (const int e = row.single(tid); e >= 0) {
        const float x = static_cast<float>(row.p[e]);
        v.m = fmaxf(v.m, x);
        v.add(x, c2);
    }
    u32x4 in[U];
    // (a wave on a short row: 16 threads as without tokens, so that its sums have the same bits)
    const int threads = T == 64 && a.m <= kShortElements<E> ? 16 : T;
    for (int c = tid < threads ? tid : row.chunks; c < row.chunks; c += U * threads) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t none = sizeof(E) == 2 ? 0xFF80FF80u : 0xFF800000u;      // -inf
            in[u] = u32x4{none, none, none, none};
            if (c + u * threads < row.chunks) in[u] = row.load(c + u * threads);
        }
        float f[U][kEpc<E>], most = v.m;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            unpack<E>(in[u], f[u]);
#pragma unroll
            for (int i = 0; i < kEpc<E>; ++i) most = fmaxf(most, f[u][i]);
        }
        v.rescale(most, c2);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < kEpc<E>; ++i) v.add(f[u][i], c2);
    }

    const float mine = v.m;
    v.join_lanes<(T < 64 ? T : 64)>(c2);
    if constexpr (T > 64) {
        if (lane == 0) ts.m[tid >> 6] = v.m, ts.s[tid >> 6] = v.s, ts.t[tid >> 6] = v.t;
        __syncthreads();
        v = Sums{};
        if (lane < T / 64) v.m = ts.m[lane], v.s = ts.s[lane], v.t = ts.t[lane];
        v.join_lanes(c2);
    }
    if (T == 1024 && a.parts > 1) {
        if (tid == 0) {
            float *o = part_sums(a, r, part);
            put_shared(o, v.m), put_shared(o + 1, v.s), put_shared(o + 2, v.t);
        }
        if constexpr (TOP) {
            uint64_t *out = part_top(a, r, part);    // (a part has more elements than kMaxTop)
            select_top<E, T, kKept>(row, in, threads, first, a.top, mine, ts, tid,
                                    [&](int rank, uint32_t key, int token) { put_shared(out + rank, rank_key(key, token)); });
        }
        if (last_part(a, r, ts, tid)) join_parts<E, T, TOP>(a, r, ts, tid, c2);
        return;
    }
    const float log_s = logf(v.s);
    if (tid == 0) store_sums<E>(a, r, v, log_s);
    if constexpr (TOP)
        select_top<E, T, kKept>(row, in, threads, 0, a.top, mine, ts, tid, [&](int rank, uint32_t key, int token) {
            if (a.top_logp) a.top_logp[r * a.top + rank] = log_prob(a, v, log_s, key_value(key));
            if (a.top_token) a.top_token[r * a.top + rank] = token;
        });
}

// dx = scale (dlogp (1[c = t] - p) - dentropy p (ln p + H)), ln p = scale x - lse.  A row without
// a token has no first term; one that has neither term, or is empty, gets zeros unread.
template <class E, int T>
__global__ void __launch_bounds__(256) k_probs_grad(ProbsGradArgs a, int slabs) {
    constexpr int kRows = 256 / T, U = 4, kSlab = T * U * kEpc<E>;
    const int tid = threadIdx.x % T;
    const int64_t item = static_cast<int64_t>(block_id<256>()) * kRows + threadIdx.x / T;
    const int64_t r = item / slabs;
    if (r >= a.n) return;
    const int slab = static_cast<int>(item - r * slabs);
    const E *x = static_cast<const E *>(a.x) + r * a.ldx;
    E *dx = static_cast<E *>(a.dx) + r * a.lddx;
    // chunks are whole in dx
    const Span<E> row(dx, a.m);
    const int t = a.token ? a.token[r] : -1;
    const bool held = static_cast<unsigned>(t) < static_cast<unsigned>(a.m);
    const float lse = a.lse[r], dl = a.dlogp && held ? a.dlogp[r] : 0.0f;
    const float dh = a.dentropy ? a.dentropy[r] : 0.0f, h = a.dentropy ? a.entropy[r] : 0.0f;
    const bool zero = lse == -INFINITY || (dl == 0.0f && dh == 0.0f);
    const float nl = -dl * a.scale, nh = -dh * a.scale;
    auto value = [&](float xv, int c) {
        const float v = fmaf(xv, a.scale, -lse), p = __builtin_amdgcn_exp2f(v * kLog2e);
        const float g = p * fmaf(nh, fmaxf(v, kFar) + h, nl);
        return c == t ? g - nl : g;
    };
    if (slab == 0) {
        const int e = row.single(tid);
        if (e >= 0) dx[e] = static_cast<E>(zero ? 0.0f : value(static_cast<float>(x[e]), e));
    }
    const int c0 = slab * U * T + tid;
    u32x4 in[U];
    if (!zero) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (c0 + u * T < row.chunks) {
                const typename Elem<E>::Vec l = *reinterpret_cast<const typename Elem<E>::Vec *>(x + row.first(c0 + u * T));
                in[u] = u32x4{l[0], l[1], l[2], l[3]};
            }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (c0 + u * T >= row.chunks) continue;
        union { u32x4 v; E e[kEpc<E>]; } o;
        o.v = u32x4{0, 0, 0, 0};
        const int c = row.first(c0 + u * T);
        if (!zero) {
            float f[kEpc<E>];
            unpack<E>(in[u], f);
#pragma unroll
            for (int i = 0; i < kEpc<E>; ++i) o.e[i] = static_cast<E>(value(f[i], c + i));
        }
        *reinterpret_cast<u32x4 *>(dx + c) = o.v;
    }
}

template <class E, int T>
hipError_t go(const ProbsArgs &a, hipStream_t s) {
    constexpr int NT = T < 256 ? 256 : T, kRows = NT / T;
    const int64_t blocks = kRows > 1 ? (a.n + kRows - 1) / kRows : a.n * a.parts;
    if (blocks > INT32_MAX - grid_row(NT)) return hipErrorInvalidValue;
    if constexpr (T >= 64)
        if (a.top) return launch_kernel(k_probs<E, T, true>, wide_grid(blocks, NT), dim3(NT), 0, s, a);
    return launch_kernel(k_probs<E, T, false>, wide_grid(blocks, NT), dim3(NT), 0, s, a);
}
template <class E>
hipError_t pick(const ProbsArgs &a, hipStream_t s) {
    if (!a.top && a.m <= kShortElements<E>) return go<E, 16>(a, s);
    if (a.m <= (a.n >= (a.top ? kManyTops : kManyRows) ? kManyElements : kWaveElements)) return go<E, 64>(a, s);
    if (a.parts > 1) return go<E, 1024>(a, s);
    if (a.n * a.parts <= kFewTeams && a.m / a.parts >= kTeamElements) return go<E, 1024>(a, s);
    return go<E, 256>(a, s);
}

template <class E, int T>
hipError_t go_grad(const ProbsGradArgs &a, hipStream_t s) {
    constexpr int kRows = 256 / T, kSlab = T * 4 * kEpc<E>;
    const int slabs = (a.m + kSlab - 1) / kSlab;
    const int64_t blocks = (a.n * slabs + kRows - 1) / kRows;
    if (blocks > INT32_MAX - grid_row(256)) return hipErrorInvalidValue;
    return launch_kernel(k_probs_grad<E, T>, wide_grid(blocks, 256), dim3(256), 0, s, a, slabs);
}
template <class E>
hipError_t pick_grad(const ProbsGradArgs &a, hipStream_t s) {
    if (a.m <= kShortElements<E>) return go_grad<E, 16>(a, s);
    if (a.m <= kWaveElements) return go_grad<E, 64>(a, s);
    return go_grad<E, 256>(a, s);
}

}  // namespace

// Rows are shared where there are fewer than compute units, in parts of at least kPartElements
// (bf16 with 20 tokens, us, at 8,192 / 16,384 / 65,536: 2 x 32,000 11.6 / 9.4 / -, 100 x 32,000 11.9 / 10.0 / -, 1 x 128,000
// 15.5 / 13.3 / 19.6, 48 x 128,000 - / 13.3 / 21.5).
int probs_parts(bool bf16, int64_t n, int m, int cus) {
    if (m <= kWaveElements) return 1;
    const int64_t want = cus / n;
    return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({want, m / kPartElements, kMaxParts})));
}
uint64_t probs_bytes(const ProbsArgs &a) {
    return a.parts > 1 ? static_cast<uint64_t>(a.n) * a.parts * (4 * sizeof(float) + a.top * sizeof(uint64_t)) : 0;
}
hipError_t launch_probs(bool bf16, const ProbsArgs &a, hipStream_t s) { return bf16 ? pick<__bf16>(a, s) : pick<float>(a, s); }
hipError_t launch_probs_grad(bool bf16, const ProbsGradArgs &a, hipStream_t s) {
    return bf16 ? pick_grad<__bf16>(a, s) : pick_grad<float>(a, s);
}

}  // namespace hwr
