// Device code shared by the operators on a routed batch: element types and
// their matrix instruction, staged tiles and their LDS layout.  (The walk
// over ragged groups: ops_groups.hpp.)
//
// All products run on 16x16 MFMA with the weights (or the right-hand factor) as
// the A operand and the rows as the B operand, so that a lane ends up with four
// neighbouring output columns of one row: D[i] of lane l is column 4 (l / 16) + i,
// row l % 16.  An operand fragment is 16 bytes a lane: lane l holds, for its
// column or row l % 16, the contraction elements of its quarter l / 16.
#pragma once

#include <type_traits>

#include "ops_internal.hpp"

namespace hwr {

typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
// 16 bytes at any element alignment
typedef uint32_t u32x4_a2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
typedef float f32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
typedef __bf16 bf16x4_a2 __attribute__((ext_vector_type(4), aligned(2)));

template <class E>
struct Elem;

template <>
struct Elem<__bf16> {
    using Frag = bf16x8;
    using Vec = u32x4_a2;
    using Out4 = bf16x4_a2;
    static constexpr int kBk = 64;    // contraction elements of a stage
    static constexpr int kEpc = 8;    // elements of a 16-byte chunk
    static __device__ f32x4 mma(Frag a, Frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};

template <>
struct Elem<float> {
    using Frag = f32x4;
    using Vec = u32x4_a4;
    using Out4 = f32x4_a4;
    static constexpr int kBk = 32;
    static constexpr int kEpc = 4;
    static __device__ f32x4 mma(Frag a, Frag b, f32x4 c) {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
        return c;
    }
};

constexpr int kStageBytes = 128;      // contraction bytes of a stage, in either tile layout

// ---------------------------------------------------------------- staged tiles
// A tile is stored in 16-byte chunks.  KC: line i is row (or column) i, 8
// chunks of contraction elements.  KS: line e is contraction element e, with
// the chunks of neighbouring columns.  Chunks are permuted within a line so
// that the fragment reads below spread over all banks: chunk c of line i is
// stored at c ^ swz(i).
template <class E, bool KS, int N>
struct Tile {
    static constexpr int kLines = KS ? Elem<E>::kBk : N;
    static constexpr int kCpl = KS ? N * (int)sizeof(E) / 16 : 8;   // chunks of a line
    static constexpr int kChunks = N * 8;
    static constexpr int kBytes = kChunks * 16;
    static __device__ int swz(int line) {
        if constexpr (!KS) return (line >> 1) & 7;
        else if constexpr (sizeof(E) == 4) return (((line >> 2) & 3) << 2) & (kCpl - 1);
        else if constexpr (kCpl >= 16) return ((line & 3) | ((line >> 3) & 1) << 2) << 1;
        else if constexpr (kCpl == 8) return (((line >> 1) & 1) | ((line >> 3) & 1) << 1) << 1;
        else if constexpr (kCpl == 4) return ((line >> 3) & 1) << 1;
        else return 0;
    }
    // Byte of the lane's share of the fragment at row (column) 0 of the tile's first
    // half.  A lane's line keeps its chunk order from one fragment to the next, so that the
    // others differ by constants, added or (within a line) xored.
    static __device__ int base(int lane) {
        const int m = lane & 15, q = lane >> 4;
        if constexpr (!KS) return m * 128 + ((q ^ swz(m)) << 4);
        else if constexpr (sizeof(E) == 4) return q * 4 * (kCpl * 16) + (((m >> 2) ^ swz(q * 4)) << 4) + (m & 3) * 4;
        else return (q * 8 + (m >> 2)) * (kCpl * 16) + ((((m & 3) >> 1) ^ swz(q * 8 + (m >> 2))) << 4) + (m & 1) * 8;
    }
    // Fragment of the 16 rows (columns) from c0 on, contraction half `sub` of the
    // stage; the tile lies at byte `at` of the LDS array.  (One offset, added once:
    // the compiler follows an array through few additions only, and reads that it
    // cannot place wait for every load in flight into LDS.)
    static __device__ typename Elem<E>::Frag frag(const char *lds, int at, int c0, int sub, int base) {
        if constexpr (!KS) {
            const int o = (base ^ (sub * 64)) + at + c0 * 128;
            return *reinterpret_cast<const typename Elem<E>::Frag *>(lds + o);
        } else if constexpr (sizeof(E) == 4) {
            const int o = (base ^ (c0 * 4)) + at + sub * 16 * (kCpl * 16);
            f32x4 v;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const float *>(lds + o + i * (kCpl * 16));
            return v;
        } else {
            // the transposing read: 16 lanes fetch 4 lines x 16 columns, lane m gets
            // column m (line + 4 has the same chunk order)
            typedef __attribute__((address_space(3))) i16x4 lds_v;
            const int o = (base ^ (c0 * 2)) + at + sub * 32 * (kCpl * 16);
            union { i16x4 h[2]; bf16x8 f; } u;
            u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v *)(lds + o));
            u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v *)(lds + o + 4 * kCpl * 16));
            return u.f;
        }
    }
};

// Elements [e, e + kEpc) of a line that has `len` elements, zeros past it; any
// element alignment.
template <class E>
__device__ inline u32x4 load_chunk(const E *line, int e, int len) {
    constexpr int kEpc = Elem<E>::kEpc;
    if (line == nullptr || e >= len) return u32x4{0, 0, 0, 0};
    if (e + kEpc <= len) {
        const typename Elem<E>::Vec v = *reinterpret_cast<const typename Elem<E>::Vec *>(line + e);
        return u32x4{v[0], v[1], v[2], v[3]};
    }
    // the end of a line: every element is loaded, of those past it the last (loads under a
    // condition each wait for the one before)
    union { u32x4 v; E s[kEpc]; } u;
    E at[kEpc];
#pragma unroll
    for (int i = 0; i < kEpc; ++i) at[i] = line[min(e + i, len - 1)];
#pragma unroll
    for (int i = 0; i < kEpc; ++i) u.s[i] = e + i < len ? at[i] : static_cast<E>(0.0f);
    return u.v;
}

// Four neighbouring elements from column c on, where the line of m columns has them.
template <class E>
__device__ inline void store_four(E *line, int c, int m, f32x4 v) {
    typename Elem<E>::Out4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = static_cast<E>(v[e]);
    if (c + 4 <= m) {
        *reinterpret_cast<typename Elem<E>::Out4 *>(line + c) = o;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c + e < m) line[c + e] = o[e];
    }
}

// Operand fragment j of V 16-byte vectors: element j of each.
__device__ inline bf16x8 column(const u32x4 (&in)[8], int j) {
    union { u32x4 v; bf16x8 f; } o;
    const uint32_t sel = j & 1 ? 0x07060302u : 0x05040100u;   // high or low halves
#pragma unroll
    for (int i = 0; i < 4; ++i) o.v[i] = __builtin_amdgcn_perm(in[2 * i + 1][j >> 1], in[2 * i][j >> 1], sel);
    return o.f;
}
__device__ inline f32x4 column(const u32x4 (&in)[4], int j) {
    return f32x4{__uint_as_float(in[0][j]), __uint_as_float(in[1][j]), __uint_as_float(in[2][j]), __uint_as_float(in[3][j])};
}

// Four values of a low-rank intermediate, at column c of its 128-byte block.  (A finite value
// whose high part would round to an infinity has the largest bf16 there: the low part holds
// the rest.)
template <class E>
__device__ inline void store_low(char *block, int c, f32x4 v) {
    if constexpr (sizeof(E) == 4) {
        *reinterpret_cast<f32x4 *>(block + c * 4) = v;
    } else {
        constexpr float kTop = 0x1.FEp127f;
        bf16x4 hi, lo;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float inner = __builtin_isfinite(v[e]) ? fminf(fmaxf(v[e], -kTop), kTop) : v[e];
            hi[e] = static_cast<__bf16>(inner);
            lo[e] = static_cast<__bf16>(__builtin_isfinite(v[e]) ? v[e] - static_cast<float>(hi[e]) : 0.0f);
        }
        *reinterpret_cast<bf16x4 *>(block + c * 2) = hi;
        *reinterpret_cast<bf16x4 *>(block + kLowBytes / 2 + c * 2) = lo;
    }
}

// Number of the workgroup in a wide_grid.  (Rows of a constant length: to read the grid's
// took 0.2 us at the start of a kernel.)
template <int THREADS>
__device__ inline int block_id() {
    return static_cast<int>(blockIdx.y * static_cast<uint32_t>(grid_row(THREADS)) + blockIdx.x);
}

// 16 bytes of every lane from memory into LDS, lane after lane from the wave's
// uniform address on.
__device__ inline void load_lds(const char *src, char *dst) {
    typedef const __attribute__((address_space(1))) void *global_p;
    typedef __attribute__((address_space(3))) void *lds_p;
    __builtin_amdgcn_global_load_lds((global_p)src, (lds_p)dst, 16, 0, 0);
}
// LDS written by other lanes of the wave before this point may be read after it, and
// the other way round (the lanes run together: the compiler has to keep the order).
__device__ inline void wave_lds() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
template <int VM>
__device__ inline void wait_vm() {    // at most VM vector-memory loads in flight
    __builtin_amdgcn_s_waitcnt(0x0F70 | (VM & 15) | (VM >> 4) << 14);
}
__device__ inline void wait_lds() { __builtin_amdgcn_s_waitcnt(0xC07F); }   // every LDS access done
__device__ inline void barrier() {    // execution and LDS order; does not wait for loads in flight
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// ---------------------------------------------------------------- staged products
// acc[i][j] += X W over `stages` stages (at least one): RF row fragments from line x0 of the
// X tile, CF column fragments from line w0 of the W tile; each buffer holds an X
// tile, then a W tile.  issue(buffer, stage) starts the loads of a stage into LDS, in
// order of stages.
//
// Two buffers and one barrier a stage.  A stage is two halves of RF groups, a group
// the CF products of one X fragment.  Fragments are read from LDS kAhead groups
// before they are multiplied, across halves and stages, in the order written here: left
// to itself the compiler reads and waits, and reads and products add up (2.1 us
// for a stage of 256 x 256 x 64 whose products take 1.0).  At the barrier, kAhead
// groups before the end of the stage, every wave has read all of its buffer: the
// loads of the stage after the next go into it, and those of the next, issued a
// stage before, have arrived.
template <class E, class XT, class WT, int RF, int CF, class Issue>
__device__ inline void run_stages(int stages, Issue issue, char *buf0, char *buf1, int x0, int w0, int lane,
                                  f32x4 (&acc)[RF][CF]) {
    using El = Elem<E>;
    constexpr int kAhead = RF / 2, kBarrier = 2 * RF - kAhead;
    typename El::Frag x[RF], w[2][CF];
    int xb = XT::base(lane), wb = WT::base(lane);
    auto read_x = [&](const char *b, int group) {        // groups 0 .. 2 RF - 1 of a stage
        x[group % RF] = XT::frag(b, 0, x0 + group % RF * 16, group / RF, xb);
    };
    auto read_w = [&](const char *b, int half, int j) { w[half][j] = WT::frag(b, XT::kBytes, w0 + j * 16, half, wb); };
    auto arrived = [&] {
        wait_lds();
        wait_vm<0>();
        barrier();
    };
    auto first = [&](const char *b) {
#pragma unroll
        for (int j = 0; j < CF; ++j) read_w(b, 0, j);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) read_x(b, i);
    };
    auto stage = [&](char *cur, char *next, int s) {
#pragma unroll
        for (int group = 0; group < 2 * RF; ++group) {
            // addresses are made where they are used (kept, they would fill the registers)
            if (group % RF == 0) asm volatile("" : "+v"(xb), "+v"(wb));
            if (group == kBarrier) {
                arrived();
                if (s + 2 < stages) issue(cur, s + 2);
            }
            const int to = group + kAhead;
            if (to < 2 * RF) read_x(cur, to);
            else read_x(next, to - 2 * RF);
#pragma unroll
            for (int j = 0; j < CF; ++j) {
                if (group == j * RF / CF) read_w(cur, 1, j);
                if (group == kBarrier + j * kAhead / (2 * CF)) read_w(next, 0, j);
            }
#pragma unroll
            for (int j = 0; j < CF; ++j) acc[group % RF][j] = El::mma(w[group / RF][j], x[group % RF], acc[group % RF][j]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // An odd stage goes first: the sums then pass through one loop, with no other way
    // to its end (merging them would cost the registers twice).
    int s = stages & 1;
    if (s) {
        issue(buf1, 0);
        arrived();
        if (stages > 1) issue(buf0, 1);
        first(buf1);
        stage(buf1, buf0, 0);
    } else {
        issue(buf0, 0);
        arrived();
        issue(buf1, 1);
        first(buf0);
    }
    for (; s < stages; s += 2) {
        stage(buf0, buf1, s);
        stage(buf1, buf0, s + 1);
    }
}

// The same with four buffers, for tiles whose products take less than the way from
// memory: three stages are in flight.  issue is also told the stage modulo 4, as a
// constant.  (Few sums: the loop may be left anywhere.)
template <class E, class XT, class WT, int RF, int CF, int LOADS, class Issue>
__device__ inline void run_stages_deep(int stages, Issue issue, char *buf0, char *buf1, char *buf2, char *buf3, int x0, int w0,
                                       int lane, f32x4 (&acc)[RF][CF]) {
    using El = Elem<E>;
    typename El::Frag x[2][RF], w[2][CF];
    const int xb = XT::base(lane), wb = WT::base(lane);
    auto read = [&](const char *b, int half) {
#pragma unroll
        for (int j = 0; j < CF; ++j) w[half][j] = WT::frag(b, XT::kBytes, w0 + j * 16, half, wb);
#pragma unroll
        for (int i = 0; i < RF; ++i) x[half][i] = XT::frag(b, 0, x0 + i * 16, half, xb);
    };
    auto multiply = [&](int half) {
#pragma unroll
        for (int i = 0; i < RF; ++i)
#pragma unroll
            for (int j = 0; j < CF; ++j) acc[i][j] = El::mma(w[half][j], x[half][i], acc[i][j]);
        __builtin_amdgcn_sched_barrier(0);
    };
    auto stage = [&](char *cur, char *next, auto slot, int s) {
        read(cur, 1);
        multiply(0);
        wait_lds();
        if (s + 3 < stages) wait_vm<2 * LOADS>();
        else wait_vm<0>();
        barrier();
        if (s + 4 < stages) issue(cur, s + 4, slot);
        read(next, 0);
        multiply(1);
    };
    constexpr std::integral_constant<int, 0> c0{};
    constexpr std::integral_constant<int, 1> c1{};
    constexpr std::integral_constant<int, 2> c2{};
    constexpr std::integral_constant<int, 3> c3{};
    issue(buf0, 0, c0);
    if (stages > 1) issue(buf1, 1, c1);
    if (stages > 2) issue(buf2, 2, c2);
    if (stages > 3) {
        issue(buf3, 3, c3);
        wait_vm<3 * LOADS>();
    } else {
        wait_vm<0>();
    }
    barrier();
    read(buf0, 0);
    for (int s = 0;;) {
        stage(buf0, buf1, c0, s);
        if (++s >= stages) break;
        stage(buf1, buf2, c1, s);
        if (++s >= stages) break;
        stage(buf2, buf3, c2, s);
        if (++s >= stages) break;
        stage(buf3, buf0, c3, s);
        if (++s >= stages) break;
    }
}

}  // namespace hwr
