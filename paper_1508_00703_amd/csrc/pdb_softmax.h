// The statistics of rows of logits (gfx950, wave64), shared by the operators over a
// vocabulary.  Internal header, not installed.
//
// Of a row z (V logits, temperature T, c = log2(e) / T):
//   m = max z,  y_j = c (z_j - m),  S = sum 2^y_j,  A = sum 2^y_j y_j.
// One pass keeps a running m per wave and rescales S and A in the rare tiles
// that raise it (a wave's maximum is raised about ln(tiles) times), so an
// element costs one exponential.  y is one fma on M = fl(c m) while |M| is below
// 2^20: what rounding M shifts, up to 2^-5, is the same for every element and is taken
// out of log S at the end.  Where |M| is larger (masks like -1e30, a type's lowest
// value, temperatures far below the logits) the shift would leave the exponential's
// range, from 2^31 on, and cost the sums their accuracy before: y is c (z - m) there
// instead.  m starts at the lowest finite float, so a logit of -inf gives 2^y = 0
// without a special case and S = 0 says that a row has nothing else.  A takes y no
// lower than kLogFloor, where 2^y is 0: 0 log 0 counts as 0.
#pragma once

#include <float.h>

#include "pdb_math.h"
#include "pdb_vec.h"

namespace pdbk {

constexpr float kLog2e = 0x1.715476p+0f;
constexpr float kLn2 = 0x1.62e430p-1f;
constexpr float kLogFloor = -160.0f;  // 2^-160 is 0 in binary32
constexpr int kTileVecs = 4;          // vectors a thread has in flight
constexpr float kNegInf = -__builtin_inff();
constexpr float kNan = __builtin_nanf("");

// The W waves that have a row (or a part of one): a block of 4 has one such team or
// four of one wave each; other teams are whole blocks.
template <int W>
struct Team {
    static constexpr int kThreads = W * kWave;
    static constexpr int kPerBlock = W == 1 ? kBlock / kWave : 1;
    static __device__ __forceinline__ int thread() {
        return W == 1 ? lane_id() : (int)threadIdx.x;
    }
    static __device__ __forceinline__ int wave() { return W == 1 ? 0 : wave_in_block(); }
    // which of the block's teams this is (the same in all its lanes)
    static __device__ __forceinline__ int here() {
        return W == 1 ? __builtin_amdgcn_readfirstlane(wave_in_block()) : 0;
    }
    // what the team wrote to LDS is seen by the team (a wave's accesses run in order)
    static __device__ __forceinline__ void sync() {
        if constexpr (W == 1) {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        } else {
            __syncthreads();
        }
    }
    // the same, with the loads and stores that are under way left under way
    static __device__ __forceinline__ void sync_lds() {
        if constexpr (W == 1) {
            sync();
        } else {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
    }
};

struct Stat {  // of a row, or of a part of one (a: in powers of 2)
    float m, s, a;
};
__device__ __forceinline__ Stat empty_stat() { return {-FLT_MAX, 0.0f, 0.0f}; }

__device__ __forceinline__ float exp2_raw(float y) { return __builtin_amdgcn_exp2f(y); }

// max over the wave (NaN ignored), by the integers in the floats' order
__device__ __forceinline__ float wave_max_f32(float v) {
    int i = __float_as_int(v);
    i ^= (i >> 31) & 0x7FFFFFFF;
    i = wave_max_dpp(i);
    i ^= (i >> 31) & 0x7FFFFFFF;
    return __int_as_float(i);
}
// a value that all lanes of the wave hold, as a scalar
__device__ __forceinline__ float wave_uniform(float v) {
    return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v)));
}

// Whether y is taken as c z - M, and how much larger it is than c (z - m) then.
__device__ __forceinline__ bool in_range(float m, float c) { return fabsf(m * c) < 0x1p20f; }
__device__ __forceinline__ float shift_of(float m, float c) {
    return in_range(m, c) ? __builtin_fmaf(m, c, -(m * c)) : 0.0f;
}
__device__ __forceinline__ float power_of(float z, float m, float c) {
    return in_range(m, c) ? __builtin_fmaf(z, c, -(m * c)) : (z - m) * c;
}

// t's sums on the maximum m >= t.m
__device__ __forceinline__ void rescale(Stat &t, float m, float c) {
    const float up = in_range(m, c) && in_range(t.m, c)
                         ? t.m * c - m * c
                         : (t.m - m) * c + (shift_of(m, c) - shift_of(t.m, c));
    const float y = fmaxf(up, 2.0f * kLogFloor);
    const float f = exp2_raw(y);
    t.a = f * __builtin_fmaf(y, t.s, t.a);
    t.s *= f;
    t.m = m;
}
__device__ __forceinline__ Stat join(Stat a, Stat b, float c) {
    const float m = fmaxf(a.m, b.m);
    rescale(a, m, c);
    rescale(b, m, c);
    return {m, a.s + b.s, a.a + b.a};
}

// The team's statistics from its waves' (each wave's m is the same in its lanes,
// its sums are spread over them); the same in every thread.
template <int W>
__device__ __forceinline__ Stat team_stat(Stat w, float c) {
    w.s = wave_sum64(w.s);
    w.a = wave_sum64(w.a);
    if constexpr (W == 1) {
        return w;
    } else {
        __shared__ float s_m[W], s_s[W], s_a[W];
        if (lane_id() == 0) {
            s_m[wave_in_block()] = w.m;
            s_s[wave_in_block()] = w.s;
            s_a[wave_in_block()] = w.a;
        }
        __syncthreads();
        Stat t = {s_m[0], s_s[0], s_a[0]};
#pragma unroll
        for (int k = 1; k < W; ++k) t = join(t, Stat{s_m[k], s_s[k], s_a[k]}, c);
        __syncthreads();
        return t;
    }
}

// A row's statistics from its parts', a part to a lane; the same in every thread.
constexpr int64_t kMostParts = kWave;
__device__ __forceinline__ Stat join_parts(const float *part_stat, int64_t i, int parts, float c) {
    const float *q = part_stat + 3 * (i * parts + lane_id());
    Stat t = empty_stat();
    if (lane_id() < parts) t = {q[0], q[1], q[2]};
    rescale(t, wave_max_f32(t.m), c);
    return {t.m, wave_sum64(t.s), wave_sum64(t.a)};
}
__device__ __forceinline__ void put_part(float *part_stat, int64_t w, const Stat &t) {
    part_stat[3 * w] = t.m;
    part_stat[3 * w + 1] = t.s;
    part_stat[3 * w + 2] = t.a;
}

// What a row's statistics say: log of the sum over exp((z - m) / T), -inf of an
// empty row, and the entropy.
__device__ __forceinline__ float log_sum(const Stat &t, float c) {
    if (t.s == 0.0f) return kNegInf;
    return (__builtin_amdgcn_logf(t.s) - shift_of(t.m, c)) * kLn2;
}
__device__ __forceinline__ float entropy_of(const Stat &t) {
    return t.s == 0.0f ? 0.0f : (__builtin_amdgcn_logf(t.s) - t.a / t.s) * kLn2;
}
// log probability of a logit: (z - m) / T - log S; -inf in a row without any
__device__ __forceinline__ float log_prob(float z, float m, float ls, float inv_t) {
    return ls == kNegInf ? kNegInf : (z - m) * inv_t - ls;
}

// ----------------------------------------------------------------------------
// A row is `full` whole vectors and a tail of rem < kVec elements.  The tail is the
// last part's: one element to a lane of the team's first wave.

template <int DT>
__device__ __forceinline__ u32x4 fill_neg_inf() {
    const uint32_t w = DT == PDB_F32 ? 0xFF800000u : DT == PDB_BF16 ? 0xFF80FF80u : 0xFC00FC00u;
    return u32x4{w, w, w, w};
}

// Where a thread's vector is, j vectors behind the team's first at `row`: an address
// that the team shares and a lane's own 32-bit offset.
template <int W>
__device__ __forceinline__ const char *vec_at(const char *row, int j) {
    return row + (int64_t)j * 16 + (uint32_t)(Team<W>::thread() * 16);
}
template <int W>
__device__ __forceinline__ char *vec_at(char *row, int j) {
    return row + (int64_t)j * 16 + (uint32_t)(Team<W>::thread() * 16);
}

// A thread's tile: kTileVecs vectors, a team apart, as they are stored; -inf from
// vector `end` on.  j: the team's first.
struct Tile {
    u32x4 r[kTileVecs];
};
template <int DT, int W>
__device__ __forceinline__ Tile load_tile(const char *row, int j, int end) {
    constexpr int kT = Team<W>::kThreads;
    Tile t;
    if (j + kTileVecs * kT <= end) {
#pragma unroll
        for (int u = 0; u < kTileVecs; ++u) t.r[u] = load16(vec_at<W>(row, j + u * kT));
    } else {
#pragma unroll
        for (int u = 0; u < kTileVecs; ++u) {
            t.r[u] = fill_neg_inf<DT>();
            if (j + u * kT + Team<W>::thread() < end) t.r[u] = load16(vec_at<W>(row, j + u * kT));
        }
    }
    return t;
}

// the largest element of a vector (NaN ignored)
template <int DT>
__device__ __forceinline__ float vec_max(u32x4 r) {
    constexpr int kV = Elem<DT>::kVec;
    float x[kV];
    unpack<DT>(r, x);
    float h = x[0];
#pragma unroll
    for (int e = 1; e < kV; ++e) h = fmaxf(h, x[e]);
    return h;
}

// N vectors' elements into the sums, on the wave's maximum t.m.
template <int DT, bool ENT, int N>
__device__ __forceinline__ void add_vecs(u32x4 (&r)[N], float c, Stat &t) {
    constexpr int kV = Elem<DT>::kVec;
    // unpacked again, after the maximum: keeping the elements would double the registers
#pragma unroll
    for (int u = 0; u < N; ++u) asm volatile("" : "+v"(r[u]));
    auto add = [&](auto y_of) {
#pragma unroll
        for (int u = 0; u < N; ++u) {
            float x[kV];
            unpack<DT>(r[u], x);
#pragma unroll
            for (int e = 0; e < kV; ++e) {
                const float y = y_of(x[e]);
                const float p = exp2_raw(y);
                t.s += p;
                if (ENT) t.a = __builtin_fmaf(p, fmaxf(y, kLogFloor), t.a);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    const float m = wave_uniform(t.m), shift = -(m * c);
    if (in_range(m, c))
        add([&](float z) { return __builtin_fmaf(z, c, shift); });
    else
        add([&](float z) { return (z - m) * c; });
    // the sums are formed here, not wherever they are next wanted
    asm volatile("" : "+v"(t.s), "+v"(t.a));
}

// A tile into the statistics; lm: the largest of each of its vectors.
template <int DT, bool ENT>
__device__ __forceinline__ void add_tile(Tile tile, float c, Stat &t, float (&lm)[kTileVecs]) {
    float all = kNegInf;
#pragma unroll
    for (int u = 0; u < kTileVecs; ++u) {
        lm[u] = vec_max<DT>(tile.r[u]);
        all = fmaxf(all, lm[u]);
    }
    if (__any(all > t.m)) rescale(t, fmaxf(t.m, wave_max_f32(all)), c);
    add_vecs<DT, ENT>(tile.r, c, t);
}

// The tail's element of this thread; -inf where it has none.
template <int DT, int W>
__device__ __forceinline__ float tail_elem(const char *row, int full, int rem) {
    const int t = Team<W>::thread();
    return t < rem ? load1<DT>(row, (int64_t)full * Elem<DT>::kVec + t) : kNegInf;
}
template <bool ENT>
__device__ __forceinline__ void add_elem(float z, float c, Stat &t) {
    if (__any(z > t.m)) rescale(t, fmaxf(t.m, wave_max_f32(z)), c);
    const float y = power_of(z, t.m, c);
    const float p = exp2_raw(y);
    t.s += p;
    if (ENT) t.a = __builtin_fmaf(p, fmaxf(y, kLogFloor), t.a);
}

// The vectors [first, end) of a row: f(j, x) replaces the elements of vector j.
template <int DT, int W, typename F>
__device__ __forceinline__ void map_row(const char *row, char *out, int first, int end, F f) {
    constexpr int kV = Elem<DT>::kVec, kT = Team<W>::kThreads;
    for (int j = first; j < end; j += kTileVecs * kT) {
        const Tile tile = load_tile<DT, W>(row, j, end);
#pragma unroll
        for (int u = 0; u < kTileVecs; ++u) {
            const int q = j + u * kT + Team<W>::thread();
            if (q >= end) break;
            float x[kV];
            unpack<DT>(tile.r[u], x);
            f(q, x);
            store16(vec_at<W>(out, j + u * kT), pack<DT>(x));
        }
    }
}
template <int DT, int W>
__device__ __forceinline__ void zero_row(char *out, int first, int end, int full, int rem) {
    constexpr int kV = Elem<DT>::kVec;
    const int t = Team<W>::thread();
    for (int j = first; j + t < end; j += Team<W>::kThreads)
        store16(vec_at<W>(out, j), u32x4{0, 0, 0, 0});
    if (t < rem) store1<DT>(out, (int64_t)full * kV + t, 0.0f);
}

// ----------------------------------------------------------------------------
// Work item w: row i, part `part` of `parts` (rows are cut only where they are few,
// so that 32 bits hold w there).
struct Work {
    int64_t i;
    int part;
    __device__ __forceinline__ Work(int64_t w, int parts) : i(w), part(0) {
        if (parts > 1) {
            i = (uint32_t)w / (uint32_t)parts;
            part = (int)((uint32_t)w - (uint32_t)i * (uint32_t)parts);
        }
    }
};

// How rows are cut into parts: up to kWantBlocks blocks when there are few rows
// (four a compute unit), none with less than a tile.
constexpr int64_t kWantBlocks = 1024;
struct Parts {
    int parts;
    int vecs;  // of a part
};
inline Parts cut_rows(int64_t n, int64_t v, int64_t vec, int64_t most) {
    const int64_t all = std::max<int64_t>(v / vec, 1), tile = (int64_t)kBlock * kTileVecs;
    int64_t parts =
        std::min(std::min(kWantBlocks / std::max<int64_t>(n, 1), cdiv(all, tile)), most);
    parts = std::max<int64_t>(parts, 1);
    const int64_t vecs = cdiv(cdiv(all, parts), kBlock) * kBlock;
    return {(int)cdiv(all, vecs), (int)vecs};
}
inline bool good_temp(float t) { return t > 0.0f && t <= FLT_MAX && kLog2e / t <= FLT_MAX; }
inline size_t stat_bytes(int64_t n) { return (size_t)align_up(n * kMostParts * 12); }
// Blocks for `work` items of a team each; every kernel here takes any number of
// items a team.
inline unsigned blocks_for(int64_t work, int per_block = 1) {
    return (unsigned)std::min<int64_t>(cdiv(work, per_block), 1 << 22);
}
// A wave to a row, instead of a block.  Rows of few vectors leave a block's threads
// idle (16,384 rows of 4,000 bf16: 30 us against 49, with the gradient 45 against 51;
// of 8,000 the block is even or ahead).  With a selection, which costs each wave and
// joins a block's, also longer rows where every compute unit still has eight (3,000 of
// 40,000 with 5 alternatives: 58 us against 66, 8,192 of 32,768 with 64: 156 against
// 165; 1,600 of 65,536 with 1: 61 against 55).
inline bool wave_rows(const Parts &cut, int64_t n, int64_t v, int64_t vec, bool selection) {
    if (cut.parts > 1) return false;
    return v <= vec * (selection ? 1024 : 512) || (selection && n >= 2048);
}

}  // namespace pdbk
