// Operators over rows of logits (gfx950, wave64): log probabilities of given
// tokens with entropy and the best alternatives, their gradient, and the
// distillation loss from a teacher's top logits with its gradient.
//
// All of them rest on the statistics of a row z (V logits, temperature T, c =
// log2(e) / T):
//   m = max z,  y_j = c (z_j - m),  S = sum 2^y_j,  A = sum 2^y_j y_j.
// One pass keeps a running m per wave and rescales S and A in the rare tiles
// that raise it (a wave's maximum is raised about ln(tiles) times), so an
// element costs one exponential.  y is one fma on M = fl(c m): what rounding M
// shifts is the same for every element and is taken out of log S at the end.
// Where |M| nears the range's end (rows of a type's lowest value) y is c (z - m)
// instead.  m starts at the lowest finite float, so a logit of -inf gives 2^y = 0
// without a special case and S = 0 says that a row has nothing else.  A takes y no
// lower than kLogFloor, where 2^y is 0: 0 log 0 counts as 0.
//
// A row is one block's, or with few rows several blocks' (parts), whose
// statistics are joined by a second kernel.
#include <float.h>

#include <type_traits>

#include "pdb_math.h"
#include "pdb_vec.h"

namespace pdbk {
namespace {

constexpr float kLog2e = 0x1.715476p+0f;
constexpr float kLn2 = 0x1.62e430p-1f;
constexpr float kLogFloor = -160.0f;  // 2^-160 is 0 in binary32
constexpr int kTileVecs = 4;          // vectors a thread has in flight
constexpr int kWaves = kBlock / kWave;
constexpr float kNegInf = -__builtin_inff();
constexpr float kNan = __builtin_nanf("");

struct Stat {  // of a row, or of a part of one (a: in powers of 2)
    float m, s, a;
};

__device__ __forceinline__ float exp2_raw(float y) { return __builtin_amdgcn_exp2f(y); }

// max over the wave (NaN ignored), by the integers in the floats' order
__device__ __forceinline__ float wave_max_f32(float v) {
    int i = __float_as_int(v);
    i ^= (i >> 31) & 0x7FFFFFFF;
    i = wave_max_dpp(i);
    i ^= (i >> 31) & 0x7FFFFFFF;
    return __int_as_float(i);
}

// Whether y may be taken as c z - M.
__device__ __forceinline__ bool in_range(float m, float c) { return fabsf(m * c) < 1e38f; }
// a value that all lanes of the wave hold, as a scalar
__device__ __forceinline__ float wave_uniform(float v) {
    return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v)));
}

// t's sums on the maximum m >= t.m
__device__ __forceinline__ void rescale(Stat &t, float m, float c) {
    const float up = in_range(m, c) ? t.m * c - m * c : (t.m - m) * c;
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

// The block's statistics from its waves', the same in every thread.
__device__ Stat block_stat(Stat w, float c) {
    __shared__ float s_m[kWaves], s_s[kWaves], s_a[kWaves];
    w.s = wave_sum64(w.s);
    w.a = wave_sum64(w.a);
    if (lane_id() == 0) {
        s_m[wave_in_block()] = w.m;
        s_s[wave_in_block()] = w.s;
        s_a[wave_in_block()] = w.a;
    }
    __syncthreads();
    Stat t = {s_m[0], s_s[0], s_a[0]};
#pragma unroll
    for (int k = 1; k < kWaves; ++k) t = join(t, Stat{s_m[k], s_s[k], s_a[k]}, c);
    __syncthreads();
    return t;
}

// What a row's statistics say: log of the sum over exp((z - m) / T), -inf of an
// empty row, and the entropy.
__device__ __forceinline__ float log_sum(const Stat &t, float c) {
    if (t.s == 0.0f) return kNegInf;
    const float l = __builtin_amdgcn_logf(t.s);
    return (in_range(t.m, c) ? l - __builtin_fmaf(t.m, c, -(t.m * c)) : l) * kLn2;
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
// last part's: one element to a lane of the first wave.

template <int DT>
__device__ __forceinline__ u32x4 fill_neg_inf() {
    const uint32_t w = DT == PDB_F32 ? 0xFF800000u : DT == PDB_BF16 ? 0xFF80FF80u : 0xFC00FC00u;
    return u32x4{w, w, w, w};
}

// A thread's tile: kTileVecs vectors, kBlock apart, as they are stored; -inf from
// vector `end` on.
struct Tile {
    u32x4 r[kTileVecs];
};
template <int DT>
__device__ __forceinline__ Tile load_tile(const char *row, int j, int end) {
    Tile t;
    if (j - (int)threadIdx.x + kTileVecs * kBlock <= end) {
#pragma unroll
        for (int u = 0; u < kTileVecs; ++u) t.r[u] = load16(row + (int64_t)(j + u * kBlock) * 16);
    } else {
#pragma unroll
        for (int u = 0; u < kTileVecs; ++u) {
            t.r[u] = fill_neg_inf<DT>();
            if (j + u * kBlock < end) t.r[u] = load16(row + (int64_t)(j + u * kBlock) * 16);
        }
    }
    return t;
}

// 2^(c (z - m)) of a teacher's logit
__device__ __forceinline__ float exp2_of(float z, float m, float c) {
    return exp2_raw(in_range(m, c) ? __builtin_fmaf(z, c, -(m * c)) : (z - m) * c);
}

// A tile into the statistics; lm: the largest of each of its vectors.
template <int DT, bool ENT>
__device__ __forceinline__ void add_tile(Tile tile, float c, Stat &t, float (&lm)[kTileVecs]) {
    constexpr int kV = Elem<DT>::kVec;
    float all = kNegInf;
#pragma unroll
    for (int u = 0; u < kTileVecs; ++u) {
        float x[kV];
        unpack<DT>(tile.r[u], x);
        float h = x[0];
#pragma unroll
        for (int e = 1; e < kV; ++e) h = fmaxf(h, x[e]);
        lm[u] = h;
        all = fmaxf(all, h);
    }
    if (__any(all > t.m)) rescale(t, fmaxf(t.m, wave_max_f32(all)), c);
    // unpacked again below: keeping the elements would double the registers
#pragma unroll
    for (int u = 0; u < kTileVecs; ++u) asm volatile("" : "+v"(tile.r[u]));
    auto add = [&](auto y_of) {
#pragma unroll
        for (int u = 0; u < kTileVecs; ++u) {
            float x[kV];
            unpack<DT>(tile.r[u], x);
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

// The tail's element of this lane; -inf where it has none.
template <int DT>
__device__ __forceinline__ float tail_elem(const char *row, int full, int rem) {
    return (int)threadIdx.x < rem ? load1<DT>(row, (int64_t)full * Elem<DT>::kVec + threadIdx.x)
                                  : kNegInf;
}
template <bool ENT>
__device__ __forceinline__ void add_elem(float z, float c, Stat &t) {
    if (__any(z > t.m)) rescale(t, fmaxf(t.m, wave_max_f32(z)), c);
    const float y = in_range(t.m, c) ? __builtin_fmaf(z, c, -(t.m * c)) : (z - t.m) * c;
    const float p = exp2_raw(y);
    t.s += p;
    if (ENT) t.a = __builtin_fmaf(p, fmaxf(y, kLogFloor), t.a);
}

// ----------------------------------------------------------------------------
// the K best of a row, ties to the lowest index
//
// A logit's rank key orders like the logit, in as many bits as its type has;
// 1 is NaN, 0 nothing.  The row's K best lie in the K best of its vectors, ordered
// by (largest key, index): an element of any other has K better ones.  So while a
// row streams by, only its vectors' maxima are looked at: those better than a bound
// are kept in LDS.  The bound is the K-th best of K or more vectors met so far.
// The first tile sets it, from the K-th best of a wave's vectors; when the kept ones
// would overflow, it is raised to the K-th best of those kept and the tile's, which
// leaves K, whatever the data.  The K vectors that remain are read again, and their
// elements put in order.  The K-th best of a set spread over the block is found by a
// binary search over the bits of its key, counting with ballots.

constexpr int kKeep = 512;             // vectors kept in LDS
constexpr int kCand = PDB_MAX_TOP * 8; // elements of K vectors
static_assert(kCand >= kKeep && kCand % kBlock == 0 && kKeep % kBlock == 0, "whole rounds");

template <int DT>
struct Key {
    static constexpr int kShift = DT == PDB_F32 ? 0 : DT == PDB_BF16 ? 16 : 13;
    static constexpr int kBits = 32 - kShift;
};
template <int DT>
__device__ __forceinline__ uint32_t rank_key(float z) {
    if (z != z) return 1;
    const uint32_t b = __float_as_uint(z + 0.0f);  // -0 ranks as 0
    return (b ^ (b & 0x80000000u ? 0xFFFFFFFFu : 0x80000000u)) >> Key<DT>::kShift;
}
template <int DT>
__device__ __forceinline__ float logit_of(uint32_t key) {
    if (key <= 1) return kNan;
    const uint32_t k = key << Key<DT>::kShift;
    const uint32_t low = (1u << Key<DT>::kShift) - 1u;
    return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~(k | low));
}

__device__ __forceinline__ int block_count(int wave_count, int &turn) {
    __shared__ int s_count[2][kWaves];
    if (lane_id() == 0) s_count[turn][wave_in_block()] = wave_count;
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) all += s_count[turn][w];
    turn ^= 1;
    return all;
}

struct Bound {  // an element passes when its key is larger, or equal at an index <= at
    uint32_t key, at;
};
__device__ __forceinline__ bool passes(const Bound &b, uint32_t key, uint32_t at) {
    return key > b.key || (key == b.key && at <= b.at);
}

// The bound that exactly the k best of the block's N * kBlock (key, index)
// pass, or every valid one (key > 0) if those are fewer.  Indices < 2^at_bits.
template <int DT, int N>
__device__ Bound kth_best(const uint32_t (&key)[N], const uint32_t (&at)[N], int k, int at_bits) {
    int turn = 0;
    uint32_t t = 0;
    int enough = 0;  // how many are >= t, once t > 0
#pragma unroll 1
    for (int b = Key<DT>::kBits - 1; b >= 0; --b) {
        const uint32_t cand = t | (1u << b);
        int w = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) w += __popcll(__ballot(key[i] >= cand));
        const int all = block_count(w, turn);
        if (all >= k) {
            t = cand;
            enough = all;
            if (all == k) break;  // these are the k best, whatever the other bits
        }
    }
    Bound r = {t, 0xFFFFFFFFu};
    if (t == 0) r.key = 1;
    if (t == 0 || enough == k) return r;
    int w = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) w += __popcll(__ballot(key[i] > t));
    const int need = k - block_count(w, turn);
    uint32_t x = at_bits >= 32 ? 0xFFFFFFFFu : (1u << at_bits) - 1u;
#pragma unroll 1
    for (int b = at_bits - 1; b >= 0; --b) {
        const uint32_t cand = x & ~(1u << b);
        w = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) w += __popcll(__ballot(key[i] == t && at[i] <= cand));
        if (block_count(w, turn) >= need) x = cand;
    }
    r.at = x;
    return r;
}

// A candidate as one word that is larger the better it is.
__device__ __forceinline__ uint64_t candidate(uint32_t key, uint32_t at) {
    return (uint64_t)key << 32 | ~at;
}
__device__ __forceinline__ uint32_t key_of(uint64_t c) { return (uint32_t)(c >> 32); }
__device__ __forceinline__ uint32_t index_of(uint64_t c) { return ~(uint32_t)c; }

constexpr int kRanked = 2 * kBlock;  // candidates that are ranked against each other, at most
struct TopLds {
    alignas(16) uint64_t c[kCand + 8];
    uint32_t rank[kRanked];
    int n;
    int add[3];  // candidates of a tile, in turn
    uint32_t wave[kWaves];
};

__device__ __forceinline__ void push(TopLds &L, uint32_t key, uint32_t at) {
    L.c[atomicAdd(&L.n, 1)] = candidate(key, at);
}

inline int bits_for(int64_t count) {
    int b = 0;
    while (b < 31 && ((int64_t)1 << b) < count) ++b;
    return b;
}

// The k best of the first n <= M candidates in L and of the given ones stay in L,
// L.n of them; returns the bound.  Every thread calls.
template <int DT, int M, int N>
__device__ __forceinline__ Bound keep_best(TopLds &L, int n, const uint32_t (&more)[N],
                                           const uint32_t (&more_at)[N], int k, int at_bits) {
    constexpr int kN = M / kBlock;
    uint32_t key[kN + N], at[kN + N];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kN; ++i) {
        const int q = i * kBlock + threadIdx.x;
        key[i] = q < n ? key_of(L.c[q]) : 0;
        at[i] = q < n ? index_of(L.c[q]) : 0;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        key[kN + i] = more[i];
        at[kN + i] = more_at[i];
    }
    if (threadIdx.x == 0) L.n = 0;
    const Bound b = kth_best<DT, kN + N>(key, at, k, at_bits);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kN + N; ++i)
        if (key[i] > 0 && passes(b, key[i], at[i])) push(L, key[i], at[i]);
    __syncthreads();
    return b;
}

// The selection over a row part, tile by tile.
template <int DT>
struct Selection {
    static constexpr int kV = Elem<DT>::kVec;
    uint32_t bound;  // its key
    float least;     // its logit: what is not larger is not kept; NaN: everything is
    int n;           // vectors in L

    // every thread; L is free.  tail: this lane's element of the row's tail, of rem,
    // which stands as vector `full`
    __device__ __forceinline__ void start(TopLds &L, float tail, int full, int rem) {
        bound = 0;
        least = kNan;
        n = rem > 0 ? 1 : 0;
        if (threadIdx.x < 3) L.add[threadIdx.x] = 0;
        if (rem > 0 && wave_in_block() == 0) {
            const int best = wave_max_dpp((int)threadIdx.x < rem ? (int)(rank_key<DT>(tail) >> 1) : 0);
            // keys have up to 32 bits: the upper 31 first
            const bool top = (int)threadIdx.x < rem && (int)(rank_key<DT>(tail) >> 1) == best;
            const bool odd = __any(top && (rank_key<DT>(tail) & 1u));
            if (threadIdx.x == 0)
                L.c[0] = candidate((uint32_t)best << 1 | (odd ? 1u : 0u), (uint32_t)full);
        }
        __syncthreads();
    }

    // The largest logit under a key: where the bound comes from this very tile,
    // equal ones count too (in later tiles they stand behind it).  0's is two keys
    // down: the one between is -0's, which equals 0.
    static __device__ __forceinline__ float below(uint32_t key) {
        const uint32_t step = key == (0x80000000u >> Key<DT>::kShift) ? 2 : 1;
        return key > 2 ? logit_of<DT>(key - step) : kNan;
    }

    // The K-th best of the wave's lanes (kReps = 1, for K that are few of them), or
    // of their vectors; the block takes the waves' best.
    template <int kReps>
    static __device__ __forceinline__ uint32_t wave_bound(const uint32_t (&key)[kReps], int k) {
        uint32_t hi = key[0], lo = key[0];
#pragma unroll
        for (int u = 1; u < kReps; ++u) {
            hi = max(hi, key[u]);
            lo = min(lo, key[u]);
        }
        // the bits above the highest in which two of them differ are everyone's
        hi = (uint32_t)wave_max_dpp((int)(hi >> 1)) << 1 | 1u;
        lo = ~((uint32_t)wave_max_dpp((int)(~lo >> 1)) << 1 | 1u);
        const int bits = 32 - __builtin_clz((hi ^ lo) | 1u);
        uint32_t t = bits >= 32 ? 0 : hi >> bits << bits;
#pragma unroll 1
        for (int bit = bits - 1; bit >= 0; --bit) {
            const uint32_t cand = t | (1u << bit);
            int c = 0;
#pragma unroll
            for (int u = 0; u < kReps; ++u) c += __popcll(__ballot(key[u] >= cand));
            if (c >= k) t = cand;
            if (c == k) break;
        }
        return t;
    }

    __device__ __forceinline__ void first_bound(TopLds &L, const float (&lm)[kTileVecs], int j,
                                                int end, int k) {
        uint32_t key[kTileVecs], t;
#pragma unroll
        for (int u = 0; u < kTileVecs; ++u)
            key[u] = j + u * kBlock < end ? rank_key<DT>(lm[u]) : 0;
        if (k <= kWave / 2) {
            const uint32_t own[1] = {max(max(key[0], key[1]), max(key[2], key[3]))};
            static_assert(kTileVecs == 4, "four vectors");
            t = wave_bound(own, k);
        } else {
            t = wave_bound(key, k);
        }
        if (lane_id() == 0) L.wave[wave_in_block()] = t;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) bound = max(bound, L.wave[w]);
        least = below(bound);
    }

    // Takes the tile (the turn-th of the part) at vector j, lm its vectors' maxima.
    __device__ __forceinline__ void take(TopLds &L, const float (&lm)[kTileVecs], int turn, int j,
                                         int end, int k, int at_bits) {
        if (turn == 0) first_bound(L, lm, j, end, k);
        int mine = 0, at = 0;
#pragma unroll
        for (int u = 0; u < kTileVecs; ++u)
            mine += !(lm[u] <= least) && j + u * kBlock < end;
        if (mine) at = n + atomicAdd(&L.add[turn % 3], mine);
        __syncthreads();
        const int all = n + L.add[turn % 3];
        if (threadIdx.x == 0) L.add[(turn + 2) % 3] = 0;  // the tile's before this one
        if (all <= kKeep) {
            if (mine) {
#pragma unroll
                for (int u = 0; u < kTileVecs; ++u)
                    if (!(lm[u] <= least) && j + u * kBlock < end)
                        L.c[at++] = candidate(rank_key<DT>(lm[u]), (uint32_t)(j + u * kBlock));
            }
            n = all;
            // of the first tile, equal ones were kept: later they are not wanted
            if (turn == 0) least = logit_of<DT>(bound);
        } else {
            uint32_t key[kTileVecs], where[kTileVecs];
#pragma unroll
            for (int u = 0; u < kTileVecs; ++u) {
                where[u] = (uint32_t)(j + u * kBlock);
                key[u] = j + u * kBlock < end ? rank_key<DT>(lm[u]) : 0;
            }
            bound = keep_best<DT, kKeep, kTileVecs>(L, n, key, where, k, at_bits).key;
            n = L.n;
            least = logit_of<DT>(bound);
        }
    }

    // L holds the elements of the vectors left that may be the part's k best, at most
    // kBlock of them
    __device__ __forceinline__ void finish(TopLds &L, const char *row, int full, int rem, int k,
                                           int at_bits) {
        const uint32_t none[1] = {0};
        __syncthreads();
        if (n > PDB_MAX_TOP) {
            bound = keep_best<DT, kKeep, 1>(L, n, none, none, k, at_bits).key;
            n = L.n;
        }
        const int vectors = n, t = threadIdx.x;
        const int j = t < vectors ? (int)index_of(L.c[t]) : 0;
        __syncthreads();
        if (t == 0) L.n = 0;
        __syncthreads();
        if (t < vectors) {
            const uint32_t from = max(bound, 1u);
            if (j < full) {
                float x[kV];
                unpack<DT>(load16(row + (int64_t)j * 16), x);
                uint32_t r[kV];
                int mine = 0;
#pragma unroll
                for (int e = 0; e < kV; ++e) {
                    r[e] = rank_key<DT>(x[e]);
                    mine += r[e] >= from;
                }
                int at = atomicAdd(&L.n, mine);
#pragma unroll
                for (int e = 0; e < kV; ++e)
                    if (r[e] >= from) L.c[at++] = candidate(r[e], (uint32_t)j * kV + e);
            } else {
#pragma unroll 1
                for (int e = 0; e < rem; ++e) {
                    const uint32_t r = rank_key<DT>(load1<DT>(row, (int64_t)j * kV + e));
                    if (r >= from) push(L, r, (uint32_t)j * kV + e);
                }
            }
        }
        __syncthreads();
        if (L.n > kBlock) keep_best<DT, kCand, 1>(L, L.n, none, none, k, at_bits + 3);
    }
};

// Each of the L.n <= kRanked candidates' rank among them: how many are better,
// every wave counting among a quarter of them.  put(rank, key, index) for ranks < k.
template <typename F>
__device__ void by_rank(TopLds &L, int k, F put) {
    const int n = L.n, t = threadIdx.x;
    for (int i = t; i < n; i += kBlock) L.rank[i] = 0;
    if (t < 8) L.c[n + t] = 0;  // better than none
    __syncthreads();
    for (int i = lane_id(); i < n; i += kWave) {
        const uint64_t own = L.c[i];
        uint32_t better = 0;
        for (int q = wave_in_block() * 8; q < n; q += kWaves * 8)
#pragma unroll
            for (int e = 0; e < 8; ++e) better += L.c[q + e] > own;
        atomicAdd(&L.rank[i], better);
    }
    __syncthreads();
    for (int i = t; i < n; i += kBlock)
        if ((int)L.rank[i] < k) put((int)L.rank[i], key_of(L.c[i]), index_of(L.c[i]));
}

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

// ----------------------------------------------------------------------------
// log probabilities

struct LogprobArgs {
    const void *z;
    int64_t ldz, n, v;
    const void *tokens;
    int index, top, at_bits;
    float inv_t, c;  // 1 / T, log2(e) / T
    float *logp, *entropy, *stats;
    int32_t *top_id;
    float *top_logp;
    int32_t *status;
    int part_vecs;  // vectors of a part, a multiple of kBlock
    int parts;
    float *part_stat;    // [n][parts][3]
    uint32_t *part_top;  // [n][parts][top][2]
};

__device__ __forceinline__ void put_skipped(const LogprobArgs &p, int64_t i) {
    if (threadIdx.x == 0) {
        if (p.logp) p.logp[i] = 0.0f;
        if (p.entropy) p.entropy[i] = 0.0f;
        if (p.stats) p.stats[2 * i] = p.stats[2 * i + 1] = 0.0f;
    }
    for (int q = threadIdx.x; q < p.top; q += kBlock) {
        if (p.top_id) p.top_id[i * p.top + q] = -1;
        if (p.top_logp) p.top_logp[i * p.top + q] = kNegInf;
    }
}

// zt: the token's logit (thread 0 writes)
__device__ __forceinline__ void put_row_stat(const LogprobArgs &p, int64_t i, float zt,
                                             const Stat &t) {
    if (threadIdx.x != 0) return;
    const float ls = log_sum(t, p.c), m = t.s == 0.0f ? 0.0f : t.m;
    if (p.logp) p.logp[i] = log_prob(zt, m, ls, p.inv_t);
    if (p.entropy) p.entropy[i] = entropy_of(t);
    if (p.stats) {
        p.stats[2 * i] = m;
        p.stats[2 * i + 1] = ls;
    }
}

template <int DT>
__device__ __forceinline__ void put_top(const LogprobArgs &p, int64_t i, const Stat &t,
                                        TopLds &L) {
    const float ls = log_sum(t, p.c), m = t.s == 0.0f ? 0.0f : t.m;
    by_rank(L, p.top, [&](int r, uint32_t key, uint32_t at) {
        if (p.top_id) p.top_id[i * p.top + r] = (int32_t)at;
        if (p.top_logp) p.top_logp[i * p.top + r] = log_prob(logit_of<DT>(key), m, ls, p.inv_t);
    });
}

template <int DT, bool TOP>
__global__ __launch_bounds__(kBlock, 6) void k_logprobs(LogprobArgs p) {
    constexpr int kV = Elem<DT>::kVec;
    __shared__ typename std::conditional<TOP, TopLds, int>::type s_top;
    const int full = (int)(p.v / kV), rest = (int)(p.v % kV);
    for (int64_t w = blockIdx.x; w < p.n * p.parts; w += gridDim.x) {
        const auto [i, part] = Work(w, p.parts);
        const int32_t tok = p.tokens ? read_token(p.tokens, p.index, i, p.v, p.status) : 0;
        if (tok < 0) {
            if (p.parts == 1) put_skipped(p, i);
            continue;
        }
        const char *row = elem_at<DT>(p.z, i * p.ldz);
        const int first = part * p.part_vecs, end = min(full, first + p.part_vecs);
        const int rem = end == full ? rest : 0;  // the tail is the last part's
        // the token's logit is wanted at the end: asked for now
        const float zt = threadIdx.x == 0 && p.logp && p.parts == 1 ? load1<DT>(row, tok) : 0.0f;
        Stat t = {-FLT_MAX, 0.0f, 0.0f};
        Selection<DT> sel;
        int j = first + (int)threadIdx.x;
        Tile tile = load_tile<DT>(row, j, end);
        const float tail = tail_elem<DT>(row, full, rem);
        if (rem > 0) add_elem<true>(tail, p.c, t);
        if constexpr (TOP) sel.start(s_top, tail, full, rem);
        for (int turn = 0; j - (int)threadIdx.x < end; ++turn, j += kTileVecs * kBlock) {
            const Tile now = tile;
            const int next = j + kTileVecs * kBlock;
            if (next - (int)threadIdx.x < end) tile = load_tile<DT>(row, next, end);
            float lm[kTileVecs];
            add_tile<DT, true>(now, p.c, t, lm);
            if constexpr (TOP) sel.take(s_top, lm, turn, j, end, p.top, p.at_bits);
        }
        t = block_stat(t, p.c);
        if constexpr (TOP) {
            sel.finish(s_top, row, full, rem, p.top, p.at_bits);
            if (p.parts == 1) {
                put_top<DT>(p, i, t, s_top);
            } else {
                uint32_t *to = p.part_top + w * p.top * 2;
                for (int q = (int)threadIdx.x; q < p.top; q += kBlock)
                    if (q >= s_top.n) to[2 * q] = to[2 * q + 1] = 0;
                by_rank(s_top, p.top, [&](int r, uint32_t key, uint32_t at) {
                    to[2 * r] = key;
                    to[2 * r + 1] = at;
                });
            }
            __syncthreads();
        }
        if (p.parts == 1) put_row_stat(p, i, zt, t);
        if (p.parts > 1 && threadIdx.x == 0) {
            p.part_stat[3 * w] = t.m;
            p.part_stat[3 * w + 1] = t.s;
            p.part_stat[3 * w + 2] = t.a;
        }
    }
}

// a row's statistics from its parts', in part order, the same in every thread
__device__ __forceinline__ Stat join_parts(const float *part_stat, int64_t i, int parts, float c) {
    const float *q = part_stat + 3 * i * parts;
    Stat t = {q[0], q[1], q[2]};
    for (int k = 1; k < parts; ++k) t = join(t, Stat{q[3 * k], q[3 * k + 1], q[3 * k + 2]}, c);
    return t;
}

constexpr int kJoin = 2048;  // candidates that the parts of a row hand over, at most

template <int DT>
__global__ __launch_bounds__(kBlock) void k_logprobs_join(LogprobArgs p) {
    __shared__ TopLds s_top;
    for (int64_t i = blockIdx.x; i < p.n; i += gridDim.x) {
        const int32_t tok = p.tokens ? read_token(p.tokens, p.index, i, p.v, nullptr) : 0;
        if (tok < 0) {
            put_skipped(p, i);
            continue;
        }
        const Stat t = join_parts(p.part_stat, i, p.parts, p.c);
        put_row_stat(p, i, p.logp ? load1<DT>(elem_at<DT>(p.z, i * p.ldz), tok) : 0.0f, t);
        if (p.top == 0) continue;
        const uint32_t *from = p.part_top + i * p.parts * p.top * 2;
        const int count = p.parts * p.top;
        if (threadIdx.x == 0) s_top.n = 0;
        __syncthreads();
        if (count <= kRanked) {
            for (int k = threadIdx.x; k < count; k += kBlock)
                if (from[2 * k] > 0) push(s_top, from[2 * k], from[2 * k + 1]);
        } else {
            constexpr int kN = kJoin / kBlock;
            uint32_t key[kN], at[kN];
#pragma unroll
            for (int q = 0; q < kN; ++q) {
                const int k = q * kBlock + threadIdx.x;
                key[q] = k < count ? from[2 * k] : 0;
                at[q] = k < count ? from[2 * k + 1] : 0;
            }
            const Bound b = kth_best<DT, kN>(key, at, p.top, p.at_bits + 3);
#pragma unroll
            for (int q = 0; q < kN; ++q)
                if (key[q] > 0 && passes(b, key[q], at[q])) push(s_top, key[q], at[q]);
        }
        __syncthreads();
        put_top<DT>(p, i, t, s_top);
        __syncthreads();
    }
}

// ----------------------------------------------------------------------------
// gradient of log probabilities and entropies

struct LogprobGradArgs {
    const void *z;
    int64_t ldz, n, v;
    const void *tokens;
    int index;
    float inv_t;
    const float *stats, *entropy, *d_logp, *d_entropy;
    void *dz;
    int64_t ldd;
    int32_t *status;
    int part_vecs;
    int parts;
};

// the vectors [first, end) of a row: f(j, x) replaces the elements of vector j
template <int DT, typename F>
__device__ __forceinline__ void map_row(const char *row, char *out, int first, int end, F f) {
    constexpr int kV = Elem<DT>::kVec;
    for (int j = first + (int)threadIdx.x; j - (int)threadIdx.x < end; j += kTileVecs * kBlock) {
        const Tile tile = load_tile<DT>(row, j, end);
#pragma unroll
        for (int u = 0; u < kTileVecs; ++u) {
            const int q = j + u * kBlock;
            if (q >= end) break;
            float x[kV];
            unpack<DT>(tile.r[u], x);
            f(q, x);
            store16(out + (int64_t)q * 16, pack<DT>(x));
        }
    }
}
template <int DT>
__device__ __forceinline__ void zero_row(char *out, int first, int end, int full, int rem) {
    constexpr int kV = Elem<DT>::kVec;
    for (int j = first + (int)threadIdx.x; j < end; j += kBlock)
        store16(out + (int64_t)j * 16, u32x4{0, 0, 0, 0});
    if ((int)threadIdx.x < rem) store1<DT>(out, (int64_t)full * kV + threadIdx.x, 0.0f);
}

template <int DT>
__global__ __launch_bounds__(kBlock) void k_logprobs_grad(LogprobGradArgs p) {
    constexpr int kV = Elem<DT>::kVec;
    const int full = (int)(p.v / kV), rest = (int)(p.v % kV);
    for (int64_t w = blockIdx.x; w < p.n * p.parts; w += gridDim.x) {
        const auto [i, part] = Work(w, p.parts);
        const int first = part * p.part_vecs, end = min(full, first + p.part_vecs);
        const int rem = end == full ? rest : 0;  // the tail is the last part's
        const int32_t tok = p.tokens ? read_token(p.tokens, p.index, i, p.v, p.status) : 0;
        const char *row = elem_at<DT>(p.z, i * p.ldz);
        char *out = elem_at<DT>(p.dz, i * p.ldd);
        const float m = p.stats[2 * i], ls = p.stats[2 * i + 1];
        if (tok < 0 || ls == kNegInf) {
            zero_row<DT>(out, first, end, full, rem);
            continue;
        }
        // dz = q (a + b log q), and d_logp / T more at the token
        const float g = p.d_logp ? p.d_logp[i] * p.inv_t : 0.0f;
        const float b = p.d_entropy ? -p.d_entropy[i] * p.inv_t : 0.0f;
        const float a = p.d_entropy ? __builtin_fmaf(b, p.entropy[i], -g) : -g;
        auto gradient = [&](float z) {
            const float lq = (z - m) * p.inv_t - ls;
            // q by its root twice: the product reaches the subnormals, which the
            // instruction's own results do not.  Where q is 0 so is the product,
            // whatever log q
            const float r = exp2_raw(lq * (0.5f * kLog2e));
            return r * (r * __builtin_fmaf(b, fmaxf(lq, kLogFloor), a));
        };
        const float tail = tail_elem<DT>(row, full, rem);
        map_row<DT>(row, out, first, end, [&](int j, float *x) {
#pragma unroll
            for (int e = 0; e < kV; ++e) x[e] = gradient(x[e]);
            const int hot = tok - j * kV;
            if (hot >= 0 && hot < kV && p.d_logp) {
#pragma unroll
                for (int e = 0; e < kV; ++e)
                    if (e == hot) x[e] += g;
            }
        });
        if ((int)threadIdx.x < rem) {
            const int at = full * kV + (int)threadIdx.x;
            store1<DT>(out, at, gradient(tail) + (at == tok && p.d_logp ? g : 0.0f));
        }
    }
}

// ----------------------------------------------------------------------------
// distillation

struct DistillArgs {
    const void *z;
    int64_t ldz, n, v;
    const int32_t *ids;
    const void *teacher;
    int teacher_dtype, k;
    float inv_t, c;
    const float *weight;
    float *loss;
    void *dz;
    int64_t ldd;
    int32_t *status;
    int part_vecs;
    int parts;         // of the gradient's blocks, or of the statistics'
    int stat_parts;
    float *part_stat;  // [n][stat_parts][3]
};

__device__ __forceinline__ float row_weight(const DistillArgs &p, int64_t i) {
    return p.weight ? p.weight[i] : 1.0f;
}

template <int DT>
__global__ __launch_bounds__(kBlock) void k_distill_stat(DistillArgs p) {
    constexpr int kV = Elem<DT>::kVec;
    const int full = (int)(p.v / kV), rest = (int)(p.v % kV);
    for (int64_t w = blockIdx.x; w < p.n * p.parts; w += gridDim.x) {
        const auto [i, part] = Work(w, p.parts);
        const int first = part * p.part_vecs, end = min(full, first + p.part_vecs);
        const int rem = end == full ? rest : 0;  // the tail is the last part's
        if (row_weight(p, i) == 0.0f) continue;
        const char *row = elem_at<DT>(p.z, i * p.ldz);
        Stat t = {-FLT_MAX, 0.0f, 0.0f};
        for (int j = first + (int)threadIdx.x; j - (int)threadIdx.x < end; j += kTileVecs * kBlock) {
            float lm[kTileVecs];
            add_tile<DT, false>(load_tile<DT>(row, j, end), p.c, t, lm);
        }
        if (rem > 0) add_elem<false>(tail_elem<DT>(row, full, rem), p.c, t);
        t = block_stat(t, p.c);
        if (threadIdx.x == 0) {
            p.part_stat[3 * w] = t.m;
            p.part_stat[3 * w + 1] = t.s;
            p.part_stat[3 * w + 2] = 0.0f;
        }
    }
}

struct TeacherLds {
    int32_t id[PDB_MAX_TEACHER];
    float p[PDB_MAX_TEACHER];  // the teacher's probability
    float z[PDB_MAX_TEACHER];  // the student's logit
};

__device__ __forceinline__ float load_teacher(const DistillArgs &p, int64_t at) {
    if (p.teacher_dtype == PDB_F32) return load1<PDB_F32>(p.teacher, at);
    return p.teacher_dtype == PDB_BF16 ? load1<PDB_BF16>(p.teacher, at)
                                       : load1<PDB_F16>(p.teacher, at);
}

// The teacher's distribution over its entries into LDS; false if it has none.
template <int DT>
__device__ bool teacher_row(const DistillArgs &p, int64_t i, const char *row, TeacherLds &L) {
    Stat t = {-FLT_MAX, 0.0f, 0.0f};
    float top = kNegInf;
    for (int j = threadIdx.x; j < p.k; j += kBlock) {
        int32_t id = p.ids[i * p.k + j];
        if (id >= p.v) {
            if (p.status) *p.status = PDB_ERR_INVALID_ARG;
            id = -1;
        }
        const float y = id < 0 ? kNegInf : load_teacher(p, i * p.k + j);
        L.id[j] = id < 0 ? -1 : id;
        L.p[j] = y;
        L.z[j] = id < 0 ? 0.0f : load1<DT>(row, id);
        top = fmaxf(top, y);
    }
    t.m = fmaxf(t.m, wave_max_f32(top));
    for (int j = threadIdx.x; j < p.k; j += kBlock) t.s += exp2_of(L.p[j], t.m, p.c);
    t = block_stat(t, p.c);
    if (t.s == 0.0f) return false;
    const float ls = log_sum(t, p.c);
    for (int j = threadIdx.x; j < p.k; j += kBlock) {
        // log p for the loss is formed again from p's own logit
        const float lp = (L.p[j] - t.m) * p.inv_t - ls;
        L.p[j] = lp;
    }
    __syncthreads();
    return true;
}

template <int DT, bool GRAD>
__global__ __launch_bounds__(kBlock) void k_distill(DistillArgs p) {
    constexpr int kV = Elem<DT>::kVec;
    __shared__ TeacherLds L;
    const int full = (int)(p.v / kV), rest = (int)(p.v % kV);
    for (int64_t w = blockIdx.x; w < p.n * p.parts; w += gridDim.x) {
        const auto [i, part] = Work(w, p.parts);
        const int first = part * p.part_vecs, end = min(full, first + p.part_vecs);
        const int rem = end == full ? rest : 0;  // the tail is the last part's
        const char *row = elem_at<DT>(p.z, i * p.ldz);
        char *out = elem_at<DT>(p.dz, i * p.ldd);
        const float wt = row_weight(p, i);
        __syncthreads();  // the row before is done with L
        if (wt == 0.0f || !teacher_row<DT>(p, i, row, L)) {
            if (part == 0 && threadIdx.x == 0 && p.loss) p.loss[i] = 0.0f;
            if (GRAD) zero_row<DT>(out, first, end, full, rem);
            continue;
        }
        const Stat t = join_parts(p.part_stat, i, p.stat_parts, p.c);
        const float ls = log_sum(t, p.c), m = t.s == 0.0f ? 0.0f : t.m;
        if (part == 0 && p.loss) {
            float sum = 0.0f;
            for (int j = threadIdx.x; j < p.k; j += kBlock) {
                const float lp = L.p[j], q = exp2_raw(lp * kLog2e);
                if (q != 0.0f) sum = __builtin_fmaf(q, lp - log_prob(L.z[j], m, ls, p.inv_t), sum);
            }
            const Stat all_s = block_stat(Stat{0.0f, sum, 0.0f}, p.c);
            if (threadIdx.x == 0) p.loss[i] = wt * all_s.s;
        }
        if constexpr (GRAD) {
            const float g = wt * p.inv_t;
            const float off = ls == kNegInf ? 0.0f : ls;
            // g q, q by its root twice: the product reaches the subnormals, which the
            // instruction's own results do not
            auto times_q = [&](float g, float z) {
                const float r = exp2_raw(((z - m) * p.inv_t - off) * (0.5f * kLog2e));
                return r * (r * g);
            };
            const float tail = tail_elem<DT>(row, full, rem);
            map_row<DT>(row, out, first, end, [&](int, float *x) {
#pragma unroll
                for (int e = 0; e < kV; ++e) x[e] = times_q(g, x[e]);
            });
            if ((int)threadIdx.x < rem) store1<DT>(out, full * kV + (int)threadIdx.x, times_q(g, tail));
            // the teacher's entries in this part: once per id, with the sum of
            // its probabilities; after the block's own stores to those places
            __syncthreads();
            for (int j = threadIdx.x; j < p.k; j += kBlock) {
                const int32_t id = L.id[j];
                // (the tail's vector, `full`, is the last part's)
                if (id < 0 || id / kV < first || id / kV >= (rem > 0 ? full + 1 : end)) continue;
                float sum = 0.0f;
                bool seen = false;
                for (int q = 0; q < p.k; ++q)
                    if (L.id[q] == id) {
                        seen |= q < j;
                        sum += exp2_raw(L.p[q] * kLog2e);
                    }
                if (!seen) store1<DT>(out, id, g * (times_q(1.0f, L.z[j]) - sum));
            }
        }
    }
}

// ----------------------------------------------------------------------------
// how rows are cut into parts

// Up to kWantBlocks blocks when there are few rows (four a compute unit), none
// with less than a tile.
constexpr int64_t kWantBlocks = 1024;
struct Parts {
    int parts;
    int vecs;  // of a part
};
Parts cut_rows(int64_t n, int64_t v, int64_t vec, int64_t most) {
    const int64_t all = std::max<int64_t>(v / vec, 1), tile = (int64_t)kBlock * kTileVecs;
    int64_t parts = std::min(std::min(kWantBlocks / std::max<int64_t>(n, 1), cdiv(all, tile)), most);
    parts = std::max<int64_t>(parts, 1);
    const int64_t vecs = cdiv(cdiv(all, parts), kBlock) * kBlock;
    return {(int)cdiv(all, vecs), (int)vecs};
}
constexpr int64_t kMostParts = 64;

bool good_temp(float t) { return t > 0.0f && t <= FLT_MAX && kLog2e / t <= FLT_MAX; }

}  // namespace
}  // namespace pdbk

using namespace pdbk;

namespace {
int64_t most_parts(int32_t top) { return top > 0 ? std::min<int64_t>(kMostParts, kJoin / top) : kMostParts; }
size_t stat_bytes(int64_t n) { return (size_t)align_up(n * kMostParts * 12); }
unsigned blocks_for(int64_t work) { return (unsigned)std::min<int64_t>(work, 1 << 22); }
}  // namespace

extern "C" int pdb_token_logprobs_workspace_bytes(int64_t n, int64_t v, int32_t top,
                                                  size_t *bytes) {
    if (!bytes || n < 0 || v < 0 || top < 0) return PDB_ERR_INVALID_ARG;
    if (n > INT32_MAX || v > INT32_MAX || top > PDB_MAX_TOP) return PDB_ERR_UNSUPPORTED;
    // rows are cut only where they are few
    const int64_t rows = std::min(n, kWantBlocks);
    *bytes = stat_bytes(rows) + (size_t)(rows * most_parts(top) * top * 8);
    return PDB_OK;
}

extern "C" int pdb_token_logprobs(const void *logits, int dtype, int64_t ldz, int64_t n, int64_t v,
                                  const void *tokens, int index, float temp, float *logp,
                                  float *entropy, float *stats, int32_t top, int32_t *top_id,
                                  float *top_logp, int32_t *status, void *ws, size_t ws_bytes,
                                  hipStream_t s) {
    int rc = check_matrix(logits, dtype, ldz, n, v);
    if (rc == PDB_OK && (tokens || logp)) rc = check_tokens(tokens, index, n);
    if (rc != PDB_OK) return rc;
    if (top < 0 || !good_temp(temp) || top > v) return PDB_ERR_INVALID_ARG;
    if (top > PDB_MAX_TOP) return PDB_ERR_UNSUPPORTED;
    if (n > 0 && v == 0) return PDB_ERR_INVALID_ARG;
    if (n == 0) return PDB_OK;
    if (!top_id && !top_logp) top = 0;
    size_t need = 0;
    rc = pdb_token_logprobs_workspace_bytes(n, v, top, &need);
    if (rc != PDB_OK) return rc;
    if (!ws || ws_bytes < need) return PDB_ERR_WORKSPACE;
    return with_dtype(dtype, [&](auto dt) -> int {
        constexpr int DT = decltype(dt)::value;
        const Parts cut = cut_rows(n, v, Elem<DT>::kVec, most_parts(top));
        LogprobArgs p = {logits, ldz, n, v, tokens, index, top,
                         bits_for(cdiv(v, Elem<DT>::kVec)), 1.0f / temp, kLog2e / temp, logp,
                         entropy, stats, top_id, top_logp, status, cut.vecs, cut.parts,
                         static_cast<float *>(ws),
                         reinterpret_cast<uint32_t *>(static_cast<char *>(ws) +
                                                      stat_bytes(std::min(n, kWantBlocks)))};
        if (top > 0)
            k_logprobs<DT, true><<<blocks_for(n * cut.parts), kBlock, 0, s>>>(p);
        else
            k_logprobs<DT, false><<<blocks_for(n * cut.parts), kBlock, 0, s>>>(p);
        PDB_LAUNCHED();
        if (cut.parts > 1) {
            k_logprobs_join<DT><<<blocks_for(n), kBlock, 0, s>>>(p);
            PDB_LAUNCHED();
        }
        return PDB_OK;
    });
}

extern "C" int pdb_token_logprobs_grad(const void *logits, int dtype, int64_t ldz, int64_t n,
                                       int64_t v, const void *tokens, int index, float temp,
                                       const float *stats, const float *entropy,
                                       const float *d_logp, const float *d_entropy, void *dlogits,
                                       int64_t ldd, int32_t *status, hipStream_t s) {
    int rc = check_matrix(logits, dtype, ldz, n, v);
    if (rc == PDB_OK) rc = check_matrix(dlogits, dtype, ldd, n, v);
    if (rc == PDB_OK && dlogits == logits && n > 1 && ldd != ldz) rc = PDB_ERR_INVALID_ARG;
    if (rc == PDB_OK && (tokens || d_logp)) rc = check_tokens(tokens, index, n);
    if (rc != PDB_OK) return rc;
    if (!good_temp(temp)) return PDB_ERR_INVALID_ARG;
    if (n == 0 || v == 0) return PDB_OK;
    if (!stats || (d_entropy && !entropy)) return PDB_ERR_INVALID_ARG;
    return with_dtype(dtype, [&](auto dt) -> int {
        constexpr int DT = decltype(dt)::value;
        const Parts cut = cut_rows(n, v, Elem<DT>::kVec, kMostParts);
        LogprobGradArgs p = {logits, ldz, n, v, tokens, index, 1.0f / temp, stats, entropy, d_logp,
                             d_entropy, dlogits, ldd, status, cut.vecs, cut.parts};
        k_logprobs_grad<DT><<<blocks_for(n * cut.parts), kBlock, 0, s>>>(p);
        PDB_LAUNCHED();
        return PDB_OK;
    });
}

extern "C" int pdb_distill_workspace_bytes(int64_t n, int64_t v, size_t *bytes) {
    if (!bytes || n < 0 || v < 0) return PDB_ERR_INVALID_ARG;
    if (n > INT32_MAX || v > INT32_MAX) return PDB_ERR_UNSUPPORTED;
    *bytes = std::max(stat_bytes(std::min(n, kWantBlocks)), (size_t)align_up(n * 12));
    return PDB_OK;
}

extern "C" int pdb_distill(const void *logits, int dtype, int64_t ldz, int64_t n, int64_t v,
                           const int32_t *ids, const void *teacher, int teacher_dtype, int32_t k,
                           float temp, const float *weight, float *loss, void *dlogits, int64_t ldd,
                           int32_t *status, void *ws, size_t ws_bytes, hipStream_t s) {
    int rc = check_matrix(logits, dtype, ldz, n, v);
    if (rc == PDB_OK && dlogits) rc = check_matrix(dlogits, dtype, ldd, n, v);
    if (rc == PDB_OK && dlogits == logits && n > 1 && ldd != ldz) rc = PDB_ERR_INVALID_ARG;
    if (rc == PDB_OK) rc = check_tokens(ids, PDB_I32, n);
    if (rc == PDB_OK) rc = check_matrix(teacher, teacher_dtype, k, n, k);
    if (rc != PDB_OK) return rc;
    if (k < 1 || !good_temp(temp) || (n > 0 && v == 0)) return PDB_ERR_INVALID_ARG;
    if (k > PDB_MAX_TEACHER || n * k > INT32_MAX) return PDB_ERR_UNSUPPORTED;
    if (n == 0) return PDB_OK;
    if (!loss) return PDB_ERR_INVALID_ARG;
    size_t need = 0;
    rc = pdb_distill_workspace_bytes(n, v, &need);
    if (rc != PDB_OK) return rc;
    if (!ws || ws_bytes < need) return PDB_ERR_WORKSPACE;
    return with_dtype(dtype, [&](auto dt) -> int {
        constexpr int DT = decltype(dt)::value;
        const Parts cut = cut_rows(n, v, Elem<DT>::kVec, kMostParts);
        DistillArgs p = {logits, ldz, n, v, ids, teacher, teacher_dtype, k, 1.0f / temp,
                         kLog2e / temp, weight, loss, dlogits, ldd, status, cut.vecs, cut.parts,
                         cut.parts, static_cast<float *>(ws)};
        k_distill_stat<DT><<<blocks_for(n * cut.parts), kBlock, 0, s>>>(p);
        PDB_LAUNCHED();
        // the loss reads the logits of every id: in place, before any part of a
        // row is overwritten
        if (!dlogits || (dlogits == logits && cut.parts > 1)) {
            p.parts = 1;
            k_distill<DT, false><<<blocks_for(n), kBlock, 0, s>>>(p);
            PDB_LAUNCHED();
            p.loss = nullptr;
        }
        if (dlogits) {
            p.parts = cut.parts;
            k_distill<DT, true><<<blocks_for(n * cut.parts), kBlock, 0, s>>>(p);
            PDB_LAUNCHED();
        }
        return PDB_OK;
    });
}
