// Log probabilities over a vocabulary (gfx950, wave64): of given tokens, with the
// entropy and the best alternatives of every row, and their gradient.
//
// Both read the logits once (the gradient writes as many): their floor is those
// bytes at the rate memory gives.  A row is one block's, a wave's where rows are many
// or short, or with few rows several blocks', joined by a second kernel.
#include <type_traits>

#include "pdb_softmax.h"

namespace pdbk {
namespace {

// ----------------------------------------------------------------------------
// the K best of a row, ties to the lowest index
//
// A logit's rank key orders like the logit, in as many bits as its type has;
// 1 is NaN, 0 nothing.  The row's K best lie in the K best of its vectors, ordered
// by (largest key, index): an element of any other has K better ones.  So while a
// row streams by, only its vectors' maxima are looked at: those better than a bound
// are kept in LDS, by each wave in a place of its own, so that the waves of a team
// wait for each other at a row's ends only (of 1,000 rows of 100,003 in 32 bits with 64
// alternatives, 89 us, a barrier every tile took 7 more).  The bound is the K-th best of
// K or more vectors met so far.  The first tile sets it, from the K-th best of a wave's
// vectors, or from the (K / W)-th best of each of W waves'; when a wave's
// kept ones would overflow, its bound is raised to the K-th best of those kept and the
// tile's, which leaves K, whatever the data.  Of the vectors kept in the end the K best
// are read again, and their elements and the row's tail put in order.  The K-th best of
// a set is found by a binary search over the bits of its key, counting with ballots.

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
// max of unsigned words over the wave (wave_max_dpp's are signed)
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
    return (uint32_t)wave_max_dpp((int)(v ^ 0x80000000u)) ^ 0x80000000u;
}

// the team's sum of its waves' counts
template <int W>
__device__ __forceinline__ int team_count(int wave_count, int &turn) {
    if constexpr (W == 1) {
        return wave_count;
    } else {
        __shared__ int s_count[2][W];
        if (lane_id() == 0) s_count[turn][wave_in_block()] = wave_count;
        __syncthreads();
        int all = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) all += s_count[turn][w];
        turn ^= 1;
        return all;
    }
}

struct Bound {  // an element passes when its key is larger, or equal at an index <= at
    uint32_t key, at;
};
__device__ __forceinline__ bool passes(const Bound &b, uint32_t key, uint32_t at) {
    return key > b.key || (key == b.key && at <= b.at);
}

// The bound that exactly the k best of the team's N (key, index) a thread pass, or
// every valid one (key > 0) if those are fewer.  Indices < 2^at_bits.
template <int DT, int W, int N>
__device__ __forceinline__ Bound kth_best(const uint32_t (&key)[N], const uint32_t (&at)[N], int k,
                                          int at_bits) {
    int turn = 0;
    uint32_t t = 0;
    int enough = 0;  // how many are >= t, once t > 0
#pragma unroll 1
    for (int b = Key<DT>::kBits - 1; b >= 0; --b) {
        const uint32_t cand = t | (1u << b);
        int w = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) w += __popcll(__ballot(key[i] >= cand));
        const int all = team_count<W>(w, turn);
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
    const int need = k - team_count<W>(w, turn);
    uint32_t x = at_bits >= 32 ? 0xFFFFFFFFu : (1u << at_bits) - 1u;
#pragma unroll 1
    for (int b = at_bits - 1; b >= 0; --b) {
        const uint32_t cand = x & ~(1u << b);
        w = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) w += __popcll(__ballot(key[i] == t && at[i] <= cand));
        if (team_count<W>(w, turn) >= need) x = cand;
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

// Room of a team's selection: vectors that each wave keeps while a row streams by,
// elements of the K vectors in the end (8 K, and a tail's 7), candidates that are
// ranked against each other.
template <int W>
struct TopLds {
    static constexpr int kTop = W == 1 ? PDB_MAX_TOP / 2 : PDB_MAX_TOP;  // largest K
    static constexpr int kKeep = 256;                                    // a wave's
    static constexpr int kCand = kTop * 8;
    static constexpr int kRanked = 512;
    static_assert(kCand >= W * kKeep && kCand >= kRanked && kKeep >= kTop, "c holds each");
    alignas(16) uint64_t c[kCand + 8];
    uint32_t rank[kRanked];
    int n;
    int held[W];                // vectors that each wave has kept
    uint32_t first[W], last[W];  // each wave's bound, of its first tile and in the end
};

template <int W>
__device__ __forceinline__ void push(TopLds<W> &L, uint32_t key, uint32_t at) {
    L.c[atomicAdd(&L.n, 1)] = candidate(key, at);
}

inline int bits_for(int64_t count) {
    int b = 0;
    while (b < 31 && ((int64_t)1 << b) < count) ++b;
    return b;
}

// The k best of the first n <= M candidates in c and of the given ones stay in c,
// `count` of them; returns the bound.  Every thread of the team calls.
template <int DT, int W, int M, int N>
__device__ __forceinline__ Bound keep_best(uint64_t *c, int &count, int n,
                                           const uint32_t (&more)[N],
                                           const uint32_t (&more_at)[N], int k, int at_bits) {
    constexpr int kT = Team<W>::kThreads, kN = M / kT;
    static_assert(M % kT == 0, "whole rounds");
    const int t = Team<W>::thread();
    uint32_t key[kN + N], at[kN + N];
    Team<W>::sync();
#pragma unroll
    for (int i = 0; i < kN; ++i) {
        const int q = i * kT + t;
        key[i] = q < n ? key_of(c[q]) : 0;
        at[i] = q < n ? index_of(c[q]) : 0;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        key[kN + i] = more[i];
        at[kN + i] = more_at[i];
    }
    if (t == 0) count = 0;
    const Bound b = kth_best<DT, W, kN + N>(key, at, k, at_bits);
    Team<W>::sync();
#pragma unroll
    for (int i = 0; i < kN + N; ++i)
        if (key[i] > 0 && passes(b, key[i], at[i]))
            c[atomicAdd(&count, 1)] = candidate(key[i], at[i]);
    Team<W>::sync();
    return b;
}

// The selection over a row part, tile by tile.
template <int DT, int W>
struct Selection {
    using Lds = TopLds<W>;
    static constexpr int kV = Elem<DT>::kVec;
    static constexpr int kT = Team<W>::kThreads;
    // the wave's
    uint32_t bound;  // its key
    float least;     // its logit: what is not larger is not kept; NaN: everything is
    int n;           // vectors kept

    static __device__ __forceinline__ uint64_t *kept(Lds &L) {
        return L.c + Team<W>::wave() * Lds::kKeep;
    }

    __device__ __forceinline__ void start() {
        bound = 0;
        least = kNan;
        n = 0;
    }

    // The largest logit under a key: where the bound comes from this very tile,
    // equal ones count too (in later tiles they stand behind it).  0's is two keys
    // down: the one between is -0's, which equals 0.
    static __device__ __forceinline__ float below(uint32_t key) {
        const uint32_t step = key == (0x80000000u >> Key<DT>::kShift) ? 2 : 1;
        return key > 2 ? logit_of<DT>(key - step) : kNan;
    }

    // The K-th best of the wave's lanes (kReps = 1, for K that are few of them), or
    // of their vectors.
    template <int kReps>
    static __device__ __forceinline__ uint32_t wave_bound(const uint32_t (&key)[kReps], int k) {
        uint32_t hi = key[0], lo = key[0];
#pragma unroll
        for (int u = 1; u < kReps; ++u) {
            hi = max(hi, key[u]);
            lo = min(lo, key[u]);
        }
        // the bits above the highest in which two of them differ are everyone's
        hi = wave_max_u32(hi);
        lo = ~wave_max_u32(~lo);
        const int bits = hi == lo ? 0 : 32 - __builtin_clz(hi ^ lo);
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

    __device__ __forceinline__ void first_bound(Lds &L, const float (&lm)[kTileVecs], int j,
                                                int end, int k) {
        uint32_t key[kTileVecs];
#pragma unroll
        for (int u = 0; u < kTileVecs; ++u) key[u] = j + u * kT < end ? rank_key<DT>(lm[u]) : 0;
        const int share = (k + W - 1) / W;
        if (share <= kWave / 2) {
            const uint32_t own[1] = {max(max(key[0], key[1]), max(key[2], key[3]))};
            static_assert(kTileVecs == 4, "four vectors");
            bound = wave_bound(own, share);
        } else {
            bound = wave_bound(key, share);
        }
        if constexpr (W > 1) {
            // every wave has `share` no worse than its own: the waves of which k / share
            // have no lesser bound than one have k no worse than that one
            if (lane_id() == 0) L.first[wave_in_block()] = bound;
            __syncthreads();
            const int waves = (k + share - 1) / share;
            uint32_t all[W];
#pragma unroll
            for (int w = 0; w < W; ++w) all[w] = L.first[w];
            bound = 0;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                int as_good = 0;
#pragma unroll
                for (int q = 0; q < W; ++q) as_good += all[q] >= all[w];
                if (as_good >= waves) bound = max(bound, all[w]);
            }
        }
        least = below(bound);
    }

    // Takes the tile (the turn-th of the part) at this thread's vector j, lm its
    // vectors' maxima.
    __device__ __forceinline__ void take(Lds &L, const float (&lm)[kTileVecs], int turn, int j,
                                         int end, int k, int at_bits) {
        if (turn == 0) first_bound(L, lm, j, end, k);
        uint64_t hot[kTileVecs];
        int mine = 0;  // the wave's
#pragma unroll
        for (int u = 0; u < kTileVecs; ++u) {
            hot[u] = __ballot(!(lm[u] <= least) && j + u * kT < end);
            mine += __popcll(hot[u]);
        }
        int at = n;
        const int all = n + mine;
        if (all <= Lds::kKeep) {
            if (mine) {
#pragma unroll
                for (int u = 0; u < kTileVecs; ++u) {
                    if (hot[u] >> lane_id() & 1)
                        kept(L)[at + lanes_below(hot[u])] =
                            candidate(rank_key<DT>(lm[u]), (uint32_t)(j + u * kT));
                    at += __popcll(hot[u]);
                }
            }
            n = all;
            // of the first tile, equal ones were kept: later they are not wanted
            if (turn == 0) least = logit_of<DT>(bound);
        } else {
            uint32_t key[kTileVecs], where[kTileVecs];
#pragma unroll
            for (int u = 0; u < kTileVecs; ++u) {
                where[u] = (uint32_t)(j + u * kT);
                key[u] = j + u * kT < end ? rank_key<DT>(lm[u]) : 0;
            }
            int &held = L.held[Team<W>::wave()];
            bound = keep_best<DT, 1, Lds::kKeep>(kept(L), held, n, key, where, k, at_bits).key;
            n = held;
            least = logit_of<DT>(bound);
        }
    }

    // The vectors that the waves have kept and that pass the best of their bounds, in
    // the first places of L, as many as have room; every wave's n and bound are the
    // team's then.
    __device__ __forceinline__ void gather(Lds &L, int k, int at_bits) {
        static_assert(W == 1 || Lds::kKeep == kT, "a wave's vectors, one a thread");
        if (lane_id() == 0) {
            L.held[Team<W>::wave()] = n;
            L.last[Team<W>::wave()] = bound;
        }
        const int t = threadIdx.x;
        if (t == 0) L.n = 0;
        __syncthreads();
        uint32_t key[W], at[W];
#pragma unroll
        for (int w = 0; w < W; ++w) bound = max(bound, L.last[w]);
        int mine = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const uint64_t c = L.c[w * Lds::kKeep + t];
            key[w] = t < L.held[w] && key_of(c) >= bound ? key_of(c) : 0;
            at[w] = index_of(c);
            mine += __popcll(__ballot(key[w] > 0));
        }
        if (lane_id() == 0) atomicAdd(&L.n, mine);
        __syncthreads();
        n = L.n;
        Bound b = {0, 0};
        if (n > Lds::kTop) b = kth_best<DT, W, W>(key, at, k, at_bits);
        bound = max(bound, b.key);
        __syncthreads();
        if (t == 0) L.n = 0;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < W; ++w)
            if (key[w] > 0 && passes(b, key[w], at[w])) push(L, key[w], at[w]);
        __syncthreads();
        n = L.n;
    }

    // L holds the elements of the vectors left that may be the part's k best, few
    // enough to be ranked.  The row's tail, whose elements stand behind all others,
    // comes in here: in a bound it would shut out equal ones before it.
    __device__ __forceinline__ void finish(Lds &L, const char *row, int full, int rem, int k,
                                           int at_bits) {
        const uint32_t none[1] = {0};
        const float tail = tail_elem<DT, W>(row, full, rem);  // asked for now
        if constexpr (W == 1) {
            Team<W>::sync();
            if (n > Lds::kTop) {
                bound = keep_best<DT, W, Lds::kKeep>(L.c, L.n, n, none, none, k, at_bits).key;
                n = L.n;
            }
        } else {
            gather(L, k, at_bits);
        }
        constexpr int kHas = (Lds::kTop + kT - 1) / kT;
        static_assert(kHas == 1, "a vector a thread");
        const int t = Team<W>::thread();
        const int j = t < n ? (int)index_of(L.c[t]) : 0;
        Team<W>::sync();
        if (t == 0) L.n = 0;
        Team<W>::sync();
        const uint32_t from = max(bound, 1u);
        if (t < n) {
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
        }
        if (t < rem) {
            const uint32_t r = rank_key<DT>(tail);
            if (r >= from) push(L, r, (uint32_t)full * kV + t);
        }
        Team<W>::sync();
        if (L.n > Lds::kRanked)
            keep_best<DT, W, Lds::kCand + kT>(L.c, L.n, L.n, none, none, k, at_bits + 3);
    }
};

// Each of the L.n <= kRanked candidates' rank among them: how many are better,
// every wave counting among its share of them.  put(rank, key, index) for ranks < k.
template <int W, typename F>
__device__ __forceinline__ void by_rank(TopLds<W> &L, int k, F put) {
    constexpr int kT = Team<W>::kThreads;
    const int n = L.n, t = Team<W>::thread();
    for (int i = t; i < n; i += kT) L.rank[i] = 0;
    if (t < 8) L.c[n + t] = 0;  // better than none
    Team<W>::sync();
    for (int i = lane_id(); i < n; i += kWave) {
        const uint64_t own = L.c[i];
        uint32_t better = 0;
        for (int q = Team<W>::wave() * 8; q < n; q += W * 8)
#pragma unroll
            for (int e = 0; e < 8; ++e) better += L.c[q + e] > own;
        if constexpr (W == 1)
            L.rank[i] = better;
        else
            atomicAdd(&L.rank[i], better);
    }
    Team<W>::sync();
    for (int i = t; i < n; i += kT)
        if ((int)L.rank[i] < k) put((int)L.rank[i], key_of(L.c[i]), index_of(L.c[i]));
}

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

template <int W>
__device__ __forceinline__ void put_skipped(const LogprobArgs &p, int64_t i) {
    const int t = Team<W>::thread();
    if (t == 0) {
        if (p.logp) p.logp[i] = 0.0f;
        if (p.entropy) p.entropy[i] = 0.0f;
        if (p.stats) p.stats[2 * i] = p.stats[2 * i + 1] = 0.0f;
    }
    for (int q = t; q < p.top; q += Team<W>::kThreads) {
        if (p.top_id) p.top_id[i * p.top + q] = -1;
        if (p.top_logp) p.top_logp[i * p.top + q] = kNegInf;
    }
}

// zt: the token's logit (one thread writes)
__device__ __forceinline__ void put_row_stat(const LogprobArgs &p, int64_t i, float zt,
                                             const Stat &t) {
    const float ls = log_sum(t, p.c), m = t.s == 0.0f ? 0.0f : t.m;
    if (p.logp) p.logp[i] = log_prob(zt, m, ls, p.inv_t);
    if (p.entropy) p.entropy[i] = entropy_of(t);
    if (p.stats) {
        p.stats[2 * i] = m;
        p.stats[2 * i + 1] = ls;
    }
}

template <int DT, int W>
__device__ __forceinline__ void put_top(const LogprobArgs &p, int64_t i, const Stat &t,
                                        TopLds<W> &L) {
    const float ls = log_sum(t, p.c), m = t.s == 0.0f ? 0.0f : t.m;
    by_rank(L, p.top, [&](int r, uint32_t key, uint32_t at) {
        if (p.top_id) p.top_id[i * p.top + r] = (int32_t)at;
        if (p.top_logp) p.top_logp[i * p.top + r] = log_prob(logit_of<DT>(key), m, ls, p.inv_t);
    });
}

// Six waves a SIMD (80 registers) hide the loads; eight would spill.
template <int DT, int W, bool TOP>
__global__ __launch_bounds__(kBlock, 6) void k_logprobs(LogprobArgs p) {
    constexpr int kV = Elem<DT>::kVec, kT = Team<W>::kThreads, kStep = kTileVecs * kT;
    using Lds = typename std::conditional<TOP, TopLds<W>, int>::type;
    __shared__ Lds s_top[Team<W>::kPerBlock];
    Lds &top = s_top[Team<W>::here()];
    const int thread = Team<W>::thread();
    const int full = (int)(p.v / kV), rest = (int)(p.v % kV);
    for (int64_t w = (int64_t)blockIdx.x * Team<W>::kPerBlock + Team<W>::here();
         w < p.n * p.parts; w += (int64_t)gridDim.x * Team<W>::kPerBlock) {
        const auto [i, part] = Work(w, p.parts);
        const int32_t tok = p.tokens ? read_token(p.tokens, p.index, i, p.v, p.status) : 0;
        if (tok < 0) {
            if (p.parts == 1) put_skipped<W>(p, i);
            continue;
        }
        const char *row = elem_at<DT>(p.z, i * p.ldz);
        const int first = part * p.part_vecs, end = min(full, first + p.part_vecs);
        const int rem = end == full ? rest : 0;  // the tail is the last part's
        // the token's logit is wanted at the end: asked for now
        const float zt = thread == 0 && p.logp && p.parts == 1 ? load1<DT>(row, tok) : 0.0f;
        Stat t = empty_stat();
        Selection<DT, W> sel;
        int j = first;
        Tile tile = load_tile<DT, W>(row, j, end);
        const float tail = tail_elem<DT, W>(row, full, rem);
        if (rem > 0) add_elem<true>(tail, p.c, t);
        if constexpr (TOP) sel.start();
        for (int turn = 0; j < end; ++turn, j += kStep) {
            const Tile now = tile;
            if (j + kStep < end) tile = load_tile<DT, W>(row, j + kStep, end);
            float lm[kTileVecs];
            add_tile<DT, true>(now, p.c, t, lm);
            if constexpr (TOP) sel.take(top, lm, turn, j + thread, end, p.top, p.at_bits);
        }
        t = team_stat<W>(t, p.c);
        if constexpr (TOP) {
            sel.finish(top, row, full, rem, p.top, p.at_bits);
            if (p.parts == 1) {
                put_top<DT>(p, i, t, top);
            } else {
                uint32_t *to = p.part_top + w * p.top * 2;
                for (int q = thread; q < p.top; q += kT)
                    if (q >= top.n) to[2 * q] = to[2 * q + 1] = 0;
                by_rank(top, p.top, [&](int r, uint32_t key, uint32_t at) {
                    to[2 * r] = key;
                    to[2 * r + 1] = at;
                });
            }
            Team<W>::sync();
        }
        if (thread == 0) {
            if (p.parts == 1)
                put_row_stat(p, i, zt, t);
            else
                put_part(p.part_stat, w, t);
        }
    }
}

constexpr int kJoin = 2048;  // candidates that the parts of a row hand over, at most

template <int DT>
__global__ __launch_bounds__(kBlock) void k_logprobs_join(LogprobArgs p) {
    constexpr int kW = kBlock / kWave;
    __shared__ TopLds<kW> s_top;
    for (int64_t i = blockIdx.x; i < p.n; i += gridDim.x) {
        const int32_t tok = p.tokens ? read_token(p.tokens, p.index, i, p.v, nullptr) : 0;
        if (tok < 0) {
            put_skipped<kW>(p, i);
            continue;
        }
        const float zt = threadIdx.x == 0 && p.logp
                             ? load1<DT>(elem_at<DT>(p.z, i * p.ldz), tok) : 0.0f;
        const Stat t = join_parts(p.part_stat, i, p.parts, p.c);
        if (threadIdx.x == 0) put_row_stat(p, i, zt, t);
        if (p.top == 0) continue;
        const uint32_t *from = p.part_top + i * p.parts * p.top * 2;
        const int count = p.parts * p.top;
        if (threadIdx.x == 0) s_top.n = 0;
        __syncthreads();
        if (count <= TopLds<kW>::kRanked) {
            // no worse than any part's K-th best
            const int last = (lane_id() + 1) * p.top - 1;
            const uint32_t least = max(wave_max_u32(lane_id() < p.parts ? from[2 * last] : 0), 1u);
            for (int k = threadIdx.x; k < count; k += kBlock)
                if (from[2 * k] >= least) push(s_top, from[2 * k], from[2 * k + 1]);
        } else {
            constexpr int kN = kJoin / kBlock;
            uint32_t key[kN], at[kN];
#pragma unroll
            for (int q = 0; q < kN; ++q) {
                const int k = q * kBlock + threadIdx.x;
                key[q] = k < count ? from[2 * k] : 0;
                at[q] = k < count ? from[2 * k + 1] : 0;
            }
            const Bound b = kth_best<DT, kW>(key, at, p.top, p.at_bits + 3);
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

template <int DT, int W>
__global__ __launch_bounds__(kBlock) void k_logprobs_grad(LogprobGradArgs p) {
    constexpr int kV = Elem<DT>::kVec;
    const int full = (int)(p.v / kV), rest = (int)(p.v % kV), thread = Team<W>::thread();
    for (int64_t w = (int64_t)blockIdx.x * Team<W>::kPerBlock + Team<W>::here();
         w < p.n * p.parts; w += (int64_t)gridDim.x * Team<W>::kPerBlock) {
        const auto [i, part] = Work(w, p.parts);
        const int first = part * p.part_vecs, end = min(full, first + p.part_vecs);
        const int rem = end == full ? rest : 0;  // the tail is the last part's
        const int32_t tok = p.tokens ? read_token(p.tokens, p.index, i, p.v, p.status) : 0;
        const char *row = elem_at<DT>(p.z, i * p.ldz);
        char *out = elem_at<DT>(p.dz, i * p.ldd);
        const float m = p.stats[2 * i], ls = p.stats[2 * i + 1];
        if (tok < 0 || ls == kNegInf) {
            zero_row<DT, W>(out, first, end, full, rem);
            continue;
        }
        // dz = q (a + b log q), and d_logp / T more at the token
        const float g = p.d_logp ? p.d_logp[i] * p.inv_t : 0.0f;
        const float b = p.d_entropy ? -p.d_entropy[i] * p.inv_t : 0.0f;
        const float a = p.d_entropy ? __builtin_fmaf(b, p.entropy[i], -g) : -g;
        auto gradient = [&](float z) {
            const float lq = __builtin_fmaf(z - m, p.inv_t, -ls);
            // q by its root twice: the product reaches the subnormals, which the
            // instruction's own results do not.  Where q is 0 so is the product,
            // whatever log q
            const float r = exp2_raw(lq * (0.5f * kLog2e));
            return r * (r * __builtin_fmaf(b, fmaxf(lq, kLogFloor), a));
        };
        const float tail = tail_elem<DT, W>(row, full, rem);
        map_row<DT, W>(row, out, first, end, [&](int j, float *x) {
#pragma unroll
            for (int e = 0; e < kV; ++e) x[e] = gradient(x[e]);
            const int hot = tok - j * kV;
            if (hot >= 0 && hot < kV && p.d_logp) {
#pragma unroll
                for (int e = 0; e < kV; ++e)
                    if (e == hot) x[e] += g;
            }
        });
        if (thread < rem) {
            const int at = full * kV + thread;
            store1<DT>(out, at, gradient(tail) + (at == tok && p.d_logp ? g : 0.0f));
        }
    }
}

}  // namespace
}  // namespace pdbk

using namespace pdbk;

namespace {
// parts of a row, so that what they hand over fits the joining block
int64_t most_parts(int32_t top) {
    return top > 0 ? std::min<int64_t>(kMostParts, kJoin / top) : kMostParts;
}
// Blocks for `work` items of a team each, of `vecs` vectors, six blocks to a compute
// unit at once.  Items that are up to half more than fit would leave most of the card
// idle behind the first: two to a team then, where that deals the blocks evenly and an
// item is long (2,048 rows of 131,072: 102 us, then 95; 8,192 of 32,768 with 5
// alternatives, a wave each: 140, then 132; but 2,040 of 40,000, five tiles long, 51,
// then 55, and 2,300 of 50,257, four and a half blocks a unit, 42, then 48).  Three turns
// and two and a half were not measured and are dealt as they come.
unsigned blocks_in_turns(int64_t work, int per_block, int64_t vecs) {
    const int64_t fit = 6 * 256 * per_block, two = cdiv(work, 2 * per_block);
    const bool even = cdiv(two, 256) * 256 - two <= two / 16;
    const bool lengthy = vecs >= 8 * kTileVecs * (kBlock / per_block);
    if (work > fit && work <= fit + fit / 2 && even && lengthy) return (unsigned)two;
    return blocks_for(work, per_block);
}
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
        constexpr int DT = decltype(dt)::value, kV = Elem<DT>::kVec, kW = kBlock / kWave;
        const Parts cut = cut_rows(n, v, kV, most_parts(top));
        const LogprobArgs p = {logits, ldz, n, v, tokens, index, top, bits_for(cdiv(v, kV)),
                               1.0f / temp, kLog2e / temp, logp, entropy, stats, top_id, top_logp,
                               status, cut.vecs, cut.parts, static_cast<float *>(ws),
                               reinterpret_cast<uint32_t *>(
                                   static_cast<char *>(ws) + stat_bytes(std::min(n, kWantBlocks)))};
        const bool wave = wave_rows(cut, n, v, kV, top > 0) && top <= TopLds<1>::kTop;
        const unsigned blocks =
            blocks_in_turns(n * cut.parts, wave ? Team<1>::kPerBlock : 1, cut.vecs);
        if (wave && top > 0)
            k_logprobs<DT, 1, true><<<blocks, kBlock, 0, s>>>(p);
        else if (wave)
            k_logprobs<DT, 1, false><<<blocks, kBlock, 0, s>>>(p);
        else if (top > 0)
            k_logprobs<DT, kW, true><<<blocks, kBlock, 0, s>>>(p);
        else
            k_logprobs<DT, kW, false><<<blocks, kBlock, 0, s>>>(p);
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
        constexpr int DT = decltype(dt)::value, kV = Elem<DT>::kVec;
        const Parts cut = cut_rows(n, v, kV, kMostParts);
        const LogprobGradArgs p = {logits, ldz, n, v, tokens, index, 1.0f / temp, stats, entropy,
                                   d_logp, d_entropy, dlogits, ldd, status, cut.vecs, cut.parts};
        if (wave_rows(cut, n, v, kV, false))
            k_logprobs_grad<DT, 1><<<blocks_for(n, Team<1>::kPerBlock), kBlock, 0, s>>>(p);
        else
            k_logprobs_grad<DT, kBlock / kWave><<<blocks_for(n * cut.parts), kBlock, 0, s>>>(p);
        PDB_LAUNCHED();
        return PDB_OK;
    });
}
