// Embedding lookup and its gradient (gfx950, wave64).
//
//   lookup    out[i] = scale * table[t_i]
//   gradient  grad[t] (+)= scale * sum_{i: t_i = t} dy[i], i ascending
//
// Both move rows and compute next to nothing: their floor is the rows' bytes at
// the copy rate.  A row is handled by a group of 2^lg lanes (up to the block),
// each lane a 16-byte vector per access, so consecutive lanes read consecutive
// bytes of a row and short rows still fill a wave.
//
// The gradient sorts the tokens (stable, so a token's positions stay ascending)
// and cuts the sorted list into tiles of R entries, whatever token they hold: a
// hot token's rows are then spread over many groups and a rare token costs one
// row.  A token whose entries lie in one tile is written by that tile; the
// parts of one that crosses tiles go to a partial buffer and are joined in
// tile order by a second kernel.  No atomics on sums: their order follows from the
// sizes and from where the tiles cut the sorted tokens, and is the same in every call
// on the same tokens.
#include "pdb_vec.h"

namespace pdbk {
namespace {

// lanes per row: the smallest power of two that covers its vectors, up to a block
inline int lanes_log2(int64_t vectors) {
    int lg = 0;
    while (lg < 8 && ((int64_t)1 << lg) < vectors) ++lg;
    return lg;
}

template <int A, int B>
struct Pair {  // elements a lane handles at once: a whole vector of the narrower type
    static constexpr int kE = Elem<A>::kVec > Elem<B>::kVec ? Elem<A>::kVec : Elem<B>::kVec;
};

// E elements at column c of a row of d; a row's last, partial vector element by element
template <int DT, int E>
__device__ __forceinline__ void load_cols(const void *p, int64_t row, int64_t c, int64_t d,
                                          float *x) {
    if (c + E <= d) {
        load_elems<DT, E>(p, row + c, x);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = c + e < d ? load1<DT>(p, row + c + e) : 0.0f;
    }
}
template <int DT, int E>
__device__ __forceinline__ void store_cols(void *p, int64_t row, int64_t c, int64_t d,
                                           const float *x) {
    if (c + E <= d) {
        store_elems<DT, E>(p, row + c, x);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (c + e < d) store1<DT>(p, row + c + e, x[e]);
    }
}

// ----------------------------------------------------------------------------
// lookup

template <int TT, int OT>
__global__ __launch_bounds__(kBlock) void k_embed_lookup(const void *__restrict__ table,
                                                         int64_t ld, int64_t v, int64_t d,
                                                         const void *__restrict__ tokens,
                                                         int index, int64_t n, float scale,
                                                         void *__restrict__ out, int64_t ldo,
                                                         int lg, int32_t *status) {
    constexpr int kE = Pair<TT, OT>::kE;
    const int lane = threadIdx.x & ((1 << lg) - 1);
    const int per = kBlock >> lg;
    const int64_t c = ((int64_t)blockIdx.y << lg | lane) * kE;
    if (c >= d) return;
    for (int64_t i = (int64_t)blockIdx.x * per + (threadIdx.x >> lg); i < n;
         i += (int64_t)gridDim.x * per) {
        const int32_t t = read_token(tokens, index, i, v, status);
        float x[kE];
        if (t >= 0) {
            load_cols<TT, kE>(table, (int64_t)t * ld, c, d, x);
#pragma unroll
            for (int e = 0; e < kE; ++e) x[e] *= scale;
        } else {
#pragma unroll
            for (int e = 0; e < kE; ++e) x[e] = 0.0f;
        }
        store_cols<OT, kE>(out, i * ldo, c, d, x);
    }
}

// ----------------------------------------------------------------------------
// gradient: tokens in order
//
// (token, position) in order, stable.  Few tokens are placed by counting, in one
// launch.  More go through a radix sort: a block of 1024 threads takes a tile of up
// to 8 x 1024 tokens, each wave a stretch of it, and ranks them by ballots (a hot
// token costs nothing extra).  A pass is two launches, the tiles' digit counts and
// the move, each block summing the counts of all tiles by itself; where that reading
// grows too long a scan of the counts stands between them.  Digits have up to 10 bits,
// so that 2^20 rows take two passes.  4M tokens of rank 32, sort and sums: 270 us in
// three passes of 7 bits, 256 in two of 10, 252 where the first pass reads the tokens
// twice instead of leaving their keys, 245 with the blocks dealt to the dies as
// tile_of_block says, 240 with tiles of 8,192 tokens, two to a compute unit, instead of
// 16,384 (255 of 6,144), and 233 with today's scan and join.  Past kSortTiles, where the
// counts would outgrow their place, the general sort of pdb_internal.h runs (8,388,608
// tokens of rank 32: 415 us, 146 of them sorting; 8.4M so: 531; 20M: 1,065, 495 sorting).

constexpr int kSortBlock = 1024;
constexpr int kSortItems = 8;
constexpr int kSortTile = kSortBlock * kSortItems;
constexpr int kSortTiles = 1024;
constexpr int64_t kSortMost = (int64_t)kSortTiles * kSortTile;
constexpr int kDigitBits = 10;  // of the widest digit
constexpr int kDigits = 1 << kDigitBits;

struct SortLds {
    union {
        struct {
            uint32_t key[kSortTile], val[kSortTile];
        };
        // per wave and digit: a count, then where its run starts
        uint32_t cnt[kSortBlock / kWave][kDigits];
    };
    uint32_t start[kDigits];                // per digit: where it starts in the tile
    uint32_t out[kDigits], all[kDigits];    // per digit: where it goes; all tiles' count
    uint32_t wave[kSortBlock / kWave];
};

__device__ __forceinline__ uint32_t digit_of(uint32_t key, int shift, int nb) {
    return (key >> shift) & ((1u << nb) - 1u);
}
// The lanes that hold the same digit: of each bit's ballot, or its complement,
// by the lane's own bit spread over a word.  All B bits of a digit are looked at
// (those above nb are 0): unrolled, they take half the instructions of a loop.
template <int B>
__device__ __forceinline__ unsigned long long digit_peers(uint32_t dg, bool valid) {
    const unsigned long long there = __ballot(valid);
    uint32_t lo = (uint32_t)there, hi = (uint32_t)(there >> 32);
#pragma unroll
    for (int b = 0; b < B; ++b) {
        const uint32_t own = (uint32_t)__builtin_amdgcn_sbfe((int)dg, b, 1);
        const unsigned long long set = __ballot(own != 0);
        lo &= ~((uint32_t)set ^ own);
        hi &= ~((uint32_t)(set >> 32) ^ own);
    }
    return (unsigned long long)hi << 32 | lo;
}

// exclusive prefix sum over the block's threads
__device__ __forceinline__ uint32_t scan_block(uint32_t v, uint32_t *s_wave) {
    const uint32_t incl = wave_incl_scan_u32(v);
    const int w = wave_in_block();
    if (lane_id() == kWave - 1) s_wave[w] = incl;
    __syncthreads();
    const uint32_t of_wave = lane_id() < w ? s_wave[lane_id()] : 0;  // the waves before
    return wave_sum_u32(of_wave) + incl - v;
}

// Item j of a thread is entry (wave * items + j) * 64 + lane of the tile.
__device__ __forceinline__ int tile_entry(int items, int j) {
    return (wave_in_block() * items + j) * kWave + lane_id();
}

// The place of each item in the tile by its digit (of up to B bits), items of one
// digit in order.
template <int B>
__device__ __forceinline__ void rank_tile(SortLds &S, const uint32_t *k, int items, int count,
                                          int shift, int nb, uint32_t *pos) {
    const int t = threadIdx.x, w = wave_in_block(), radix = 1 << nb;
    for (int i = lane_id(); i < radix; i += kWave) S.cnt[w][i] = 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kSortItems; ++j) {
        if (j >= items) continue;
        const bool valid = tile_entry(items, j) < count;
        const uint32_t dg = digit_of(k[j], shift, nb);
        const unsigned long long peers = digit_peers<B>(dg, valid);
        const unsigned r = lanes_below(peers);
        // of the wave's items before this one (a wave's LDS accesses run in order)
        const uint32_t before =
            __hip_atomic_load(&S.cnt[w][dg], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT);
        __builtin_amdgcn_wave_barrier();
        if (valid && r == 0)
            __hip_atomic_store(&S.cnt[w][dg], before + (uint32_t)__popcll(peers), __ATOMIC_RELAXED,
                               __HIP_MEMORY_SCOPE_WAVEFRONT);
        __builtin_amdgcn_wave_barrier();
        pos[j] = before + r;
    }
    __syncthreads();
    uint32_t sum = 0;
    if (t < radix) {
#pragma unroll
        for (int q = 0; q < kSortBlock / kWave; ++q) {
            const uint32_t c = S.cnt[q][t];
            S.cnt[q][t] = sum;
            sum += c;
        }
    }
    const uint32_t start = scan_block(sum, S.wave);
    if (t < radix) S.start[t] = start;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kSortItems; ++j) {
        if (j >= items) continue;
        const uint32_t dg = digit_of(k[j], shift, nb);
        pos[j] += S.start[dg] + S.cnt[w][dg];
    }
}

// a token as a sort key: padding goes behind every row of the table
__device__ __forceinline__ uint32_t token_key(const void *tokens, int index, int64_t i, int64_t v,
                                              int32_t *status) {
    const int32_t t = read_token(tokens, index, i, v, status);
    return t < 0 ? (uint32_t)v : (uint32_t)t;
}

// Up to kRankTokens tokens: a token's place is the number of those that go before
// it, counted.  n^2 comparisons of two instructions each, all compute units at
// it, cost less than the launches of a radix sort.  A block has all keys in LDS and
// 64 tokens to place, each wave every 16th 64 of the keys (9,000 tokens of rank 32, sums
// and all: 28 us, sorted 31; 12,000: 31, sorted 31).  Of tokens that one pass sorts, only
// half as many (8,000 of 200 rows: 28 us counted, 22 sorted; 6,200: 23 both ways).
constexpr int kRankTokens = 12288;
constexpr int64_t rank_tokens(int bits) {
    return bits <= kDigitBits ? kRankTokens / 2 : kRankTokens;
}
__global__ __launch_bounds__(kSortBlock) void k_token_rank(const void *__restrict__ tokens,
                                                           int index, int n, int64_t v,
                                                           uint32_t *__restrict__ keys,
                                                           uint32_t *__restrict__ vals,
                                                           int32_t *status) {
    __shared__ __align__(16) uint32_t s_key[kRankTokens];
    __shared__ uint32_t s_before[kWave];
    const int blocks = (n + kWave - 1) / kWave, mine = blockIdx.x;
    uint32_t k[kRankTokens / kSortBlock];
#pragma unroll
    for (int j = 0; j < kRankTokens / kSortBlock; ++j) {  // all loads before the first is used
        const int i = j * kSortBlock + (int)threadIdx.x;
        k[j] = i < n ? token_key(tokens, index, i, v, status) : 0xFFFFFFFFu;  // before none
    }
#pragma unroll
    for (int j = 0; j < kRankTokens / kSortBlock; ++j) s_key[j * kSortBlock + threadIdx.x] = k[j];
    if (threadIdx.x < kWave) s_before[threadIdx.x] = 0;
    __syncthreads();
    const int lane = lane_id();
    const uint32_t own = s_key[mine * kWave + lane];
    uint32_t before = 0;
    for (int q = wave_in_block(); q < blocks; q += kSortBlock / kWave) {
        const uint4 *k = reinterpret_cast<const uint4 *>(s_key + q * kWave);
        if (q == mine) {  // equal ones among these 64: by position
            for (int j = 0; j < kWave; ++j) {
                const uint32_t o = s_key[q * kWave + j];
                before += o < own || (o == own && j < lane);
            }
        } else {
            // an equal one counts where it stands before
            const uint32_t most = q < mine ? own + 1 : own;
#pragma unroll
            for (int j = 0; j < kWave / 4; ++j) {
                const uint4 o = k[j];
                before += o.x < most;
                before += o.y < most;
                before += o.z < most;
                before += o.w < most;
            }
        }
    }
    atomicAdd(&s_before[lane], before);
    __syncthreads();
    const int i = mine * kWave + (int)threadIdx.x;
    if (threadIdx.x < kWave && i < n) {
        keys[s_before[threadIdx.x]] = own;
        vals[s_before[threadIdx.x]] = (uint32_t)i;
    }
}

// The keys that a pass sorts: of the tokens (FIRST), or as the pass before left them.
struct SortIn {
    const void *tokens;
    int index;
    int64_t v;
    int32_t *status;
    const uint32_t *keys, *vals;
    int64_t n;
    int items, shift, nb, tiles;
};
template <bool FIRST>
__device__ __forceinline__ uint32_t sort_key(const SortIn &in, int64_t i, int32_t *status) {
    return FIRST ? token_key(in.tokens, in.index, i, in.v, status) : in.keys[i];
}

// Digit counts of each tile, [tile][digit].
template <bool FIRST>
__global__ __launch_bounds__(kSortBlock) void k_token_sort_count(SortIn in,
                                                                 uint32_t *__restrict__ hist) {
    constexpr int kCopies = 4;  // of the counts, for a quarter of the waves each
    __shared__ uint32_t s_cnt[kCopies][kDigits];
    const int t = threadIdx.x;
    uint32_t *mine = s_cnt[wave_in_block() % kCopies];
    if (t < (1 << in.nb))
#pragma unroll
        for (int q = 0; q < kCopies; ++q) s_cnt[q][t] = 0;
    static_assert(kDigits <= kSortBlock, "a digit a thread");
    __syncthreads();
    const int64_t base = (int64_t)blockIdx.x * in.items * kSortBlock;
    uint32_t k[kSortItems];
#pragma unroll
    for (int j = 0; j < kSortItems; ++j) {  // all loads before the first is used
        const int64_t i = base + j * kSortBlock + t;
        k[j] = j < in.items && i < in.n ? sort_key<FIRST>(in, i, in.status) : 0;
    }
#pragma unroll
    for (int j = 0; j < kSortItems; ++j) {
        if (j >= in.items) continue;
        const bool valid = base + j * kSortBlock + t < in.n;
        const uint32_t dg = digit_of(k[j], in.shift, in.nb);
        // a digit that many lanes hold is counted once for all of them: adds to one
        // LDS address go one after another
        const uint32_t d0 = (uint32_t)__builtin_amdgcn_readfirstlane((int)dg);
        const unsigned long long same = __ballot(valid && dg == d0);
        const bool hot = __popcll(same) >= 4;
        if (hot && lane_id() == 0) atomicAdd(&mine[d0], (uint32_t)__popcll(same));
        if (valid && !(hot && dg == d0)) atomicAdd(&mine[dg], 1u);
    }
    __syncthreads();
    if (t < (1 << in.nb)) {
        uint32_t all = 0;
#pragma unroll
        for (int q = 0; q < kCopies; ++q) all += s_cnt[q][t];
        hist[((int64_t)blockIdx.x << in.nb) + t] = all;
    }
}

// Of many tiles or wide digits: each digit's count in the tiles before, in place of
// its counts, and behind the last tile its count in all.  A block has 32 digits, half a
// wave every 32nd part of the tiles (489 tiles of 1,024 digits: 5.0 us; 64 digits and a
// wave every 16th part: 7.2).
constexpr int kScanDigits = 32, kScanParts = kSortBlock / kScanDigits;
constexpr int kScanTiles = 16;  // counts that a lane has in flight
__global__ __launch_bounds__(kSortBlock) void k_token_sort_scan(uint32_t *__restrict__ hist,
                                                                int tiles, int nb) {
    __shared__ uint32_t s_sum[kScanParts][kScanDigits];
    const int part = threadIdx.x / kScanDigits, mine = threadIdx.x % kScanDigits;
    const int d = (int)blockIdx.x * kScanDigits + mine;
    const int per = (tiles + kScanParts - 1) / kScanParts;
    const int from = part * per, to = min(tiles, from + per);
    uint32_t c[kScanTiles], sum = 0;
    auto load = [&](int q0) {
#pragma unroll
        for (int q = 0; q < kScanTiles; ++q)
            c[q] = q0 + q < to ? hist[((int64_t)(q0 + q) << nb) + d] : 0;
    };
    for (int q0 = from; q0 < to; q0 += kScanTiles) {
        load(q0);
#pragma unroll
        for (int q = 0; q < kScanTiles; ++q) sum += c[q];
    }
    s_sum[part][mine] = sum;
    __syncthreads();
    uint32_t before = 0;
#pragma unroll
    for (int q = 0; q < kScanParts; ++q) before += q < part ? s_sum[q][mine] : 0;
    for (int q0 = from; q0 < to; q0 += kScanTiles) {
        if (per > kScanTiles) load(q0);
#pragma unroll
        for (int q = 0; q < kScanTiles; ++q) {
            if (q0 + q < to) hist[((int64_t)(q0 + q) << nb) + d] = before;
            before += c[q];
        }
    }
    if (part == kScanParts - 1) hist[((int64_t)tiles << nb) + d] = before;
}

// Block b's tile: the blocks of one die (b mod 8) have neighbouring tiles, whose
// stretches of a digit lie next to each other and meet in that die's cache.
__device__ __forceinline__ int tile_of_block(int b, int tiles) {
    const int die = b & 7;
    return die * (tiles >> 3) + min(die, tiles & 7) + (b >> 3);
}

// One pass, on digits of up to B bits; the first one's values are positions.  scanned:
// hist is as k_token_sort_scan leaves it.
template <int B, bool FIRST>
__global__ __launch_bounds__(kSortBlock) void k_token_sort_move(
    SortIn in, const uint32_t *__restrict__ hist, bool scanned, uint32_t *__restrict__ keys,
    uint32_t *__restrict__ vals) {
    __shared__ SortLds S;
    const int items = in.items, shift = in.shift, nb = in.nb, tiles = in.tiles;
    const int t = threadIdx.x, radix = 1 << nb, tile = tile_of_block((int)blockIdx.x, tiles);
    const int64_t base = (int64_t)tile * items * kSortBlock;
    const int count = (int)min((int64_t)items * kSortBlock, in.n - base);
    uint32_t k[kSortItems], p[kSortItems], pos[kSortItems];
#pragma unroll
    for (int j = 0; j < kSortItems; ++j) {
        if (j >= items) continue;
        const int e = tile_entry(items, j);
        k[j] = e < count ? sort_key<FIRST>(in, base + e, nullptr) : 0;
        p[j] = FIRST ? (uint32_t)(base + e) : e < count ? in.vals[base + e] : 0;
    }
    // where each digit of this tile goes: every smaller digit, and this one in
    // the tiles before
    uint32_t mine = 0, all = 0;
    if (scanned) {
        if (t < radix) {
            mine = hist[((int64_t)tile << nb) + t];
            all = hist[((int64_t)tiles << nb) + t];
        }
    } else {
        if (t < radix) S.all[t] = S.out[t] = 0;
        __syncthreads();
#pragma unroll 8
        for (int q = t >> nb; q < tiles; q += kSortBlock >> nb) {
            const uint32_t c = hist[((int64_t)q << nb) + (t & (radix - 1))];
            all += c;
            mine += q < tile ? c : 0;
        }
        atomicAdd(&S.all[t & (radix - 1)], all);
        atomicAdd(&S.out[t & (radix - 1)], mine);
        __syncthreads();
        mine = t < radix ? S.out[t] : 0;
        all = t < radix ? S.all[t] : 0;
    }
    const uint32_t smaller = scan_block(all, S.wave);
    if (t < radix) S.out[t] = mine + smaller;
    __syncthreads();
    rank_tile<B>(S, k, items, count, shift, nb, pos);
    __syncthreads();  // the counts' place is the tile's now
#pragma unroll
    for (int j = 0; j < kSortItems; ++j) {
        if (j >= items) continue;
        if (tile_entry(items, j) < count) {
            S.key[pos[j]] = k[j];
            S.val[pos[j]] = p[j];
        }
    }
    __syncthreads();
    // in the tile's order: consecutive threads write a digit's consecutive slots
    for (int e = t; e < count; e += kSortBlock) {
        const uint32_t kk = S.key[e], dg = digit_of(kk, shift, nb);
        const uint32_t to = S.out[dg] + ((uint32_t)e - S.start[dg]);
        keys[to] = kk;
        vals[to] = S.val[e];
    }
}

// tokens to sort keys, for the general sort
__global__ __launch_bounds__(kBlock) void k_token_keys(const void *__restrict__ tokens, int index,
                                                       int64_t n, int64_t v,
                                                       uint32_t *__restrict__ keys,
                                                       int32_t *status) {
    for (int64_t i = blockIdx.x * (int64_t)kBlock + threadIdx.x; i < n;
         i += (int64_t)gridDim.x * kBlock)
        keys[i] = token_key(tokens, index, i, v, status);
}

// ----------------------------------------------------------------------------
// gradient: sums

// E elements at column c of a row, as they are stored
template <int DT, int E>
struct RawCols {
    u32x4 r[E / Elem<DT>::kVec];
};
template <int DT, int E>
__device__ __forceinline__ RawCols<DT, E> load_raw(const void *p, int64_t row, int64_t c,
                                                   int64_t d) {
    constexpr int kV = Elem<DT>::kVec;
    RawCols<DT, E> x;
    if (c + E <= d) {
#pragma unroll
        for (int k = 0; k < E / kV; ++k) x.r[k] = load16(elem_at<DT>(p, row + c + k * kV));
    } else {
        float f[E];
        load_cols<DT, E>(p, row, c, d, f);
#pragma unroll
        for (int k = 0; k < E / kV; ++k) x.r[k] = pack<DT>(f + k * kV);
    }
    return x;
}
template <int DT, int E>
__device__ __forceinline__ void unpack_raw(const RawCols<DT, E> &x, float *f) {
    constexpr int kV = Elem<DT>::kVec;
#pragma unroll
    for (int k = 0; k < E / kV; ++k) unpack<DT>(x.r[k], f + k * kV);
}

// grad[t] at columns c.. from a finished sum and what it held (accumulate)
template <int GT, int E>
__device__ __forceinline__ void put_row(void *grad, int64_t ldg, uint32_t t, int64_t c, int64_t d,
                                        float scale, bool accumulate, const RawCols<GT, E> &old,
                                        const float *sum) {
    float x[E];
    if (accumulate) {
        unpack_raw<GT, E>(old, x);
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = __builtin_fmaf(scale, sum[e], x[e]);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = scale * sum[e];
    }
    store_cols<GT, E>(grad, (int64_t)t * ldg, c, d, x);
}

// Zeros in those of the 64 rows from r0 on that `free` names.  Rows without gaps that
// begin anywhere, or are long, are cleared in stretches, whole aligned vectors wherever
// rows end (131,072 rows of 2,047 floats: 295 us row by row, 186 so; of 2,048: 193).
template <int GT>
__device__ __forceinline__ void zero_rows(void *grad, int64_t ldg, int64_t r0, int64_t d, int lg,
                                          unsigned long long free) {
    constexpr int kE = Elem<GT>::kVec;
    const float zero[kE] = {};
    if (ldg == d && (d % kE != 0 || d >= 256)) {
        while (free) {
            const int from = __builtin_ctzll(free);
            const unsigned long long rest = ~(free >> from);
            const int rows = rest ? __builtin_ctzll(rest) : kWave;  // (from 0 on then)
            free = rows + from >= kWave ? 0 : free >> (from + rows) << (from + rows);
            char *a = elem_at<GT>(grad, (r0 + from) * d);
            char *z = a + (int64_t)rows * d * Elem<GT>::kSize;
            char *a16 = a + (-(uintptr_t)a & 15), *z16 = z - ((uintptr_t)z & 15);
            if (a16 > z16) a16 = z16 = z;
            for (char *q = a + threadIdx.x * Elem<GT>::kSize; q < a16; q += kBlock * Elem<GT>::kSize)
                store1<GT>(q, 0, 0.0f);
            for (char *q = a16 + threadIdx.x * 16; q < z16; q += kBlock * 16)
                store16(q, u32x4{0, 0, 0, 0});
            for (char *q = z16 + threadIdx.x * Elem<GT>::kSize; q < z; q += kBlock * Elem<GT>::kSize)
                store1<GT>(q, 0, 0.0f);
        }
        return;
    }
    const int lane = threadIdx.x & ((1 << lg) - 1);
    for (int q = threadIdx.x >> lg; q < kWave; q += kBlock >> lg)
        if ((free >> q) & 1ull)
            for (int64_t c = (int64_t)lane * kE; c < d; c += (int64_t)kE << lg)
                store_cols<GT, kE>(grad, (r0 + q) * ldg, c, d, zero);
}

constexpr int kAhead = 4;         // rows a lane has in flight
constexpr int kStaged = 1024;     // entries of a block's tiles, in LDS
constexpr int kDirect = kBlock;   // tokens that the direct kernel takes

struct GradArgs {
    const void *dy;
    int64_t ldy;
    const uint32_t *keys, *vals;  // sorted
    const void *tokens;           // the direct kernel's
    int index;
    int64_t n, d, v;
    int R, lg, zero_lg;    // entries of a tile; lanes of a row (log2)
    int64_t span;          // entries of a block's tiles
    int64_t sum_blocks, zero_blocks;
    float scale;
    void *grad;
    int64_t ldg;
    float *part;  // [sum_blocks][2][d]
    int32_t *status;
};

// first entry whose key is >= t
__device__ __forceinline__ int64_t lower_bound_key(const uint32_t *keys, int64_t lo, int64_t hi,
                                                   uint32_t t) {
    while (lo < hi) {
        const int64_t mid = (lo + hi) >> 1;
        if (keys[mid] < t)
            lo = mid + 1;
        else
            hi = mid;
    }
    return lo;
}

// The blocks that sum and those that write zeros alternate: the first wait for
// scattered rows, the second for nothing.  -1: nothing to do.
__device__ __forceinline__ int64_t sum_block(const GradArgs &p, int64_t x, bool &zero) {
    const int64_t both = 2 * min(p.sum_blocks, p.zero_blocks);
    zero = x < both ? x & 1 : p.zero_blocks > p.sum_blocks;
    return x < both ? x >> 1 : x - (both >> 1);
}

// One tile of R sorted entries per group, a block's tiles one after another.  A
// token that lies in one tile is written by its group.  One that crosses tiles of
// the block is joined in LDS by the group where it begins.  One that crosses blocks
// goes to the partials: slot 0 of a block is what it adds to a token that began
// before it, slot 1 to one that goes on after it.
template <int DT, int GT, bool ACC>
__global__ __launch_bounds__(kBlock) void k_embed_tiles(GradArgs p) {
    constexpr int kE = Pair<DT, GT>::kE;
    __shared__ uint32_t s_key[kStaged + 2], s_val[kStaged];
    __shared__ float s_head[kBlock * kE];  // of each group, what it adds to a token from before it
    __shared__ unsigned long long s_free;
    bool zero;
    const int64_t block = sum_block(p, blockIdx.x, zero);
    if (!ACC && zero) {
        if (blockIdx.y > 0) return;
        for (int64_t r0 = block * kWave; r0 < p.v; r0 += p.zero_blocks * kWave) {
            if (wave_in_block() == 0) {
                const int64_t r = r0 + lane_id();
                bool free = false;
                if (r < p.v) {
                    const int64_t at = lower_bound_key(p.keys, 0, p.n, (uint32_t)r);
                    free = at >= p.n || p.keys[at] != (uint32_t)r;
                }
                const unsigned long long m = __ballot(free);
                if (lane_id() == 0) s_free = m;
            }
            __syncthreads();
            zero_rows<GT>(p.grad, p.ldg, r0, p.d, p.zero_lg, s_free);
            __syncthreads();
        }
        return;
    }
    const int groups = kBlock >> p.lg, g = threadIdx.x >> p.lg;
    const int lane = threadIdx.x & ((1 << p.lg) - 1);
    const int64_t from = block * p.span;
    // the block's entries, and the key on either side of them (none: 2^32 - 1,
    // which is no row's)
    const int here = (int)min(p.span, p.n - from);
    for (int i = threadIdx.x; i < here + 2; i += kBlock) {
        const int64_t e = from + i - 1;
        s_key[i] = e >= 0 && e < p.n ? p.keys[e] : 0xFFFFFFFFu;
        if (i < here) s_val[i] = p.vals[from + i];
    }
    __syncthreads();
    const int64_t c = ((int64_t)blockIdx.y << p.lg | lane) * kE;
    const int e0 = g * p.R, e1 = min(here, e0 + p.R);
    const bool live = e0 < here && c < p.d;
    const uint32_t none = (uint32_t)p.v;  // padding, which comes last
    float sum[kE];
#pragma unroll
    for (int q = 0; q < kE; ++q) sum[q] = 0.0f;
    // whether the tile's first token began before it
    const bool opened = live && s_key[e0] == s_key[e0 + 1] && s_key[e0] != none;
    bool began = opened;
    auto put_head = [&]() {
#pragma unroll
        for (int q = 0; q < kE; ++q) s_head[q * kBlock + threadIdx.x] = sum[q];
    };
    for (int e = e0; live && e < e1; e += kAhead) {
        RawCols<DT, kE> x[kAhead];
        RawCols<GT, kE> old[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int at = min(e + k, e1 - 1);
            const uint32_t t = s_key[at + 1];
            if (t == none) break;
            x[k] = load_raw<DT, kE>(p.dy, (int64_t)s_val[at] * p.ldy, c, p.d);
            if (ACC && s_key[at + 2] != t)
                old[k] = load_raw<GT, kE>(p.grad, (int64_t)t * p.ldg, c, p.d);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (e + k >= e1) break;
            const uint32_t t = s_key[e + k + 1];
            if (t == none) break;
            float f[kE];
            unpack_raw<DT, kE>(x[k], f);
#pragma unroll
            for (int q = 0; q < kE; ++q) sum[q] += f[q];
            if (s_key[e + k + 2] == t) continue;
            if (began)
                put_head();
            else
                put_row<GT, kE>(p.grad, p.ldg, t, c, p.d, p.scale, ACC, old[k], sum);
            began = false;
#pragma unroll
            for (int q = 0; q < kE; ++q) sum[q] = 0.0f;
        }
    }
    const uint32_t last = live ? s_key[e1] : none;
    const bool goes_on = last != none && s_key[e1 + 1] == last;
    if (goes_on && began) put_head();
    __syncthreads();
    // what the later tiles of the block add to token t, from group q on
    auto add_heads = [&](uint32_t t, int q) {
        for (; q < groups && q * p.R < here && s_key[q * p.R + 1] == t; ++q)
#pragma unroll
            for (int k = 0; k < kE; ++k)
                sum[k] += s_head[k * kBlock + (q << p.lg) + lane];
    };
    if (goes_on && !began) {  // it began in this tile
        add_heads(last, g + 1);
        if (s_key[here + 1] == last) {
            store_cols<PDB_F32, kE>(p.part, (block * 2 + 1) * p.d, c, p.d, sum);
        } else {
            RawCols<GT, kE> old;
            if (ACC) old = load_raw<GT, kE>(p.grad, (int64_t)last * p.ldg, c, p.d);
            put_row<GT, kE>(p.grad, p.ldg, last, c, p.d, p.scale, ACC, old, sum);
        }
    }
    if (g == 0 && opened) {
#pragma unroll
        for (int q = 0; q < kE; ++q) sum[q] = 0.0f;
        add_heads(s_key[0], 0);
        store_cols<PDB_F32, kE>(p.part, block * 2 * p.d, c, p.d, sum);
    }
}

// Tokens that cross the summing blocks' spans: the group of the span where one
// begins adds the later spans' slots to its own, in order, as long as a span's first
// entry holds the token (slots and first entries are read together: waiting for one
// to know whether to read the other would double the trips).  A run of more than
// kOwn spans is added by the whole block, every group each G-th span and then the
// groups' sums pairwise.  Groups are narrow, 8 lanes where rows are not wider than a
// grid, so that a hot token's run is spread over many of them (3M tokens of 32 columns,
// Zipf: 145 us, with 16 lanes of blocks twice as large 151).
constexpr int kJoinBlock = 256, kJoinLg = 3;
template <int GT, int E, bool ACC>
__global__ __launch_bounds__(kJoinBlock) void k_embed_join(GradArgs p) {
    constexpr int kJoinAhead = 32 / E, kOwn = 4 * kJoinAhead;  // slots in flight; four trips
    __shared__ float s_sum[kJoinBlock * E / 2];
    // the groups whose tokens' runs are long, and those tokens
    __shared__ int s_long[kJoinBlock];
    __shared__ uint32_t s_token[kJoinBlock];
    __shared__ int s_count;
    const int lane = threadIdx.x & ((1 << p.lg) - 1);
    const int groups = kJoinBlock >> p.lg, g = threadIdx.x >> p.lg;
    const int64_t span0 = (int64_t)blockIdx.x * groups, span = span0 + g;
    const int64_t c = ((int64_t)blockIdx.y << p.lg | lane) * E;
    const bool live = c < p.d;
    // adds slot 0 of the spans from, from + step, ... below `to`, as long as they
    // begin with t
    auto add_slots = [&](float *sum, uint32_t t, int64_t from, int64_t to, int64_t step) {
        to = min(to, p.sum_blocks);
        for (int64_t q = from; q < to; q += step * kJoinAhead) {
            uint32_t key[kJoinAhead];
            float x[kJoinAhead][E];
#pragma unroll
            for (int k = 0; k < kJoinAhead; ++k) {
                const int64_t at = min(q + k * step, p.sum_blocks - 1);
                key[k] = p.keys[at * p.span];
                load_cols<PDB_F32, E>(p.part, at * 2 * p.d, c, p.d, x[k]);
            }
#pragma unroll
            for (int k = 0; k < kJoinAhead; ++k) {
                if (q + k * step >= to || key[k] != t) return;
#pragma unroll
                for (int e = 0; e < E; ++e) sum[e] += x[k][e];
            }
        }
    };
    if (threadIdx.x == 0) s_count = 0;
    __syncthreads();
    if (span < p.sum_blocks - 1) {
        const int64_t e0 = span * p.span, e1 = e0 + p.span, far = span + 1 + kOwn;
        const uint32_t t = p.keys[e1 - 1], next = p.keys[e1];
        const uint32_t before = e0 > 0 ? p.keys[e0 - 1] : 0xFFFFFFFFu;
        const uint32_t there = far < p.sum_blocks ? p.keys[far * p.span] : 0xFFFFFFFFu;
        // it goes on, and began in this span
        if (t < (uint32_t)p.v && next == t && before != t) {
            if (there == t) {
                if (lane == 0) {
                    const int k = atomicAdd(&s_count, 1);
                    s_long[k] = g;
                    s_token[k] = t;
                }
            } else if (live) {
                RawCols<GT, E> old;
                if (ACC) old = load_raw<GT, E>(p.grad, (int64_t)t * p.ldg, c, p.d);
                float sum[E];
                load_cols<PDB_F32, E>(p.part, (span * 2 + 1) * p.d, c, p.d, sum);
                add_slots(sum, t, span + 1, far, 1);
                put_row<GT, E>(p.grad, p.ldg, t, c, p.d, p.scale, ACC, old, sum);
            }
        }
    }
    __syncthreads();
    const int count = s_count;
    for (int k = 0; k < count; ++k) {
        const int64_t from = span0 + s_long[k];
        const uint32_t t = s_token[k];
        RawCols<GT, E> old;
        if (ACC && g == 0 && live) old = load_raw<GT, E>(p.grad, (int64_t)t * p.ldg, c, p.d);
        float sum[E];
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] = 0.0f;
        if (live) {
            if (g == 0) load_cols<PDB_F32, E>(p.part, (from * 2 + 1) * p.d, c, p.d, sum);
            add_slots(sum, t, from + 1 + g, p.sum_blocks, groups);
        }
        for (int half = groups >> 1; half >= 1; half >>= 1) {
            if (g >= half && g < 2 * half)
#pragma unroll
                for (int e = 0; e < E; ++e)
                    s_sum[e * (kJoinBlock / 2) + threadIdx.x - (half << p.lg)] = sum[e];
            __syncthreads();
            if (g < half)
#pragma unroll
                for (int e = 0; e < E; ++e) sum[e] += s_sum[e * (kJoinBlock / 2) + threadIdx.x];
            __syncthreads();
        }
        if (g == 0 && live)
            put_row<GT, E>(p.grad, p.ldg, t, c, p.d, p.scale, ACC, old, sum);
    }
}

// Few tokens: no sort.  A group per token; the first of equal ones sums them all.
template <int DT, int GT, bool ACC>
__global__ __launch_bounds__(kBlock) void k_embed_direct(GradArgs p) {
    constexpr int kE = Pair<DT, GT>::kE;
    __shared__ int32_t s_tok[kDirect];
    __shared__ unsigned long long s_used;
    const int n = (int)p.n;
    if (threadIdx.x < n) s_tok[threadIdx.x] = read_token(p.tokens, p.index, threadIdx.x, p.v, p.status);
    __syncthreads();
    if ((int64_t)blockIdx.x >= p.sum_blocks) {  // zeros in the rows without tokens
        if (blockIdx.y > 0) return;
        for (int64_t r0 = ((int64_t)blockIdx.x - p.sum_blocks) * kWave; r0 < p.v;
             r0 += p.zero_blocks * kWave) {
            if (threadIdx.x == 0) s_used = 0;
            __syncthreads();
            if (threadIdx.x < n) {
                const int64_t at = s_tok[threadIdx.x] - r0;
                if (s_tok[threadIdx.x] >= 0 && at >= 0 && at < kWave)
                    atomicOr(&s_used, 1ull << at);
            }
            __syncthreads();
            const int64_t rows = p.v - r0;
            const unsigned long long there = rows >= kWave ? ~0ull : (1ull << rows) - 1ull;
            zero_rows<GT>(p.grad, p.ldg, r0, p.d, p.zero_lg, there & ~s_used);
            __syncthreads();
        }
        return;
    }
    // a group's part of its wave, and the tokens compared at a time
    const int lw = min(p.lg, 6), step = 1 << lw;
    const int lane = threadIdx.x & ((1 << p.lg) - 1), in_wave = lane_id() & (step - 1);
    const int first = lane_id() & ~(step - 1);
    const int i = (int)blockIdx.x * (kBlock >> p.lg) + (threadIdx.x >> p.lg);
    const int64_t c = ((int64_t)blockIdx.y << p.lg | lane) * kE;
    const int32_t t = i < n ? s_tok[i] : -1;
    bool mine = t >= 0;
    float sum[kE];
#pragma unroll
    for (int q = 0; q < kE; ++q) sum[q] = 0.0f;
    RawCols<GT, kE> old;
    if (ACC && mine && c < p.d) old = load_raw<GT, kE>(p.grad, (int64_t)t * p.ldg, c, p.d);
    for (int j0 = 0; j0 < n; j0 += step) {
        const bool same = mine && j0 + in_wave < n && s_tok[j0 + in_wave] == t;
        unsigned long long m = __ballot(same) >> first;
        if (step < 64) m &= (1ull << step) - 1ull;
        if (mine && m && j0 + (int)__builtin_ctzll(m) < i) mine = false;  // not the first
        while (mine && m) {
            RawCols<DT, kE> x[kAhead];
            int count = 0;
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                if (!m) break;
                const int j = j0 + (int)__builtin_ctzll(m);
                m &= m - 1;
                if (c < p.d) x[k] = load_raw<DT, kE>(p.dy, (int64_t)j * p.ldy, c, p.d);
                count = k + 1;
            }
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                if (k >= count) break;
                float f[kE];
                unpack_raw<DT, kE>(x[k], f);
#pragma unroll
                for (int q = 0; q < kE; ++q) sum[q] += f[q];
            }
        }
    }
    if (mine && c < p.d) put_row<GT, kE>(p.grad, p.ldg, (uint32_t)t, c, p.d, p.scale, ACC, old, sum);
}

// ----------------------------------------------------------------------------

// Entries per tile.  Enough tiles that n d / R elements, about 2^22, fill the
// card's lanes with one vector each; not fewer than 8, so that few sums cross tiles,
// nor more than a block's tiles have room for in LDS.
inline int tile_rows(int64_t n, int64_t d, int lg) {
    const int groups = kBlock >> lg;
    const int64_t r = (n * d) >> 22;
    return (int)std::min<int64_t>(std::max<int64_t>(r, groups > kStaged / 8 ? kStaged / groups : 8),
                                  std::min(256, kStaged / groups));
}

struct GradWs {
    uint32_t *keys, *kA, *vA, *kB, *vB, *hist, *scan_tmp;
    float *part;
    size_t total;
};
GradWs grad_ws_layout(void *base, int64_t n, int64_t d) {
    GradWs w = {};
    w.total = (size_t)kAlign;  // never none: callers pass one workspace for any n
    if (n <= kDirect) return w;
    char *p = static_cast<char *>(base);
    size_t off = 0;
    auto take = [&](int64_t bytes) {
        char *at = p + off;
        off += (size_t)align_up(bytes);
        return at;
    };
    const int64_t st = cdiv(n, kTile);
    // spans of a block's tiles, for the wider of a lane's shares of a row
    const int lg = lanes_log2(cdiv(std::max<int64_t>(d, 1), 4));
    const int lg8 = lanes_log2(cdiv(std::max<int64_t>(d, 1), 8));
    const int64_t spans = std::max(cdiv(n, (int64_t)tile_rows(n, d, lg) << (8 - lg)),
                                   cdiv(n, (int64_t)tile_rows(n, d, lg8) << (8 - lg8)));
    w.kA = reinterpret_cast<uint32_t *>(take(4 * n));
    w.vA = reinterpret_cast<uint32_t *>(take(4 * n));
    if (n > rank_tokens(0)) {
        if (n > kSortMost) w.keys = reinterpret_cast<uint32_t *>(take(4 * n));
        w.kB = reinterpret_cast<uint32_t *>(take(4 * n));
        w.vB = reinterpret_cast<uint32_t *>(take(4 * n));
        w.hist = reinterpret_cast<uint32_t *>(
            take(4 * std::max<int64_t>(256 * st, kDigits * (kSortTiles + 1))));
        w.scan_tmp = reinterpret_cast<uint32_t *>(take(4 * (int64_t)scan_tmp_elems(256 * st)));
    }
    w.part = reinterpret_cast<float *>(take(spans * 2 * d * 4));
    w.total = off;
    return w;
}

// Counts that every block of the move sums by itself; more go through a scan.
constexpr int64_t kDirectCounts = 1 << 15;

// The tokens in order (padding as v, last) and their positions.
int sort_tokens(const GradWs &w, const void *tokens, int index, int64_t n, int64_t v,
                int32_t *status, uint32_t **keys, uint32_t **vals, hipStream_t s) {
    int bits = 1;
    while (((int64_t)1 << bits) <= v) ++bits;
    *keys = w.kA;
    *vals = w.vA;
    if (n <= rank_tokens(bits)) {
        k_token_rank<<<(unsigned)cdiv(n, kWave), kSortBlock, 0, s>>>(tokens, index, (int)n, v, w.kA,
                                                                     w.vA, status);
        PDB_LAUNCHED();
        return PDB_OK;
    }
    if (n > kSortMost) {
        k_token_keys<<<grid_for(n, kBlock, 4096), kBlock, 0, s>>>(tokens, index, n, v, w.keys,
                                                                  status);
        PDB_LAUNCHED();
        PDB_HIP(radix_sort_pairs(w.keys, nullptr, n, bits, w.kA, w.vA, w.kB, w.vB, w.hist,
                                 w.scan_tmp, keys, vals, s));
        return PDB_OK;
    }
    // about 256 tiles, one a compute unit (1M tokens of 64 columns: 84 us; with 128
    // tiles 92, with 512 90)
    const int items = (int)std::min<int64_t>(kSortItems, cdiv(n, 256 * kSortBlock));
    const int tiles = (int)cdiv(n, (int64_t)items * kSortBlock);
    const int passes = (bits + kDigitBits - 1) / kDigitBits, step = (bits + passes - 1) / passes;
    SortIn in = {tokens, index, v, status, nullptr, nullptr, n, items, 0, 0, tiles};
    for (; in.shift < bits; in.shift += step) {
        const int nb = in.nb = std::min(step, bits - in.shift);
        const bool first = in.shift == 0;
        if (first)
            k_token_sort_count<true><<<tiles, kSortBlock, 0, s>>>(in, w.hist);
        else
            k_token_sort_count<false><<<tiles, kSortBlock, 0, s>>>(in, w.hist);
        PDB_LAUNCHED();
        const bool scan = nb >= 6 && (int64_t)tiles << nb > kDirectCounts;
        if (scan) {
            k_token_sort_scan<<<(1 << nb) / kScanDigits, kSortBlock, 0, s>>>(w.hist, tiles, nb);
            PDB_LAUNCHED();
        }
        uint32_t *tk = in.keys == w.kA ? w.kB : w.kA, *tv = in.keys == w.kA ? w.vB : w.vA;
        if (nb <= 8 && first)
            k_token_sort_move<8, true><<<tiles, kSortBlock, 0, s>>>(in, w.hist, scan, tk, tv);
        else if (nb <= 8)
            k_token_sort_move<8, false><<<tiles, kSortBlock, 0, s>>>(in, w.hist, scan, tk, tv);
        else if (first)
            k_token_sort_move<kDigitBits, true><<<tiles, kSortBlock, 0, s>>>(in, w.hist, scan, tk,
                                                                             tv);
        else
            k_token_sort_move<kDigitBits, false><<<tiles, kSortBlock, 0, s>>>(in, w.hist, scan, tk,
                                                                              tv);
        PDB_LAUNCHED();
        in.keys = *keys = tk;
        in.vals = *vals = tv;
    }
    return PDB_OK;
}

template <int DT, int GT, bool ACC>
int embed_grad(GradArgs p, const GradWs &w, hipStream_t s) {
    constexpr int kE = Pair<DT, GT>::kE;
    const int64_t vectors = cdiv(p.d, kE);
    p.lg = lanes_log2(vectors);
    p.zero_lg = lanes_log2(cdiv(p.d, Elem<GT>::kVec));
    p.zero_blocks = ACC ? 0 : std::min<int64_t>(cdiv(p.v, kWave), 1 << 18);
    const int64_t slices = cdiv(vectors, 1 << p.lg), per = kBlock >> p.lg;
    if (slices > 65535) return PDB_ERR_UNSUPPORTED;
    if (p.n <= kDirect) {
        p.sum_blocks = cdiv(p.n, per);
        const dim3 grid((unsigned)(p.sum_blocks + p.zero_blocks), (unsigned)slices);
        k_embed_direct<DT, GT, ACC><<<grid, kBlock, 0, s>>>(p);
        PDB_LAUNCHED();
        return PDB_OK;
    }
    uint32_t *keys, *vals;
    const int rc = sort_tokens(w, p.tokens, p.index, p.n, p.v, p.status, &keys, &vals, s);
    if (rc != PDB_OK) return rc;
    p.keys = keys;
    p.vals = vals;
    p.part = w.part;
    p.R = tile_rows(p.n, p.d, p.lg);
    p.span = per * p.R;
    p.sum_blocks = cdiv(p.n, p.span);
    const dim3 grid((unsigned)(p.sum_blocks + p.zero_blocks), (unsigned)slices);
    k_embed_tiles<DT, GT, ACC><<<grid, kBlock, 0, s>>>(p);
    PDB_LAUNCHED();
    if (p.sum_blocks == 1) return PDB_OK;
    const int lg = p.lg;
    p.lg = std::min(lg, kJoinLg);
    while (p.lg < lg && cdiv(vectors, 1 << p.lg) > 65535) ++p.lg;
    const dim3 join((unsigned)cdiv(p.sum_blocks, kJoinBlock >> p.lg),
                    (unsigned)cdiv(vectors, 1 << p.lg));
    k_embed_join<GT, kE, ACC><<<join, kJoinBlock, 0, s>>>(p);
    PDB_LAUNCHED();
    return PDB_OK;
}

}  // namespace
}  // namespace pdbk

using namespace pdbk;

extern "C" int pdb_embed_lookup(const void *table, int dtype, int64_t ld, int64_t v, int64_t d,
                                const void *tokens, int index, int64_t n, float scale, void *out,
                                int out_dtype, int64_t ldo, int32_t *status, hipStream_t s) {
    int rc = check_matrix(table, dtype, ld, v, d);
    if (rc == PDB_OK) rc = check_tokens(tokens, index, n);
    if (rc == PDB_OK) rc = check_matrix(out, out_dtype, ldo, n, d);
    if (rc != PDB_OK) return rc;
    if (n == 0 || d == 0) return PDB_OK;
    return with_dtype(dtype, [&](auto tt) -> int {
        return with_dtype(out_dtype, [&](auto ot) -> int {
            constexpr int TT = decltype(tt)::value, OT = decltype(ot)::value;
            const int64_t vectors = cdiv(d, Pair<TT, OT>::kE);
            const int lg = lanes_log2(vectors);
            const dim3 grid((unsigned)grid_for(n, kBlock >> lg), (unsigned)cdiv(vectors, 1 << lg));
            if (cdiv(vectors, 1 << lg) > 65535) return PDB_ERR_UNSUPPORTED;
            k_embed_lookup<TT, OT><<<grid, kBlock, 0, s>>>(table, ld, v, d, tokens, index, n, scale,
                                                           out, ldo, lg, status);
            PDB_LAUNCHED();
            return PDB_OK;
        });
    });
}

extern "C" int pdb_embed_grad_workspace_bytes(int64_t n, int64_t v, int64_t d, size_t *bytes) {
    if (!bytes || n < 0 || v < 0 || d < 0) return PDB_ERR_INVALID_ARG;
    if (n > INT32_MAX || v > INT32_MAX || d > INT32_MAX) return PDB_ERR_UNSUPPORTED;
    *bytes = grad_ws_layout(nullptr, n, d).total;
    return PDB_OK;
}

extern "C" int pdb_embed_grad(const void *dy, int dtype, int64_t ldy, const void *tokens, int index,
                              int64_t n, void *grad, int grad_dtype, int64_t ldg, int64_t v,
                              int64_t d, float scale, int accumulate, int32_t *status, void *ws,
                              size_t ws_bytes, hipStream_t s) {
    int rc = check_matrix(dy, dtype, ldy, n, d);
    if (rc == PDB_OK) rc = check_tokens(tokens, index, n);
    if (rc == PDB_OK) rc = check_matrix(grad, grad_dtype, ldg, v, d);
    if (rc != PDB_OK) return rc;
    if (accumulate != 0 && accumulate != 1) return PDB_ERR_INVALID_ARG;
    if (v == 0 || d == 0 || (n == 0 && accumulate)) return PDB_OK;
    const GradWs w = grad_ws_layout(ws, n, d);
    if (!ws || ws_bytes < w.total) return PDB_ERR_WORKSPACE;
    GradArgs p = {};
    p.dy = dy;
    p.ldy = ldy;
    p.tokens = tokens;
    p.index = index;
    p.n = n;
    p.d = d;
    p.v = v;
    p.scale = scale;
    p.grad = grad;
    p.ldg = ldg;
    p.status = status;
    return with_dtype(grad_dtype, [&](auto gt) -> int {
        return with_dtype(dtype, [&](auto dt) -> int {
            constexpr int DT = decltype(dt)::value, GT = decltype(gt)::value;
            return accumulate ? embed_grad<DT, GT, true>(p, w, s)
                              : embed_grad<DT, GT, false>(p, w, s);
        });
    });
}
