// The gated recurrence h_t = f_t h_{t-1} + (1 - f_t) x_t over packed sequences and its
// backward pass (gfx950, wave64).
//
// A row acts on the state as the map h -> a h + c, and maps compose: (a1, c1) then
// (a2, c2) is (a2 a1, a2 c1 + c2).  The rows are cut into tiles, whatever sequences they
// hold, and the channels into strips of 128 bytes of a row: a block has a tile of a strip
// in registers, some rows of a vector of channels to a thread, and reads it once.  The
// threads' maps are joined through LDS, the tiles' through the workspace while the blocks
// run: each publishes its map, waits for the state behind the tile REACH before and
// applies the maps between, in thirds (so the sums do not depend on who was first), and
// publishes the state behind its own.  Tiles are dealt by a counter, so a block waits
// only for blocks that have begun.  A row that begins a sequence takes its first state in
// place of what enters: its map is "cut", a = -0 (gates are never negative, so products
// and selects keep the mark), and nothing of another sequence passes it, not even a NaN.
//
// The bound is the bytes.  131,072 rows of 1,024 channels in 16 bits take 168 us, 4.8 TB/s
// (in launches that read the rows twice: 504), the gradient's 65,536 158 us, 4.2 TB/s.
// What stands before the bytes:
// * waiting: for a tile's loads, its join, and the chain.  Without the chain's waits the
//   same rows took as long, but 32,768 of 2,048 channels 95 us where they took 102 (99 now),
//   since a late tile delays those behind it.  Tiles of half the rows took a third longer, the
//   latencies being a tile's whatever its size.
// * the vector unit, 13 operations and two transcendental ones an element and pass: gates
//   that cost nothing would have saved 10 us of the 102.
// * registers: two numbers an element (the map behind each row) keep the forward pass of 16
//   bits at two blocks a unit.  Loading the next tile's rows under the chain, or keeping
//   x and gate and computing gates twice, for three blocks, gained nothing.
#include "pdb_vec.h"
#include "pdb_softmax.h"
#include "../../include/pdb_layers.h"

namespace pdbk {
namespace {

constexpr int kStripLanes = 8;                   // lanes over 128 bytes of a row
constexpr int kRowLanes = kBlock / kStripLanes;  // 32

// Rows of a thread: two numbers an element, in the backward four.  (In the backward of 16
// bits four rows spill 15 registers at three blocks a unit, and take 161 us; at two blocks,
// without spills, 178; eight rows 237.)
template <int DT, bool BACK>
struct Shape {
    static constexpr int V = Elem<DT>::kVec;
    static constexpr int kRows = BACK ? 4 : 8;
    static constexpr int kTileRows = kRowLanes * kRows;
    static constexpr int kSlots = kStripLanes * V;  // channels of a strip
    static_assert(kTileRows % PDB_SCAN_MARK == 0 && PDB_SCAN_MARK % kRows == 0,
                  "a mark is at the first row of some thread");
};

struct Map {
    float a, c;
};
__device__ __forceinline__ bool is_cut(float a) { return __float_as_uint(a) == 0x80000000u; }
__device__ __forceinline__ float apply(Map m, float h) {
    return is_cut(m.a) ? m.c : __builtin_fmaf(m.a, h, m.c);
}
// first, then second
__device__ __forceinline__ Map then(Map first, Map second) {
    return is_cut(second.a) ? second : Map{second.a * first.a, __builtin_fmaf(second.a, first.c, second.c)};
}

// f = 1 / (1 + e^-g) and k = 1 - f, each with its own relative accuracy at either end.
// From t = 2^126 on (g below -87.3) 1 / (1 + t) is no normal number and the reciprocal
// gives 0: f is 0 there, to within 2^-126, but k is 1.  So k = t f is taken with an f of at
// least 2^-126, which leaves it within its rounding below t = 2^102 and makes it 1 or more,
// up to infinity, where f was 0; in between the product is 1 but for rounding.
struct Gate {
    float f, k;
};
__device__ __forceinline__ Gate gate_of(float g) {
    const float t = exp2_raw(g * -kLog2e);
    const float f = __builtin_amdgcn_rcpf(1.0f + t);
    // (the minimum that keeps what is no number: neither is k then)
    return {f, __builtin_elementwise_minimum(t * fmaxf(f, 0x1p-126f), 1.0f)};
}

struct Scan {
    const void *x, *gate, *dy;
    int64_t ldx, ldg, lddy;
    int64_t n, d;
    const int32_t *starts;
    int32_t b, len;  // len: rows of every sequence where starts is NULL
    const float *h0;
    float *state;  // the backward's dh0
    const float *d_state;
    void *y, *dgate;
    int64_t ldy, lddg;
    float *marks;
    const float *marks_in;
    int32_t *status;
    int32_t tiles, strips;
    // in the order of the chain (the backward's from the last tile on); NULL of one
    // tile and one launch
    unsigned long long *total;  // [tiles][strips][slots]: the tiles' maps
    uint32_t *leave;            // the same: the states behind them
    uint32_t *ticket;           // [0]: tiles dealt; [1]: 0 once a wait has lasted too long
    int32_t *first;             // [tiles]: what first_edge says of each
};

// ----------------------------------------------------------------------------
// rows and sequences

// A tile's rows of sequences, [lo, hi), and which sequences begin and end with its rows
// (-1 elsewhere).
template <int N>
struct Edges {
    int32_t begin[N], end[N];
    int64_t lo, hi;
    uint32_t dealt;  // the tile's place in the chain's order
    int32_t first;
};

// How many of starts[0 .. b] lie below `row`: a search in 64 parts, the same in every
// lane (any values: at most log64 b steps, all indexes inside).
__device__ __forceinline__ int starts_below(const int32_t *starts, int64_t count, int64_t row) {
    int64_t lo = 0, len = count;
    while (len > 0) {
        const int64_t step = (len + kWave - 1) / kWave, at = lo + lane_id() * step;
        const bool below = at < lo + len && starts[at] < row;
        const int c = __popcll(__ballot(below));
        if (c == 0) return (int)lo;
        const int64_t from = lo + (int64_t)(c - 1) * step + 1;
        len = min(step - 1, lo + len - from);
        lo = from;
    }
    return (int)lo;
}

// A strip's channels are in slots: channel q of the vector of lane cl in slot
// q kStripLanes + cl, so that neighbouring lanes' are neighbours in LDS (vector by vector
// the threads' maps met in the same banks: a third of the backward's time).
__device__ __forceinline__ constexpr int slot_at(int q, int cl) { return q * kStripLanes + cl; }

// The channel of a slot of a strip, -1 of none; `own`: -1 also where it is the vector's
// before, with which the row's last one shares channels.
template <int V, bool WIDE>
__device__ __forceinline__ int64_t channel_of(const Scan &p, int strip, int slot, bool own) {
    const int64_t c = ((int64_t)strip * kStripLanes + slot % kStripLanes) * V;
    const int64_t at = (WIDE ? min(c, p.d - V) : c) + slot / kStripLanes;
    return c < p.d && at < p.d && !(own && at < c) ? at : -1;
}

// kPlain if the rows [r0, r1) neither begin nor end a sequence and all belong to one;
// else the first of the offsets that lies at r0 or behind (0 without offsets).  By one
// wave.
constexpr int32_t kPlain = -1;
__device__ __forceinline__ int32_t first_edge(const Scan &p, int64_t r0, int64_t r1, bool last_tile) {
    if (!p.starts) {
        const uint32_t o = (uint32_t)r0 % (uint32_t)max(p.len, 1);
        return r1 <= p.n && o > 0 && o + (r1 - r0) < (uint32_t)p.len ? kPlain : 0;
    }
    const int32_t *starts = p.starts;
    const int64_t lo = starts[0], hi = starts[p.b];
    const int at = starts_below(starts, (int64_t)p.b + 1, r0 + (r0 == 0 ? INT32_MIN : 0));
    const int64_t next = at <= p.b ? starts[at] : INT64_MAX;
    // (a tile that ends with a sequence's last row has an edge: the offset is r1)
    return r0 >= lo && r1 <= min(hi, p.n) && !last_tile && next > r1 ? kPlain : at;
}

// Fills `e` for the rows from r0 on, by one wave; first: what first_edge gave.  Empty
// sequences at the tile's rows (the last tile: or behind) get their states, those of
// `from`.
template <int V, bool WIDE, int N>
__device__ __forceinline__ void find_edges(const Scan &p, int64_t r0, bool last_tile, int strip,
                                           const float *from, int32_t first, Edges<N> &e) {
    const int l = lane_id();
    for (int i = l; i < N; i += kWave) e.begin[i] = e.end[i] = -1;
    Team<1>::sync();
    int64_t lo = 0, hi = p.n;
    const int64_t r1 = r0 + N;
    if (!p.starts) {
        for (int i = l; i < N; i += kWave) {
            const int64_t r = r0 + i;
            if (r >= p.n) break;
            const uint32_t s = (uint32_t)r / (uint32_t)p.len, o = (uint32_t)r - s * (uint32_t)p.len;
            if (o == 0) e.begin[i] = (int)s;
            if (o == (uint32_t)p.len - 1) e.end[i] = (int)s;
        }
    } else {
        const int32_t *starts = p.starts;
        // The first few offsets by scalar loads, which do not wait behind the tile's rows.
        // (Their order is not relied on: what lies outside the tile is left out.)
        const auto *at_once = (const __attribute__((address_space(4))) int32_t *)starts;
        constexpr int kFew = 4;
        const int64_t j1 = __builtin_amdgcn_readfirstlane(first);
        int64_t few[kFew + 2];  // offsets j1 - 1 .. j1 + kFew
#pragma unroll
        for (int i = 0; i < kFew + 2; ++i) {
            const int64_t j = j1 - 1 + i;
            few[i] = j < 0 ? INT64_MIN : j > p.b ? INT64_MAX : (int64_t)at_once[j];
        }
        lo = max((int64_t)at_once[0], (int64_t)0);
        hi = min((int64_t)at_once[p.b], p.n);
        bool done = false;
#pragma unroll
        for (int i = 1; i <= kFew; ++i) {
            const int64_t j = j1 - 1 + i, at = few[i], next = few[i + 1], before = few[i - 1];
            done |= j > p.b || at > r1;
            // empty sequences have states to write: below
            if (!done && j < p.b && next <= at) break;
            if (!done && l == 0) {
                if (j < p.b && at >= r0 && at < r1) e.begin[at - r0] = (int)j;
                if (j > 0 && before < at && at > r0) e.end[at - 1 - r0] = (int)j - 1;
            }
        }
        for (int64_t j0 = first; !done; j0 += kWave) {
            const int64_t j = j0 + l;
            const bool have = j <= p.b;
            const int64_t at = have ? starts[j] : INT64_MAX;
            const int64_t next = j < p.b ? starts[j + 1] : INT64_MAX;
            const int64_t before = have && j > 0 ? starts[j - 1] : INT64_MIN;
            if (have && at <= r1) {
                if (j < p.b && at < next && at >= r0 && at < r1) e.begin[at - r0] = (int)j;
                if (j > 0 && before < at && at > r0) e.end[at - 1 - r0] = (int)j - 1;
            }
            const bool none = have && j < p.b && next <= at && (at < r1 || last_tile);
            for (unsigned long long m = p.state ? __ballot(none) : 0ull; m; m &= m - 1) {
                const int64_t i = j0 + __ffsll(m) - 1;  // rare: a channel to a lane
                const int64_t c = l < kStripLanes * V ? channel_of<V, WIDE>(p, strip, l, true) : -1;
                if (c >= 0)
                    p.state[i * p.d + c] = from ? from[i * p.d + c] : 0.0f;
            }
            if (!__any(have && at <= r1)) break;
        }
    }
    if (l == 0) {
        e.lo = lo;
        e.hi = hi;
    }
}

// Whether a wave's rows of a tile have no edges and are all of sequences.
template <int N>
__device__ __forceinline__ bool plain_wave(const Edges<N> &e, int64_t r0, int wave) {
    constexpr int kOf = N / (kBlock / kWave);
    static_assert(kOf <= kWave, "a row to a lane");
    const int i = wave * kOf + lane_id() % kOf;
    const bool edge = e.begin[i] >= 0 || e.end[i] >= 0 || r0 + i < e.lo || r0 + i >= e.hi;
    return !__any(edge);
}

// Offsets that descend or leave 0 .. n, a share of them to a block.
__device__ __forceinline__ void check_starts(const Scan &p) {
    if (!p.status || !p.starts) return;
    for (int64_t j = (int64_t)blockIdx.x * kBlock + threadIdx.x; j <= p.b;
         j += (int64_t)gridDim.x * kBlock) {
        const int32_t at = p.starts[j];
        if (at < 0 || at > p.n || (j > 0 && p.starts[j - 1] > at)) *p.status = PDB_ERR_INVALID_ARG;
    }
}

// A thread's vector of a row.
template <int DT, bool WIDE>
__device__ __forceinline__ u32x4 load_vec(const void *m, int64_t ld, int64_t row, int64_t c0,
                                          int64_t d) {
    const char *at = elem_at<DT>(m, row * ld + c0);
    if constexpr (WIDE) {
        return load16(at);
    } else {
        float x[Elem<DT>::kVec];
#pragma unroll
        for (int q = 0; q < Elem<DT>::kVec; ++q) x[q] = q < d ? load1<DT>(at, q) : 0.0f;
        return pack<DT>(x);
    }
}
// Only from element `own` on: a row's last vector may share channels with the one before.
template <int DT, bool WIDE>
__device__ __forceinline__ void store_vec(void *m, int64_t ld, int64_t row, int64_t c0, int64_t d,
                                          int own, const float *x) {
    char *at = elem_at<DT>(m, row * ld + c0);
    if (WIDE && own == 0) {
        store16(at, pack<DT>(x));
    } else {
#pragma unroll
        for (int q = 0; q < Elem<DT>::kVec; ++q)
            if (q >= own && (WIDE || q < d)) store1<DT>(at, q, x[q]);
    }
}
// V floats of row i of a b x d (or marks) array without gaps, zeros of NULL
template <int V, bool WIDE>
__device__ __forceinline__ void load_row(const float *m, int64_t i, int64_t c0, int64_t d, float *x) {
#pragma unroll
    for (int q = 0; q < V; ++q) x[q] = m && (WIDE || q < d) ? m[i * d + c0 + q] : 0.0f;
}
template <int V, bool WIDE>
__device__ __forceinline__ void store_row(float *m, int64_t i, int64_t c0, int64_t d, int own,
                                          const float *x) {
#pragma unroll
    for (int q = 0; q < V; ++q)
        if (q >= own && (WIDE || q < d)) m[i * d + c0 + q] = x[q];
}

// ----------------------------------------------------------------------------
// tiles

// Where a block and a thread are.
template <int DT, bool WIDE, bool BACK>
struct Place {
    static constexpr int V = Elem<DT>::kVec, kRows = Shape<DT, BACK>::kRows;
    int turn, tile, strip, rl, cl, own;  // turn: the tile's place in the chain
    int64_t r0, row, c0;
    bool act;
    __device__ __forceinline__ Place(const Scan &p, uint32_t w) {
        turn = (int)(w / (uint32_t)p.strips);
        strip = (int)(w - (uint32_t)turn * (uint32_t)p.strips);
        tile = BACK ? p.tiles - 1 - turn : turn;
        rl = threadIdx.x / kStripLanes;
        cl = threadIdx.x % kStripLanes;
        r0 = (int64_t)tile * Shape<DT, BACK>::kTileRows;
        row = r0 + rl * kRows;
        // the last vector ends with the row: it may share channels with the one before,
        // which has them (the states may be written over h0)
        const int64_t c = ((int64_t)strip * kStripLanes + cl) * V;
        act = c < p.d;
        c0 = WIDE ? min(c, p.d - V) : c;
        own = (int)(c - c0);
    }
};

// A thread's vectors of its rows of a matrix; zeros behind row n.
template <int DT, bool WIDE, int R>
__device__ __forceinline__ void load_rows(const Scan &p, const void *m, int64_t ld, int64_t row,
                                          int64_t c0, bool act, u32x4 (&raw)[R]) {
    if (act && row + R <= p.n) {
#pragma unroll
        for (int r = 0; r < R; ++r) raw[r] = load_vec<DT, WIDE>(m, ld, row + r, c0, p.d);
    } else {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            raw[r] = u32x4{0, 0, 0, 0};
            if (act && row + r < p.n) raw[r] = load_vec<DT, WIDE>(m, ld, row + r, c0, p.d);
        }
    }
}

// The slot of a lane of a wave (strips of 32-bit channels: of two lanes).
template <int V>
__device__ __forceinline__ int slot_of() {
    return lane_id() & (kStripLanes * V - 1);
}

// The threads' maps of a tile, and what enters each thread's rows: each wave joins its
// own row lanes, a slot to a lane, in row order or (BACK) from the last to the first.
constexpr int kWaves = kBlock / kWave, kWaveRows = kRowLanes / kWaves;
template <int V, bool BACK>
struct Joint {
    static constexpr int kSlots = kStripLanes * V;
    Map part[kRowLanes][kSlots + kStripLanes];  // (rows a vector apart in the banks)
    Map wave[kWaves][kSlots];
    // the i-th row lane of a wave, and the i-th wave, in order
    static __device__ __forceinline__ int lane_at(int wave, int i) {
        return wave * kWaveRows + (BACK ? kWaveRows - 1 - i : i);
    }
    static __device__ __forceinline__ int wave_at(int i) { return BACK ? kWaves - 1 - i : i; }

    __device__ __forceinline__ void put(int rl, int cl, const float *a, const float *c) {
#pragma unroll
        for (int q = 0; q < V; ++q) part[rl][slot_at(q, cl)] = Map{a[q], c[q]};
    }
    // after the wave's put
    __device__ __forceinline__ void join(int w) {
        Team<1>::sync();
        const int slot = slot_of<V>();
        Map m = part[lane_at(w, 0)][slot];
#pragma unroll
        for (int i = 1; i < kWaveRows; ++i) m = then(m, part[lane_at(w, i)][slot]);
        wave[w][slot] = m;
    }
    // after all waves' join
    __device__ __forceinline__ Map total() const {
        const int slot = slot_of<V>();
        Map m = wave[wave_at(0)][slot];
#pragma unroll
        for (int i = 1; i < kWaves; ++i) m = then(m, wave[wave_at(i)][slot]);
        return m;
    }
    // h enters the tile: what enters each row lane of the wave, in the place of its map
    __device__ __forceinline__ void spread(int w, float h) {
        const int slot = slot_of<V>();
#pragma unroll
        for (int i = 0; i < kWaves - 1; ++i) {
            if (wave_at(i) == w) break;
            h = apply(wave[wave_at(i)][slot], h);
        }
#pragma unroll
        for (int i = 0; i < kWaveRows; ++i) {
            const int r = lane_at(w, i);
            const Map m = part[r][slot];
            part[r][slot].c = h;
            h = apply(m, h);
        }
        Team<1>::sync();
    }
    __device__ __forceinline__ void get(int rl, int cl, float *h) const {
#pragma unroll
        for (int q = 0; q < V; ++q) h[q] = part[rl][slot_at(q, cl)].c;
    }
};

// ----------------------------------------------------------------------------
// the chain over tiles

// A tile for the block, by one wave: its place in the chain's order.
__device__ __forceinline__ uint32_t deal(const Scan &p) {
    uint32_t w = blockIdx.x;
    if (p.ticket) {
        if (lane_id() == 0)
            w = __hip_atomic_fetch_add(p.ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        w = __builtin_amdgcn_readfirstlane(w);
    }
    return w;
}

// Tiles that a hop of the chain passes, each of them a map that the block fetches: of few
// strips more, where the chain is all that takes time (131,072 rows of 16 bits: of 64
// channels 40 us with 16, 26 with 49; of 128 43 and 35; of 256 56 and 59; of 1,024 168 and
// 182.  The gradient of 65,536 rows: of 64 channels 48 and 28, of 256 66 and 59, of 512 92
// and 103).
constexpr int kReach = 16, kFarReach = 49;
constexpr int64_t kFewStrips = 2, kFewStripsBack = 4;
constexpr int64_t kPatience = 2000000000;  // ticks of the 100 MHz clock: 20 s
constexpr int64_t kUneasy = 100000;       // 1 ms

// What a tile's place and edges are found by comes from the workspace.  Where something
// else has written there nothing promises its values, so neither is taken further than the
// matrices and offsets reach: a place behind the last tile ends the block, with a status,
// rows behind n are never taken as rows without edges, and no offset is before the first;
// one wave reads them, so that the block's waves take one path.
__device__ __forceinline__ bool on_grid(const Scan &p, uint32_t dealt) {
    if (dealt < (uint32_t)p.tiles * (uint32_t)p.strips) return true;
    if (p.status && threadIdx.x == 0) *p.status = PDB_ERR_DEVICE;
    return false;
}
__device__ __forceinline__ int32_t first_of(const Scan &p, int tile, int64_t r0, int rows) {
    const int32_t first = p.first[tile];
    return first == kPlain && r0 + rows <= p.n ? kPlain : max(first, 0);
}

template <typename T>
__device__ __forceinline__ T peek(const T *at) {
    return __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <typename T>
__device__ __forceinline__ void post(T *at, T word) {
    __hip_atomic_store(at, word, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// The words of the chain carry their own readiness: all ones is "not yet" (a NaN that
// no arithmetic here gives; one that comes from outside is replaced by another).
__device__ __forceinline__ unsigned long long word_of(Map m) {
    const unsigned long long w =
        (unsigned long long)__float_as_uint(m.a) << 32 | __float_as_uint(m.c);
    return w == ~0ull ? 0x7FC000007FC00000ull : w;
}
__device__ __forceinline__ Map map_of(unsigned long long w) {
    return {__uint_as_float((uint32_t)(w >> 32)), __uint_as_float((uint32_t)w)};
}
__device__ __forceinline__ uint32_t word_of(float h) {
    return __float_as_uint(h) == ~0u ? 0x7FC00000u : __float_as_uint(h);
}

// Whether a wait since t0 has lasted too long, here or in any other block: a chain whose
// words were overwritten ends, in all its blocks.
__device__ __forceinline__ bool give_up(const Scan &p, int64_t t0) {
    const int64_t waited = now_ticks() - t0;
    if (waited < kUneasy) return false;
    if (peek(p.ticket + 1) == 0u) return true;
    if (waited < kPatience) return false;
    post(p.ticket + 1, 0u);
    return true;
}

// Where a lane's words of the chain are; -1 of a lane without a slot.
template <int V>
struct Link {
    int64_t slots, at;
    bool mine;
    __device__ __forceinline__ Link(const Scan &p, int turn, int strip) {
        constexpr int kSlots = kStripLanes * V;
        slots = (int64_t)p.strips * kSlots;
        at = (int64_t)turn * slots + (int64_t)strip * kSlots + slot_of<V>();
        mine = lane_id() < kSlots;
    }
};

// Whether what leaves a tile does not hang on what enters it, in any slot of the strip: the
// state behind it is published with its map then.  (Not slot by slot: a gate that is no
// number hides a cut, and each slot is published once, here or in chain_end.)
__device__ __forceinline__ bool all_cut(Map m) { return __all(is_cut(m.a)); }

// What the waves of a block fetch of the chain: the maps of the REACH - 1 tiles before
// its own, a third of them to each of three waves, which makes one map of them.
template <int V, int REACH>
struct Fetched {
    static constexpr int kEach = (REACH - 1) / 3;
    static_assert(3 * kEach == REACH - 1, "thirds");
    Map map[3][kStripLanes * V];  // the nearest third first
    float leave[kStripLanes * V];
    int late, cut;  // a wait given up; a cut among the maps, so that no state is waited for
};
template <int V, int REACH>
__device__ __forceinline__ void fetch_maps(const Scan &p, int turn, int strip, int third,
                                           Fetched<V, REACH> &f) {
    constexpr int kEach = Fetched<V, REACH>::kEach;
    if (!p.ticket) return;
    const Link<V> l(p, turn, strip);
    const int64_t t0 = now_ticks();
    unsigned long long w[kEach];
    while (true) {
        bool missing = false;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            // (maps of no tile are neither asked for nor applied)
            const int back = third * kEach + j + 1;
            w[j] = back <= turn ? peek(p.total + (l.at - back * l.slots)) : 0ull;
        }
#pragma unroll
        for (int j = 0; j < kEach; ++j) missing |= w[j] == ~0ull;
        if (!__any(missing)) break;
        if (__any(give_up(p, t0))) {
            f.late = 1;
            break;
        }
        __builtin_amdgcn_s_sleep(1);
    }
    Map m = {1.0f, 0.0f};
#pragma unroll
    for (int j = kEach - 1; j >= 0; --j)
        if (third * kEach + j < turn) m = then(m, map_of(w[j]));
    f.map[third][slot_of<V>()] = m;
    // (a tile with a sequence's beginning has cuts in all its slots)
    if (all_cut(m)) __hip_atomic_store(&f.cut, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
}

// The block's own map, and the state behind the tile REACH before.
template <int V, int REACH>
__device__ __forceinline__ void chain_wait(const Scan &p, int turn, int strip, Map m,
                                           Fetched<V, REACH> &f) {
    if (!p.ticket) return;
    const Link<V> l(p, turn, strip);
    if (turn < p.tiles - 1 && l.mine) post(p.total + l.at, word_of(m));
    if (all_cut(m) && turn + REACH < p.tiles && l.mine) post(p.leave + l.at, word_of(m.c));
    uint32_t h = 0;
    if (turn >= REACH) {
        const int64_t t0 = now_ticks();
        while (true) {
            h = peek(p.leave + (l.at - REACH * l.slots));
            if (!__any(h == ~0u)) break;
            if (__hip_atomic_load(&f.cut, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP)) break;
            if (__any(give_up(p, t0))) {
                f.late = 1;
                break;
            }
            __builtin_amdgcn_s_sleep(1);
        }
    }
    f.leave[slot_of<V>()] = __uint_as_float(h);
}
// What enters the tile, from both, by every wave; `first`, one of them, publishes the state
// behind the tile, whose map is m.  A wait that was given up ends with NaN and a status.
template <int V, int REACH>
__device__ __forceinline__ float chain_end(const Scan &p, int turn, int strip, Map m, bool first,
                                           const Fetched<V, REACH> &f) {
    if (!p.ticket) return 0.0f;
    float h = f.leave[slot_of<V>()];
#pragma unroll
    for (int j = 2; j >= 0; --j) h = apply(f.map[j][slot_of<V>()], h);
    if (f.late) {
        h = kNan;  // seen by whoever uses the result
        if (p.status) *p.status = PDB_ERR_DEVICE;
    }
    const Link<V> l(p, turn, strip);
    if (first && !all_cut(m) && turn + REACH < p.tiles && l.mine) post(p.leave + l.at, word_of(apply(m, h)));
    return h;
}

// ----------------------------------------------------------------------------
// the kernels

template <typename F>
__device__ __forceinline__ void either(bool plain, F f) {
    if (plain)
        f(std::true_type());
    else
        f(std::false_type());
}

template <int DT, bool WIDE, int REACH>
__global__ __launch_bounds__(kBlock, 2) void k_scan(Scan p) {
    using S = Shape<DT, false>;
    using At = Place<DT, WIDE, false>;
    constexpr int V = S::V, R = S::kRows;
    __shared__ Joint<V, false> s;
    __shared__ Edges<S::kTileRows> e;
    __shared__ Fetched<V, REACH> fetched;
    const int wave = __builtin_amdgcn_readfirstlane(wave_in_block());
    check_starts(p);
    if (wave == 0) {
        const uint32_t w = deal(p);
        const int32_t first = p.ticket ? 0 : first_edge(p, 0, S::kTileRows, true);
        if (lane_id() == 0) {
            e.dealt = w;
            e.first = first;
            fetched.late = fetched.cut = 0;
        }
    }
    __syncthreads();
    const uint32_t dealt = __builtin_amdgcn_readfirstlane(e.dealt);
    if (!on_grid(p, dealt)) return;
    const At at(p, dealt);
    int32_t first = 0;
    if (p.ticket && wave == 0) first = first_of(p, at.tile, at.r0, S::kTileRows);
    u32x4 rx[R], rg[R];
    load_rows<DT, WIDE>(p, p.gate, p.ldg, at.row, at.c0, at.act, rg);
    load_rows<DT, WIDE>(p, p.x, p.ldx, at.row, at.c0, at.act, rx);
    if (p.ticket) {
        if (threadIdx.x == 0) e.first = first;
        Team<kWaves>::sync_lds();
    }
    first = __builtin_amdgcn_readfirstlane(e.first);
    bool plain = first == kPlain;
    if (!plain) {
        if (wave == 1)
            find_edges<V, WIDE>(p, at.r0, at.tile == p.tiles - 1, at.strip, p.h0, first, e);
        Team<kWaves>::sync_lds();
        plain = plain_wave(e, at.r0, wave);
    }
    const int64_t lo = plain ? 0 : e.lo, hi = plain ? p.n : e.hi;
    float a[R][V], c[R][V];
    either(plain, [&](auto is_plain) {
        constexpr bool kPlain = decltype(is_plain)::value;
        float ra[V], rc[V];
#pragma unroll
        for (int q = 0; q < V; ++q) ra[q] = 1.0f, rc[q] = 0.0f;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t row = at.row + r;
            if (kPlain || (row >= lo && row < hi)) {
                float x[V], g[V];
                unpack<DT>(rx[r], x);
                unpack<DT>(rg[r], g);
                const int begin = kPlain ? -1 : e.begin[at.rl * R + r];
                if (begin >= 0) {
                    if (at.act) load_row<V, WIDE>(p.h0, begin, at.c0, p.d, rc);
                    // now: when the states are written h0 may be gone
                    if (r == 0 && p.marks && row % PDB_SCAN_MARK == 0 && at.act)
                        store_row<V, WIDE>(p.marks, row / PDB_SCAN_MARK, at.c0, p.d, at.own, rc);
#pragma unroll
                    for (int q = 0; q < V; ++q) ra[q] = -0.0f;
                }
#pragma unroll
                for (int q = 0; q < V; ++q) {
                    const Gate w = gate_of(g[q]);
                    rc[q] = __builtin_fmaf(w.f, rc[q], w.k * x[q]);
                    ra[q] *= w.f;
                }
            }
#pragma unroll
            for (int q = 0; q < V; ++q) a[r][q] = ra[q], c[r][q] = rc[q];
            // a row after another: all of them unpacked at once would not fit
            __builtin_amdgcn_sched_barrier(0);
        }
    });
    s.put(at.rl, at.cl, a[R - 1], c[R - 1]);
    s.join(wave);
    __syncthreads();
    const Map m = s.total();
    if (wave == 0)
        chain_wait<V, REACH>(p, at.turn, at.strip, m, fetched);
    else
        fetch_maps<V, REACH>(p, at.turn, at.strip, wave - 1, fetched);
    __syncthreads();
    s.spread(wave, chain_end<V, REACH>(p, at.turn, at.strip, m, wave == 0, fetched));
    float h[V];
    s.get(at.rl, at.cl, h);
    if (!at.act) return;
    either(plain, [&](auto is_plain) {
        constexpr bool kPlain = decltype(is_plain)::value;
        if (p.marks && at.row % PDB_SCAN_MARK == 0 && at.row < p.n &&
            (kPlain || e.begin[at.rl * R] < 0))
            store_row<V, WIDE>(p.marks, at.row / PDB_SCAN_MARK, at.c0, p.d, at.own, h);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t row = at.row + r;
            if (!kPlain && (row < lo || row >= hi)) continue;
            float out[V];
#pragma unroll
            for (int q = 0; q < V; ++q)
                out[q] = kPlain ? __builtin_fmaf(a[r][q], h[q], c[r][q])
                                : apply(Map{a[r][q], c[r][q]}, h[q]);
            store_vec<DT, WIDE>(p.y, p.ldy, row, at.c0, p.d, at.own, out);
            if constexpr (!kPlain) {
                const int end = e.end[at.rl * R + r];
                if (end >= 0 && p.state)
                    store_row<V, WIDE>(p.state, end, at.c0, p.d, at.own, out);
            }
        }
    });
}

// The backward pass of a tile.  Going back, a row acts on e (what the rows behind it
// ask of the state before them) as e -> f (dy + e); a row that ends a sequence takes
// d_state in place of e.  The states come from the mark that the tile begins with, so
// that only e passes along the chain.
template <int DT, bool WIDE, int REACH>
__global__ __launch_bounds__(kBlock, REACH == kReach ? 3 : 2) void k_scan_grad(Scan p) {
    using S = Shape<DT, true>;
    using At = Place<DT, WIDE, true>;
    constexpr int V = S::V, R = S::kRows;
    __shared__ Joint<V, false> forth;
    __shared__ Joint<V, true> back;
    __shared__ Edges<S::kTileRows> e;
    __shared__ Fetched<V, REACH> fetched;
    const int wave = __builtin_amdgcn_readfirstlane(wave_in_block());
    check_starts(p);
    if (wave == 0) {
        const uint32_t w = deal(p);
        const int32_t first = p.ticket ? 0 : first_edge(p, 0, S::kTileRows, true);
        if (lane_id() == 0) {
            e.dealt = w;
            e.first = first;
            fetched.late = fetched.cut = 0;
        }
    }
    __syncthreads();
    const uint32_t dealt = __builtin_amdgcn_readfirstlane(e.dealt);
    if (!on_grid(p, dealt)) return;
    const At at(p, dealt);
    int32_t first = 0;
    if (p.ticket && wave == 0) first = first_of(p, at.tile, at.r0, S::kTileRows);
    const int64_t ch = channel_of<V, WIDE>(p, at.strip, slot_of<V>(), false);
    const float mark =
        ch >= 0 && at.r0 < p.n ? p.marks_in[at.r0 / PDB_SCAN_MARK * p.d + ch] : 0.0f;
    u32x4 rx[R], rg[R], ry[R];
    load_rows<DT, WIDE>(p, p.gate, p.ldg, at.row, at.c0, at.act, rg);
    load_rows<DT, WIDE>(p, p.x, p.ldx, at.row, at.c0, at.act, rx);
    load_rows<DT, WIDE>(p, p.dy, p.lddy, at.row, at.c0, at.act, ry);
    if (p.ticket) {
        if (threadIdx.x == 0) e.first = first;
        Team<kWaves>::sync_lds();
    }
    first = __builtin_amdgcn_readfirstlane(e.first);
    bool plain = first == kPlain;
    if (!plain) {
        if (wave == 1)
            find_edges<V, WIDE>(p, at.r0, at.tile == p.tiles - 1, at.strip, p.d_state, first, e);
        Team<kWaves>::sync_lds();
        plain = plain_wave(e, at.r0, wave);
    }
    const int64_t lo = plain ? 0 : e.lo, hi = plain ? p.n : e.hi;
    float f[R][V], k[R][V];
    either(plain, [&](auto is_plain) {
        constexpr bool kPlain = decltype(is_plain)::value;
        float a[V], c[V];
#pragma unroll
        for (int q = 0; q < V; ++q) a[q] = 1.0f, c[q] = 0.0f;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float x[V], g[V];
            unpack<DT>(rx[r], x);
            unpack<DT>(rg[r], g);
#pragma unroll
            for (int q = 0; q < V; ++q) {
                const Gate w = gate_of(g[q]);
                f[r][q] = w.f;
                k[r][q] = w.k;
            }
            if (!kPlain && (at.row + r < lo || at.row + r >= hi)) continue;
            const int begin = kPlain ? -1 : e.begin[at.rl * R + r];
            if (begin >= 0) {
                if (at.act) load_row<V, WIDE>(p.h0, begin, at.c0, p.d, c);
#pragma unroll
                for (int q = 0; q < V; ++q) a[q] = -0.0f;
            }
#pragma unroll
            for (int q = 0; q < V; ++q) {
                c[q] = __builtin_fmaf(f[r][q], c[q], k[r][q] * x[q]);
                a[q] *= f[r][q];
            }
        }
        forth.put(at.rl, at.cl, a, c);
#pragma unroll
        for (int q = 0; q < V; ++q) a[q] = 1.0f, c[q] = 0.0f;
#pragma unroll
        for (int r = R - 1; r >= 0; --r) {
            if (!kPlain && (at.row + r < lo || at.row + r >= hi)) continue;
            const int end = kPlain ? -1 : e.end[at.rl * R + r];
            if (end >= 0) {
                if (at.act) load_row<V, WIDE>(p.d_state, end, at.c0, p.d, c);
#pragma unroll
                for (int q = 0; q < V; ++q) a[q] = -0.0f;
            }
            float dy[V];
            unpack<DT>(ry[r], dy);
#pragma unroll
            for (int q = 0; q < V; ++q) {
                c[q] = f[r][q] * (dy[q] + c[q]);
                a[q] *= f[r][q];
            }
        }
        back.put(at.rl, at.cl, a, c);
    });
    forth.join(wave);
    back.join(wave);
    __syncthreads();
    const Map m = back.total();
    if (wave == 0)
        chain_wait<V, REACH>(p, at.turn, at.strip, m, fetched);
    else
        fetch_maps<V, REACH>(p, at.turn, at.strip, wave - 1, fetched);
    float h[V], g[V];
    forth.spread(wave, mark);
    forth.get(at.rl, at.cl, h);
    __syncthreads();
    back.spread(wave, chain_end<V, REACH>(p, at.turn, at.strip, m, wave == 0, fetched));
    back.get(at.rl, at.cl, g);
    if (!at.act) return;
    either(plain, [&](auto is_plain) {
        constexpr bool kPlain = decltype(is_plain)::value;
        float gap[R][V];  // h_{t-1} - x_t
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (!kPlain && (at.row + r < lo || at.row + r >= hi)) continue;
            const int begin = kPlain ? -1 : e.begin[at.rl * R + r];
            if (begin >= 0) load_row<V, WIDE>(p.h0, begin, at.c0, p.d, h);
            float x[V];
            unpack<DT>(rx[r], x);
#pragma unroll
            for (int q = 0; q < V; ++q) {
                gap[r][q] = h[q] - x[q];
                h[q] = __builtin_fmaf(f[r][q], h[q], k[r][q] * x[q]);
            }
        }
#pragma unroll
        for (int r = R - 1; r >= 0; --r) {
            if (!kPlain && (at.row + r < lo || at.row + r >= hi)) continue;
            const int end = kPlain ? -1 : e.end[at.rl * R + r];
            if (end >= 0) load_row<V, WIDE>(p.d_state, end, at.c0, p.d, g);
            float dy[V], dx[V], dg[V];
            unpack<DT>(ry[r], dy);
#pragma unroll
            for (int q = 0; q < V; ++q) {
                const float t = dy[q] + g[q];
                dx[q] = k[r][q] * t;
                g[q] = f[r][q] * t;
                dg[q] = gap[r][q] * (k[r][q] * g[q]);
            }
            store_vec<DT, WIDE>(p.y, p.ldy, at.row + r, at.c0, p.d, at.own, dx);
            store_vec<DT, WIDE>(p.dgate, p.lddg, at.row + r, at.c0, p.d, at.own, dg);
            if constexpr (!kPlain) {
                const int begin = e.begin[at.rl * R + r];
                if (begin >= 0 && p.state)
                    store_row<V, WIDE>(p.state, begin, at.c0, p.d, at.own, g);
            }
        }
    });
}

// A chain's words before it begins, and the tiles' first edges: a tile to a wave.
__global__ __launch_bounds__(kBlock) void k_scan_clear(Scan p, int64_t words, int rows) {
    const int64_t at = (int64_t)blockIdx.x * kBlock + threadIdx.x, all = (int64_t)gridDim.x * kBlock;
    for (int64_t i = at; i < words; i += all) p.ticket[i] = i == 0 ? 0u : ~0u;
    for (int64_t t = at / kWave; t < p.tiles; t += all / kWave) {
        const int32_t f = first_edge(p, t * rows, (t + 1) * rows, t == p.tiles - 1);
        if (lane_id() == 0) p.first[t] = f;
    }
}

// Sequences of one row each: no state but the one that is given passes along.
template <int DT, bool WIDE>
__global__ __launch_bounds__(kBlock) void k_scan_step(Scan p, int64_t vecs) {
    constexpr int V = Elem<DT>::kVec;
    for (int64_t w = (int64_t)blockIdx.x * kBlock + threadIdx.x; w < p.n * vecs;
         w += (int64_t)gridDim.x * kBlock) {
        const int64_t i = w / vecs, c = (w - i * vecs) * V;
        const int64_t c0 = WIDE ? min(c, p.d - V) : c;
        float x[V], g[V], h[V];
        unpack<DT>(load_vec<DT, WIDE>(p.x, p.ldx, i, c0, p.d), x);
        unpack<DT>(load_vec<DT, WIDE>(p.gate, p.ldg, i, c0, p.d), g);
        load_row<V, WIDE>(p.h0, i, c0, p.d, h);
        const int own = (int)(c - c0);
        if (p.marks && i % PDB_SCAN_MARK == 0)
            store_row<V, WIDE>(p.marks, i / PDB_SCAN_MARK, c0, p.d, own, h);
#pragma unroll
        for (int q = 0; q < V; ++q) {
            const Gate k = gate_of(g[q]);
            h[q] = __builtin_fmaf(k.f, h[q], k.k * x[q]);
        }
        store_vec<DT, WIDE>(p.y, p.ldy, i, c0, p.d, own, h);
        if (p.state) store_row<V, WIDE>(p.state, i, c0, p.d, own, h);
    }
}

// No rows at all: the states are the first ones, or zeros.
__global__ __launch_bounds__(kBlock) void k_scan_none(const float *from, float *state, int64_t count) {
    for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < count;
         i += (int64_t)gridDim.x * kBlock)
        state[i] = from ? from[i] : 0.0f;
}

struct Cut {
    int64_t tiles, strips, slots;  // slots: of a tile
};
Cut cut_of(int64_t n, int64_t d, int dtype, bool back) {
    const int64_t v = 16 / dtype_size(dtype), strips = cdiv(std::max<int64_t>(d, 1), kStripLanes * v),
                  rows = kRowLanes * (back ? 4 : 8);
    return {std::max<int64_t>(cdiv(n, rows), 1), strips, strips * kStripLanes * v};
}
// The chain's words: the counter (in a line of its own), the maps, the states.
int64_t scan_words(const Cut &c) { return kAlign / 4 + c.tiles * c.slots * 3; }
// ... and the tiles' first edges.
int64_t scan_bytes(const Cut &c) { return align_up((scan_words(c) + c.tiles) * 4); }
size_t scan_ws_bytes(int64_t n, int64_t d) {
    // the most tiles, the widest strips
    return (size_t)scan_bytes(cut_of(n, d, PDB_BF16, true));
}

// Blocks of a launch; more are dealt to the next one.
constexpr int64_t kAtOnce = 1 << 20;
static_assert(kAtOnce <= kMostBlocks, "a launch takes them");

template <bool GRAD>
int run_scan(Scan p, int dtype, void *ws, size_t ws_bytes, hipStream_t stream) {
    const Cut cut = cut_of(p.n, p.d, dtype, GRAD);
    if (p.n == 0 && !p.starts) {
        if (!p.state) return PDB_OK;
        k_scan_none<<<grid_for((int64_t)p.b * p.d, kBlock, 4096), kBlock, 0, stream>>>(
            GRAD ? p.d_state : p.h0, p.state, (int64_t)p.b * p.d);
        PDB_LAUNCHED();
        return PDB_OK;
    }
    const bool step = !GRAD && !p.starts && p.len == 1;
    if (!step && (!ws || !aligned_to(ws, 8) || ws_bytes < scan_ws_bytes(p.n, p.d)))
        return PDB_ERR_WORKSPACE;
    if (cut.tiles * cut.strips > INT32_MAX) return PDB_ERR_UNSUPPORTED;
    p.tiles = (int32_t)cut.tiles;
    p.strips = (int32_t)cut.strips;
    if ((cut.tiles > 1 || cut.strips > kAtOnce) && !step) {
        p.ticket = static_cast<uint32_t *>(ws);
        p.total = reinterpret_cast<unsigned long long *>(static_cast<char *>(ws) + kAlign);
        p.leave = reinterpret_cast<uint32_t *>(p.total + cut.tiles * cut.slots);
        p.first = reinterpret_cast<int32_t *>(p.ticket + scan_words(cut));
    }
    return with_dtype(dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        auto go = [&](auto wide) -> int {
            constexpr bool W = decltype(wide)::value;
            if (step) {
                const int64_t vecs = cdiv(p.d, Elem<DT>::kVec);
                k_scan_step<DT, W><<<grid_for(p.n * vecs, kBlock), kBlock, 0, stream>>>(p, vecs);
                PDB_LAUNCHED();
                return PDB_OK;
            }
            if (p.ticket) {
                const int64_t words = scan_words(cut);
                k_scan_clear<<<grid_for(std::max(words / 4, cut.tiles * kWave), kBlock, 2048), kBlock, 0,
                               stream>>>(p, words, Shape<DT, GRAD>::kTileRows);
                PDB_LAUNCHED();
            }
            const bool few = cut.tiles > kReach && cut.strips <= (GRAD ? kFewStripsBack : kFewStrips);
            // the counter deals on from launch to launch
            for (int64_t left = cut.tiles * cut.strips; left > 0; left -= kAtOnce) {
                const unsigned grid = (unsigned)std::min(left, kAtOnce);
                if constexpr (GRAD) {
                    if (few)
                        k_scan_grad<DT, W, kFarReach><<<grid, kBlock, 0, stream>>>(p);
                    else
                        k_scan_grad<DT, W, kReach><<<grid, kBlock, 0, stream>>>(p);
                } else {
                    if (few)
                        k_scan<DT, W, kFarReach><<<grid, kBlock, 0, stream>>>(p);
                    else
                        k_scan<DT, W, kReach><<<grid, kBlock, 0, stream>>>(p);
                }
                PDB_LAUNCHED();
            }
            return PDB_OK;
        };
        return p.d >= Elem<DT>::kVec ? go(std::true_type()) : go(std::false_type());
    });
}

int check_floats(const void *p) { return aligned_to(p, 4) ? PDB_OK : PDB_ERR_INVALID_ARG; }

int check_sequences(int64_t n, int64_t d, const int32_t *starts, int64_t b) {
    if (n < 0 || d < 0 || b < 0 || !aligned_to(starts, 4)) return PDB_ERR_INVALID_ARG;
    if (n > INT32_MAX || d > INT32_MAX || b >= INT32_MAX) return PDB_ERR_UNSUPPORTED;
    if (!starts && (b == 0 ? n > 0 : n % b != 0)) return PDB_ERR_INVALID_ARG;
    return PDB_OK;
}

}  // namespace
}  // namespace pdbk

using namespace pdbk;

extern "C" int pdb_gated_scan_workspace_bytes(int64_t n, int64_t d, size_t *bytes) {
    if (!bytes || n < 0 || d < 0) return PDB_ERR_INVALID_ARG;
    if (n > INT32_MAX || d > INT32_MAX) return PDB_ERR_UNSUPPORTED;
    *bytes = scan_ws_bytes(n, d);
    return PDB_OK;
}

extern "C" int pdb_gated_scan(const void *x, int64_t ldx, const void *gate, int64_t ldg, int dtype,
                              int64_t n, int64_t d, const int32_t *starts, int64_t b,
                              const float *h0, void *y, int64_t ldy, float *state, float *marks,
                              int32_t *status, void *ws, size_t ws_bytes, hipStream_t stream) {
    if (int e = check_matrix(x, dtype, ldx, n, d)) return e;
    if (int e = check_matrix(gate, dtype, ldg, n, d)) return e;
    if (int e = check_matrix(y, dtype, ldy, n, d)) return e;
    if (int e = check_sequences(n, d, starts, b)) return e;
    if (check_floats(h0) || check_floats(state) || check_floats(marks)) return PDB_ERR_INVALID_ARG;
    if (b == 0 || d == 0) return PDB_OK;
    Scan p = {};
    p.x = x, p.ldx = ldx, p.gate = gate, p.ldg = ldg, p.n = n, p.d = d;
    p.starts = starts, p.b = (int32_t)b, p.len = starts ? 0 : (int32_t)(n / b);
    p.h0 = h0, p.state = state, p.y = y, p.ldy = ldy, p.marks = marks, p.status = status;
    return run_scan<false>(p, dtype, ws, ws_bytes, stream);
}

extern "C" int pdb_gated_scan_grad(const void *dy, int64_t lddy, const void *x, int64_t ldx,
                                   const void *gate, int64_t ldg, int dtype, int64_t n, int64_t d,
                                   const int32_t *starts, int64_t b, const float *h0,
                                   const float *marks, const float *d_state, void *dx,
                                   int64_t lddx, void *dgate, int64_t lddg, float *dh0,
                                   int32_t *status, void *ws, size_t ws_bytes, hipStream_t stream) {
    if (int e = check_matrix(dy, dtype, lddy, n, d)) return e;
    if (int e = check_matrix(x, dtype, ldx, n, d)) return e;
    if (int e = check_matrix(gate, dtype, ldg, n, d)) return e;
    if (int e = check_matrix(dx, dtype, lddx, n, d)) return e;
    if (int e = check_matrix(dgate, dtype, lddg, n, d)) return e;
    if (int e = check_sequences(n, d, starts, b)) return e;
    if (check_floats(h0) || check_floats(marks) || check_floats(d_state) || check_floats(dh0))
        return PDB_ERR_INVALID_ARG;
    if (n > 0 && d > 0 && !marks) return PDB_ERR_INVALID_ARG;
    if (b == 0 || d == 0) return PDB_OK;
    Scan p = {};
    p.dy = dy, p.lddy = lddy, p.x = x, p.ldx = ldx, p.gate = gate, p.ldg = ldg, p.n = n, p.d = d;
    p.starts = starts, p.b = (int32_t)b, p.len = starts ? 0 : (int32_t)(n / b);
    p.h0 = h0, p.marks_in = marks, p.d_state = d_state, p.state = dh0;
    p.y = dx, p.ldy = lddx, p.dgate = dgate, p.lddg = lddg, p.status = status;
    return run_scan<true>(p, dtype, ws, ws_bytes, stream);
}
