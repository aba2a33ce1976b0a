// The gated recurrence h_t = f_t h_{t-1} + (1 - f_t) x_t over packed sequences and its
// backward pass (gfx950, wave64).
//
// A row acts on the state as the map h -> a h + c, and maps compose: (a1, c1) then
// (a2, c2) is (a2 a1, a2 c1 + c2).  The rows are cut into tiles of kTileRows, whatever
// sequences they hold, and the channels into strips of 128 bytes of a row: a block has
// a tile of a strip in registers, kRows rows of a vector of channels to a thread, and
// reads it once.  The threads' maps are joined through LDS, the tiles' through the
// workspace while the blocks run: each publishes its map, waits for the state behind
// the tile kReach before and applies the maps between, in order (so the sums do not
// depend on who was first), and publishes the state behind its own.  Tiles are dealt
// by a counter, so a block waits only for blocks that have begun.  A row that begins a
// sequence takes its first state in place of what enters: its map is "cut", a = -0
// (gates are never negative, so products and selects keep the mark), and nothing of
// another sequence passes it, not even a NaN.
#include "pdb_vec.h"
#include "pdb_softmax.h"
#include "../../include/pdb_layers.h"

namespace pdbk {
namespace {

constexpr int kStripLanes = 8;                         // lanes over 128 bytes of a row
constexpr int kRowLanes = kBlock / kStripLanes;        // 32
constexpr int kRows = 8;                               // rows of a thread
constexpr int kTileRows = kRowLanes * kRows;           // 256
static_assert(kTileRows % PDB_SCAN_MARK == 0 && PDB_SCAN_MARK % kRows == 0,
              "a mark is at the first row of some thread");

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

// A gate as the smaller of f and 1 - f, negative (also -0) where that is 1 - f: both
// keep their relative accuracy, at either end.
__device__ __forceinline__ float small_gate(float g) {
    const float t = exp2_raw(-fabsf(g) * kLog2e);
    const float s = t * __builtin_amdgcn_rcpf(1.0f + t);
    return __uint_as_float(__float_as_uint(s) | (~__float_as_uint(g) & 0x80000000u));
}
struct Gate {
    float f, k;  // k = 1 - f
};
__device__ __forceinline__ Gate open_gate(float w) {
    const float s = fabsf(w), l = 1.0f - s;
    return (int)__float_as_uint(w) < 0 ? Gate{l, s} : Gate{s, l};
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
    // in the order of the chain (the backward's from the last tile on); NULL of one tile
    unsigned long long *total;  // [tiles][strips][slots]: the tiles' maps
    uint32_t *leave;            // the same: the states behind them
    uint32_t *ticket;  // [0]: tiles dealt; [1]: 0 once a wait has lasted too long
};

// The sequences that begin and end with the rows of a tile, -1 elsewhere.
struct Edges {
    int32_t begin[kTileRows], end[kTileRows];
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

// Fills `e` for the rows from r0 on; [lo, hi) are the rows of sequences.  True if the
// tile has neither edges nor rows of no sequence.  Empty sequences at the tile's rows
// (the last tile: or behind) get their states, those of `from`.
template <int V, bool WIDE>
__device__ __forceinline__ bool find_edges(const Scan &p, int64_t r0, bool last_tile, int64_t c0,
                                           int own, bool act, const float *from, Edges &e, int64_t &lo,
                                           int64_t &hi) {
    int any = 0;
    const int t = threadIdx.x;
    e.begin[t] = e.end[t] = -1;
    static_assert(kTileRows == kBlock, "a row to a thread");
    if (!p.starts) {
        lo = 0;
        hi = p.n;
        const int64_t r = r0 + t;
        if (r < p.n) {
            const uint32_t s = (uint32_t)r / (uint32_t)p.len, o = (uint32_t)r - s * (uint32_t)p.len;
            if (o == 0) e.begin[t] = (int)s;
            if (o == (uint32_t)p.len - 1) e.end[t] = (int)s;
            any = e.begin[t] >= 0 || e.end[t] >= 0;
        } else {
            any = 1;
        }
        return !__syncthreads_or(any);
    }
    __syncthreads();
    const int32_t *starts = p.starts;
    lo = std::max<int64_t>(starts[0], 0);
    hi = std::min<int64_t>(starts[p.b], p.n);
    if (r0 < lo || r0 + kTileRows > hi) any = 1;
    const int64_t r1 = r0 + kTileRows;
    const int64_t first = starts_below(starts, (int64_t)p.b + 1, r0 + (r0 == 0 ? INT32_MIN : 0));
    // all threads take part in a turn, so that the empty sequences' states are written
    // by whole rows of lanes
    for (int64_t j0 = first;; j0 += kBlock) {
        const int64_t j = j0 + t;
        const bool have = j <= p.b;
        const int64_t at = have ? starts[j] : INT64_MAX;
        const int64_t next = j < p.b ? starts[j + 1] : INT64_MAX;
        const int64_t before = have && j > 0 ? starts[j - 1] : INT64_MIN;
        const bool mine = have && (at < r1 || last_tile);
        if (have && at <= r1) {
            if (j < p.b && at < next && at >= r0 && at < r1) {
                e.begin[at - r0] = (int)j;
                any = 1;
            }
            if (j > 0 && before < at && at > r0) {
                e.end[at - 1 - r0] = (int)j - 1;
                any = 1;
            }
        }
        const bool none = mine && j < p.b && next <= at;
        if (__syncthreads_or(none) && p.state) {
            // rare: walk the turn's sequences, the empty ones' states by their channels
            for (int64_t i = j0; i < std::min<int64_t>(j0 + kBlock, p.b); ++i) {
                const int64_t a0 = starts[i], a1 = starts[i + 1];
                if (a1 > a0 || !(a0 < r1 || last_tile)) continue;
                if (act && threadIdx.x < kStripLanes)
                    for (int q = own; q < V; ++q)
                        if (WIDE || c0 + q < p.d)
                            p.state[i * p.d + c0 + q] = from ? from[i * p.d + c0 + q] : 0.0f;
            }
        }
        if (!__syncthreads_or(have && at <= r1)) break;
    }
    return !__syncthreads_or(any);
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

// What a block shares: the threads' maps, then what enters each thread's rows.
template <int V>
struct Shared {
    static constexpr int kSlots = kStripLanes * V;
    Map part[kRowLanes][kSlots];
    float enter[kRowLanes][kSlots];
    Edges edges;
};

// The slot of a lane of the first wave (strips of 32-bit channels: of two lanes).
template <int V>
__device__ __forceinline__ int slot_of() {
    return lane_id() & (Shared<V>::kSlots - 1);
}

// Joins the threads' maps (in row order, or from the last row lane to the first) by the
// first wave, a slot to a lane: total is the tile's map.
template <int V, bool BACK>
__device__ __forceinline__ Map join_total(const Shared<V> &s) {
    const int slot = slot_of<V>();
    Map m = s.part[BACK ? kRowLanes - 1 : 0][slot];
#pragma unroll 8
    for (int r = 1; r < kRowLanes; ++r) m = then(m, s.part[BACK ? kRowLanes - 1 - r : r][slot]);
    return m;
}
template <int V, bool BACK>
__device__ __forceinline__ void join_enter(Shared<V> &s, float h) {
    const int slot = slot_of<V>();
#pragma unroll 8
    for (int i = 0; i < kRowLanes; ++i) {
        const int r = BACK ? kRowLanes - 1 - i : i;
        s.enter[r][slot] = h;
        h = apply(s.part[r][slot], h);
    }
}

template <int V>
__device__ __forceinline__ void put_part(Shared<V> &s, int rl, int cl, const float *a, const float *c) {
#pragma unroll
    for (int q = 0; q < V; ++q) s.part[rl][cl * V + q] = Map{a[q], c[q]};
}
template <int V>
__device__ __forceinline__ void get_enter(const Shared<V> &s, int rl, int cl, float *h) {
#pragma unroll
    for (int q = 0; q < V; ++q) h[q] = s.enter[rl][cl * V + q];
}

// Where a block and a thread are.
template <int DT, bool WIDE>
struct Place {
    static constexpr int V = Elem<DT>::kVec;
    int turn, tile, strip, rl, cl, own;  // turn: the tile's place in the chain
    int64_t r0, row, c0;
    bool act;
    __device__ __forceinline__ Place(const Scan &p, uint32_t w, bool back) {
        turn = (int)(w / (uint32_t)p.strips);
        strip = (int)(w - (uint32_t)turn * (uint32_t)p.strips);
        tile = back ? p.tiles - 1 - turn : turn;
        rl = threadIdx.x / kStripLanes;
        cl = threadIdx.x % kStripLanes;
        r0 = (int64_t)tile * kTileRows;
        row = r0 + rl * kRows;
        // the last vector ends with the row: it may share channels with the one before,
        // which has them (the states may be written over h0)
        const int64_t c = ((int64_t)strip * kStripLanes + cl) * V;
        act = c < p.d;
        c0 = WIDE ? min(c, p.d - V) : c;
        own = (int)(c - c0);
    }
};

// The block's place in the chain's order.
__device__ __forceinline__ uint32_t next_tile(const Scan &p) {
    if (!p.ticket) return blockIdx.x;
    __shared__ uint32_t w;
    if (threadIdx.x == 0)
        w = __hip_atomic_fetch_add(p.ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    return w;
}

constexpr int kReach = 16;
constexpr int64_t kPatience = 200000000;  // ticks of the 100 MHz clock: 2 s
constexpr int64_t kUneasy = 100000;       // 1 ms

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

// What enters the tile at `turn` of strip `strip`, whose map is m: by the first wave, a
// slot to a lane.  A wait that lasts kPatience ends with NaN and a status.
template <int V>
__device__ __forceinline__ float chain(const Scan &p, int turn, int strip, Map m) {
    constexpr int kSlots = Shared<V>::kSlots;
    if (!p.ticket) return 0.0f;
    const int64_t slots = (int64_t)p.strips * kSlots;
    const int64_t at = (int64_t)turn * slots + (int64_t)strip * kSlots + slot_of<V>();
    const bool first_of_slot = lane_id() < kSlots, next = turn < p.tiles - 1;
    if (next && first_of_slot) post(p.total + at, word_of(m));
    unsigned long long w[kReach - 1];
    uint32_t h = 0;
    bool late = false;
    const int64_t t0 = now_ticks();
    if (turn >= kReach) {
        while (true) {
            h = peek(p.leave + (at - kReach * slots));
            if (!__any(h == ~0u)) break;
            if ((late = give_up(p, t0))) break;
            __builtin_amdgcn_s_sleep(4);
        }
    }
    const int maps = turn >= kReach ? kReach - 1 : turn;
    while (!late) {
        bool missing = false;
#pragma unroll
        for (int j = 0; j < kReach - 1; ++j) {
            w[j] = 0;
            if (j < maps) w[j] = peek(p.total + (at - (int64_t)(maps - j) * slots));
        }
#pragma unroll
        for (int j = 0; j < kReach - 1; ++j) missing |= w[j] == ~0ull;
        if (!__any(missing)) break;
        late = give_up(p, t0);
        __builtin_amdgcn_s_sleep(2);
    }
    float enter = __uint_as_float(h);
    if (late) {
        enter = kNan;  // seen by whoever uses the result
        if (p.status) *p.status = PDB_ERR_DEVICE;
    } else {
#pragma unroll
        for (int j = 0; j < kReach - 1; ++j)
            if (j < maps) enter = apply(map_of(w[j]), enter);
    }
    if (turn + kReach < p.tiles && first_of_slot) post(p.leave + at, word_of(apply(m, enter)));
    return enter;
}

template <int DT, bool WIDE>
__global__ __launch_bounds__(kBlock, 2) void k_scan(Scan p) {
    constexpr int V = Elem<DT>::kVec;
    __shared__ Shared<V> s;
    const Place<DT, WIDE> at(p, next_tile(p), false);
    int64_t lo, hi;
    const bool plain =
        find_edges<V, WIDE>(p, at.r0, at.tile == p.tiles - 1, at.c0, at.own, at.act, p.h0, s.edges, lo, hi);
    check_starts(p);
    float a[kRows][V], c[kRows][V];
    auto local = [&](auto is_plain) {
        constexpr bool kPlain = decltype(is_plain)::value;
        u32x4 rx[kRows], rg[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            rx[r] = rg[r] = u32x4{0, 0, 0, 0};
            if (at.act && (kPlain || at.row + r < p.n)) {
                rx[r] = load_vec<DT, WIDE>(p.x, p.ldx, at.row + r, at.c0, p.d);
                rg[r] = load_vec<DT, WIDE>(p.gate, p.ldg, at.row + r, at.c0, p.d);
            }
        }
        float ra[V], rc[V];
#pragma unroll
        for (int q = 0; q < V; ++q) ra[q] = 1.0f, rc[q] = 0.0f;
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const int64_t row = at.row + r;
            if (kPlain || (row >= lo && row < hi)) {
                float x[V], g[V];
                unpack<DT>(rx[r], x);
                unpack<DT>(rg[r], g);
                const int begin = kPlain ? -1 : s.edges.begin[at.rl * kRows + r];
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
                    const Gate w = open_gate(small_gate(g[q]));
                    rc[q] = __builtin_fmaf(w.f, rc[q], w.k * x[q]);
                    ra[q] *= w.f;
                }
            }
#pragma unroll
            for (int q = 0; q < V; ++q) a[r][q] = ra[q], c[r][q] = rc[q];
        }
    };
    if (plain)
        local(std::true_type());
    else
        local(std::false_type());
    put_part(s, at.rl, at.cl, a[kRows - 1], c[kRows - 1]);
    __syncthreads();
    if (wave_in_block() == 0) {
        const Map m = join_total<V, false>(s);
        join_enter<V, false>(s, chain<V>(p, at.turn, at.strip, m));
    }
    __syncthreads();
    float h[V];
    get_enter(s, at.rl, at.cl, h);
    auto finish = [&](auto is_plain) {
        constexpr bool kPlain = decltype(is_plain)::value;
        if (p.marks && at.row % PDB_SCAN_MARK == 0 && at.row < p.n &&
            (kPlain || s.edges.begin[at.rl * kRows] < 0))
            store_row<V, WIDE>(p.marks, at.row / PDB_SCAN_MARK, at.c0, p.d, at.own, h);
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const int64_t row = at.row + r;
            if (!kPlain && (row < lo || row >= hi)) continue;
            float out[V];
#pragma unroll
            for (int q = 0; q < V; ++q)
                out[q] = kPlain ? __builtin_fmaf(a[r][q], h[q], c[r][q])
                                : apply(Map{a[r][q], c[r][q]}, h[q]);
            store_vec<DT, WIDE>(p.y, p.ldy, row, at.c0, p.d, at.own, out);
            if constexpr (!kPlain) {
                const int end = s.edges.end[at.rl * kRows + r];
                if (end >= 0 && p.state) store_row<V, WIDE>(p.state, end, at.c0, p.d, at.own, out);
            }
        }
    };
    if (!at.act) return;
    if (plain)
        finish(std::true_type());
    else
        finish(std::false_type());
}

// The backward pass of a tile.  Going back, a row acts on e (what the rows behind it
// ask of the state before them) as e -> f (dy + e); a row that ends a sequence takes
// d_state in place of e.  The states come from the mark that the tile begins with.
template <int DT, bool WIDE>
__global__ __launch_bounds__(kBlock, 2) void k_scan_grad(Scan p) {
    constexpr int V = Elem<DT>::kVec;
    __shared__ Shared<V> s;
    const Place<DT, WIDE> at(p, next_tile(p), true);
    int64_t lo, hi;
    const bool plain =
        find_edges<V, WIDE>(p, at.r0, at.tile == p.tiles - 1, at.c0, at.own, at.act, p.d_state, s.edges, lo, hi);
    check_starts(p);
    float w[kRows][V], x[kRows][V];
    u32x4 ry[kRows];
    auto inside = [&](int64_t row) { return row >= lo && row < hi; };
    auto load = [&](auto is_plain) {
        constexpr bool kPlain = decltype(is_plain)::value;
        u32x4 rx[kRows], rg[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            rx[r] = rg[r] = ry[r] = u32x4{0, 0, 0, 0};
            if (at.act && (kPlain || at.row + r < p.n)) {
                rg[r] = load_vec<DT, WIDE>(p.gate, p.ldg, at.row + r, at.c0, p.d);
                ry[r] = load_vec<DT, WIDE>(p.dy, p.lddy, at.row + r, at.c0, p.d);
                rx[r] = load_vec<DT, WIDE>(p.x, p.ldx, at.row + r, at.c0, p.d);
            }
        }
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            float g[V];
            unpack<DT>(rg[r], g);
            unpack<DT>(rx[r], x[r]);
#pragma unroll
            for (int q = 0; q < V; ++q) w[r][q] = small_gate(g[q]);
        }
    };
    // the thread's map of e, from its last row to its first
    auto back = [&](auto is_plain) {
        constexpr bool kPlain = decltype(is_plain)::value;
        float a[V], c[V];
#pragma unroll
        for (int q = 0; q < V; ++q) a[q] = 1.0f, c[q] = 0.0f;
#pragma unroll
        for (int r = kRows - 1; r >= 0; --r) {
            if (!kPlain && !inside(at.row + r)) continue;
            const int end = kPlain ? -1 : s.edges.end[at.rl * kRows + r];
            if (end >= 0) {
                if (at.act) load_row<V, WIDE>(p.d_state, end, at.c0, p.d, c);
#pragma unroll
                for (int q = 0; q < V; ++q) a[q] = -0.0f;
            }
            float dy[V];
            unpack<DT>(ry[r], dy);
#pragma unroll
            for (int q = 0; q < V; ++q) {
                const float f = open_gate(w[r][q]).f;
                c[q] = f * (dy[q] + c[q]);
                a[q] *= f;
            }
        }
        put_part(s, at.rl, at.cl, a, c);
    };
    // the thread's map of h, and, with what enters, h_{t-1} - x_t in the place of x_t
    auto forth = [&](auto is_plain, float *h, bool last) {
        constexpr bool kPlain = decltype(is_plain)::value;
        float a[V];
#pragma unroll
        for (int q = 0; q < V; ++q) a[q] = 1.0f;
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            if (!kPlain && !inside(at.row + r)) continue;
            const int begin = kPlain ? -1 : s.edges.begin[at.rl * kRows + r];
            if (begin >= 0) {
                if (at.act) load_row<V, WIDE>(p.h0, begin, at.c0, p.d, h);
#pragma unroll
                for (int q = 0; q < V; ++q) a[q] = -0.0f;
            }
#pragma unroll
            for (int q = 0; q < V; ++q) {
                const Gate g = open_gate(w[r][q]);
                const float now = __builtin_fmaf(g.f, h[q], g.k * x[r][q]);
                if (last) x[r][q] = h[q] - x[r][q];
                h[q] = now;
                a[q] *= g.f;
            }
        }
        if (!last) put_part(s, at.rl, at.cl, a, h);
    };
    auto both = [&](auto f) {
        if (plain)
            f(std::true_type());
        else
            f(std::false_type());
    };
    both(load);
    {
        float h[V];
#pragma unroll
        for (int q = 0; q < V; ++q) h[q] = 0.0f;
        both([&](auto t) { forth(t, h, false); });
        __syncthreads();
        if (wave_in_block() == 0) {
            // the mark, by slots
            const int slot = slot_of<V>();
            float m = 0.0f;
            const int64_t cs = ((int64_t)at.strip * kStripLanes + slot / V) * V;
            const int64_t ch = (WIDE ? min(cs, p.d - V) : cs) + slot % V;
            if (cs < p.d && ch < p.d && at.r0 < p.n)
                m = p.marks_in[at.r0 / PDB_SCAN_MARK * p.d + ch];
            join_enter<V, false>(s, m);
        }
        __syncthreads();
        get_enter(s, at.rl, at.cl, h);
        both([&](auto t) { forth(t, h, true); });
        __syncthreads();
    }
    both(back);
    __syncthreads();
    if (wave_in_block() == 0) {
        const Map m = join_total<V, true>(s);
        join_enter<V, true>(s, chain<V>(p, at.turn, at.strip, m));
    }
    __syncthreads();
    if (!at.act) return;
    float e[V];
    get_enter(s, at.rl, at.cl, e);
    both([&](auto is_plain) {
        constexpr bool kPlain = decltype(is_plain)::value;
#pragma unroll
        for (int r = kRows - 1; r >= 0; --r) {
            if (!kPlain && !inside(at.row + r)) continue;
            const int end = kPlain ? -1 : s.edges.end[at.rl * kRows + r];
            if (end >= 0) load_row<V, WIDE>(p.d_state, end, at.c0, p.d, e);
            float dy[V], dx[V], dg[V];
            unpack<DT>(ry[r], dy);
#pragma unroll
            for (int q = 0; q < V; ++q) {
                const Gate g = open_gate(w[r][q]);
                const float t = dy[q] + e[q];
                dx[q] = g.k * t;
                dg[q] = t * x[r][q] * (g.f * g.k);
                e[q] = g.f * t;
            }
            store_vec<DT, WIDE>(p.y, p.ldy, at.row + r, at.c0, p.d, at.own, dx);
            store_vec<DT, WIDE>(p.dgate, p.lddg, at.row + r, at.c0, p.d, at.own, dg);
            if constexpr (!kPlain) {
                const int begin = s.edges.begin[at.rl * kRows + r];
                if (begin >= 0 && p.state) store_row<V, WIDE>(p.state, begin, at.c0, p.d, at.own, e);
            }
        }
    });
}

// A chain's words before it begins.
__global__ __launch_bounds__(kBlock) void k_scan_clear(uint32_t *words, int64_t count) {
    for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < count;
         i += (int64_t)gridDim.x * kBlock)
        words[i] = i == 0 ? 0u : ~0u;
}

// Sequences of one row each: no state but the one that is given passes along.
template <int DT, bool WIDE>
__global__ __launch_bounds__(kBlock) void k_scan_step(Scan p, int64_t vecs) {
    constexpr int V = Elem<DT>::kVec;
    const int64_t w = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (w >= p.n * vecs) return;
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
        const Gate k = open_gate(small_gate(g[q]));
        h[q] = __builtin_fmaf(k.f, h[q], k.k * x[q]);
    }
    store_vec<DT, WIDE>(p.y, p.ldy, i, c0, p.d, own, h);
    if (p.state) store_row<V, WIDE>(p.state, i, c0, p.d, own, h);
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
Cut cut_of(int64_t n, int64_t d, int dtype) {
    const int64_t v = 16 / dtype_size(dtype), strips = cdiv(std::max<int64_t>(d, 1), kStripLanes * v);
    return {std::max<int64_t>(cdiv(n, kTileRows), 1), strips, strips * kStripLanes * v};
}
// The chain's words: the counter (in a line of its own), the maps, the states.
int64_t scan_words(const Cut &c) { return kAlign / 4 + c.tiles * c.slots * 3; }
size_t scan_ws_bytes(int64_t n, int64_t d) {
    return (size_t)align_up(scan_words(cut_of(n, d, PDB_BF16)) * 4);  // the widest strips
}

template <bool GRAD>
int run_scan(Scan p, int dtype, void *ws, size_t ws_bytes, hipStream_t stream) {
    const Cut cut = cut_of(p.n, p.d, dtype);
    if (p.n == 0 && !p.starts) {
        if (!p.state) return PDB_OK;
        k_scan_none<<<grid_for((int64_t)p.b * p.d, kBlock, 4096), kBlock, 0, stream>>>(
            GRAD ? p.d_state : p.h0, p.state, (int64_t)p.b * p.d);
        PDB_LAUNCHED();
        return PDB_OK;
    }
    if (!ws || !aligned_to(ws, 8) || ws_bytes < scan_ws_bytes(p.n, p.d)) return PDB_ERR_WORKSPACE;
    if (cut.tiles * cut.strips > INT32_MAX) return PDB_ERR_UNSUPPORTED;
    p.tiles = (int32_t)cut.tiles;
    p.strips = (int32_t)cut.strips;
    if (cut.tiles > 1) {
        p.ticket = static_cast<uint32_t *>(ws);
        p.total = reinterpret_cast<unsigned long long *>(static_cast<char *>(ws) + kAlign);
        p.leave = reinterpret_cast<uint32_t *>(p.total + cut.tiles * cut.slots);
    }
    return with_dtype(dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        auto go = [&](auto wide) -> int {
            constexpr bool W = decltype(wide)::value;
            const unsigned grid = (unsigned)(cut.tiles * cut.strips);
            if (!GRAD && !p.starts && p.len == 1 && p.n > 0) {
                const int64_t vecs = cdiv(p.d, Elem<DT>::kVec);
                if (cdiv(p.n * vecs, kBlock) > INT32_MAX) return PDB_ERR_UNSUPPORTED;
                k_scan_step<DT, W><<<(unsigned)cdiv(p.n * vecs, kBlock), kBlock, 0, stream>>>(p, vecs);
                PDB_LAUNCHED();
                return PDB_OK;
            }
            if (p.ticket) {
                const int64_t words = scan_words(cut);
                k_scan_clear<<<grid_for(words, kBlock * 4, 2048), kBlock, 0, stream>>>(p.ticket, words);
            }
            if constexpr (GRAD)
                k_scan_grad<DT, W><<<grid, kBlock, 0, stream>>>(p);
            else
                k_scan<DT, W><<<grid, kBlock, 0, stream>>>(p);
            PDB_LAUNCHED();
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
