// Verification of drafted tokens against the target's probabilities, from given random
// numbers; with nothing drafted, the drawing of a token (gfx950, wave64).
//
// The answers are choices: whether u q(x) < p(x), and where a running sum over the
// vocabulary passes u R.  In binary32 a sum over 131,072 entries is off by 1e-6 and more,
// as much as many an entry has; so what an answer hangs on is in binary64, and the rest is
// not.  (An exponential in binary64 is 29 instructions: over all rows they would take 93 us
// where memory takes 31, 64 sequences of 5 drafted tokens of 131,072 in 16 bits.)
//
// 1. every row's maximum and sum, one pass at the rate of memory: exponentials in
//    binary32, sums of 32 of them added in binary64.  The sums are within kNear of the
//    true ones; the few tokens that stand nearer than that to the bar get them exactly.
//    31 us there, 5.9 TB/s.  Where each sequence stops: 5 us, latency; 100 us more, two rows
//    in binary64 by a block, where a token did stand so near (a token in some 40,000, one
//    such call in two hundred).
// 2. of the row at which each sequence stopped, chunk by chunk in binary64: the sums of
//    e_p and e_q (exp of logits below the row's maximum), and those over the entries that
//    p has more of, e_p > r e_q with r = S_p / S_q: by step 1's r, since their exact r is
//    known only behind this step.  Entries within kNear of it have sums of their own, and
//    the range of their e_p / e_q is kept.  (They may be many: logits of 16 bits lie on a
//    grid, and so does e_p / e_q.)  21 us, of which the vector unit is busy for 12.
// 3. with S_p and S_q, a chunk's residual is A - r B, and the same of the entries near r if
//    r is below their range (a chunk with r inside it is done again); the chunk that the
//    random number picks is run through entry by entry.  9 us, latency.
// Without drafted tokens step 1 is left out: chunks have maxima of their own.
#include "pdb_softmax.h"

namespace pdbk {
namespace {

// Consecutive entries of a thread: a chunk is kBlock times as many.  Drawing alone, without
// drafted tokens, is bound by the exponentials (256 rows of 131,072: 40 us with 16, 46 with
// 8); behind a draft by latency and registers (1 sequence of four: 20 us with 8, 23 with 16;
// 64 of five: 70 and 73).
constexpr int each_of(int32_t k) { return k == 0 ? 16 : 8; }
constexpr double kLowest = -700.0;  // powers below this count as 0
// What step 1's sums may be off by, relatively, two rows of them.  In units of 2^-24: an
// exponential's power by 3 of its size (c = log2(e) / T, the difference, the product) times
// ln 2, where the size, averaged over a row's weights, is below log2 of the row's length,
// 31; the exponential by 2; a sum of 32 by 31.  That is below 100 a row; 512 is kNear.
constexpr double kNear = 0x1p-15;

// 2^f by the series of e^(f ln 2) through f^12, |f| <= 1/2; what is left out is below 2e-16.
__device__ __forceinline__ double exp2_series(double f) {
    double r = 0x1.c3bd650fc2983p-36;
    r = fma(r, f, 0x1.e8cac7351bb22p-32);
    r = fma(r, f, 0x1.e4cf5158b8ec7p-28);
    r = fma(r, f, 0x1.b5253d395e7c1p-24);
    r = fma(r, f, 0x1.62c0223a5c822p-20);
    r = fma(r, f, 0x1.ffcbfc588b0c5p-17);
    r = fma(r, f, 0x1.430912f86c786p-13);
    r = fma(r, f, 0x1.5d87fe78a6730p-10);
    r = fma(r, f, 0x1.3b2ab6fba4e77p-7);
    r = fma(r, f, 0x1.c6b08d704a0bfp-5);
    r = fma(r, f, 0x1.ebfbdff82c58ep-3);
    r = fma(r, f, 0x1.62e42fefa39efp-1);
    return fma(r, f, 1.0);
}
// e^y for y <= 0 (0 below kLowest, NaN of NaN)
__device__ __forceinline__ double exp_f64(double y) {
    const double t = y * 0x1.71547652b82fep+0;
    const double n = __builtin_rint(t);
    return y < kLowest ? 0.0 : __builtin_amdgcn_ldexp(exp2_series(t - n), (int)n);
}
// The same of (z - m) / T, with the powers 2^(j / 64) in LDS: t = n + j / 64 + f, |f| <=
// 1/128, and five terms of the series (what is left out is below 5e-14).  Half of
// exp_f64's operations in binary64.
struct Powers {
    double at[64];
    __device__ __forceinline__ void fill() {  // then a barrier
        const int t = threadIdx.x;
        if (t < 64) at[t] = t < 33 ? exp2_series(t / 64.0) : 2.0 * exp2_series((t - 64) / 64.0);
    }
    // by: 64 log2(e) / T
    __device__ __forceinline__ double exp(double z, double m, double by) const {
        const double t = (z - m) * by;
        const double shifted = t + 0x1.8p52;  // t's nearest whole number is in its low bits
        const int k = (int)(uint32_t)__builtin_bit_cast(uint64_t, shifted);
        const double f = t - (shifted - 0x1.8p52);
        double r = 0x1.3b2ab6fba4e77p-31;
        r = fma(r, f, 0x1.c6b08d704a0bfp-23);
        r = fma(r, f, 0x1.ebfbdff82c58ep-15);
        r = fma(r, f, 0x1.62e42fefa39efp-7);
        r = fma(r, f, 1.0) * at[k & 63];
        // (2^-1010 and up: the power goes into the exponent's bits)
        const int hi = __double2hiint(r) + ((k >> 6) << 20);
        return t < kLowest * 0x1.71547652b82fep+6 ? 0.0 : __hiloint2double(hi, __double2loint(r));
    }
};

__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
__device__ __forceinline__ double wave_before_f64(double v) {  // the sum over the lanes below
    double s = v;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const double t = __shfl_up(s, o);
        if (lane_id() >= o) s += t;
    }
    s = __shfl_up(s, 1);
    return lane_id() == 0 ? 0.0 : s;
}

struct Sum {  // of a row, or of a part: the sum of exp((z - m) / T)
    double m, s;
};
__device__ __forceinline__ void raise(Sum &t, double m, double inv_t) {
    if (m > t.m) {
        t.s *= exp_f64((t.m - m) * inv_t);
        t.m = m;
    }
}
struct Choice {
    double mp, mq;   // the largest logits of the rows p and q
    double r;        // S_p / S_q as step 1 has them; 0 without q
    int32_t at, x;   // where the sequence stopped; the refused token, -1 if none
};
struct Chunk {
    double m, sp, sq;  // m: what the powers of p are below
    double a, b;       // of the entries with e_p > r e_q: the sums of e_p and of e_q
    double an, bn, lo, hi;  // of those near it the same, and the range of e_p / e_q
};
struct Verify {
    const void *target, *draft, *tokens;
    int64_t ldt, ldq, v;
    int32_t b, k, index;
    const float *u;
    double inv_t, by;  // 1 / T, 64 log2(e) / T
    float c;           // log2(e) / T
    int32_t *out, *accepted, *status;
    int32_t parts, vecs;  // of a row in step 1; vectors of a part
    int64_t chunks;
    Sum *part;       // [rows][parts]: the targets' rows, then the drafts'
    Choice *choice;  // [b]
    Chunk *chunk;    // [b][chunks]
};

// How many tokens a sequence has, the same in every lane.
__device__ __forceinline__ int drafted(const Verify &p, int64_t i) {
    bool bad = false;
    if (lane_id() < p.k)
        bad = read_token(p.tokens, p.index, i * p.k + lane_id(), p.v, nullptr) < 0;
    const unsigned long long none = __ballot(bad);
    return none ? __ffsll(none) - 1 : p.k;
}

// ----------------------------------------------------------------------------
// step 1

template <int DT>
__global__ __launch_bounds__(kBlock) void k_verify_sums(Verify p) {
    constexpr int V = Elem<DT>::kVec, kW = kBlock / kWave;
    const Work w(blockIdx.x, p.parts);
    const int64_t targets = (int64_t)p.b * (p.k + 1);
    const bool of_draft = w.i >= targets;
    const int64_t r = of_draft ? w.i - targets : w.i;
    const int per = of_draft ? p.k : p.k + 1;
    const int64_t seq = r / per;
    const int have = drafted(p, seq), j = (int)(r - seq * per);
    if (of_draft ? j >= have : j > have) return;
    const char *row = of_draft ? elem_at<DT>(p.draft, r * p.ldq) : elem_at<DT>(p.target, r * p.ldt);
    const int full = (int)(p.v / V), rem = (int)(p.v - (int64_t)full * V);
    const int first = w.part * p.vecs, end = min(full, first + p.vecs);
    // A tile's powers are above the exact ones of its maximum by shift_of, which is taken
    // out in binary64, and raising the maximum scales in binary64 too: rows that rise from
    // tile to tile would add up that rounding.
    Stat t = {-FLT_MAX, 0.0f, 0.0f};  // of a tile
    double s = 0.0, down = 1.0;
    auto raise_to = [&](float m) {
        s *= exp_f64(((double)t.m - (double)m) * ((double)p.c * 0x1.62e42fefa39efp-1));
        down = exp2_series(-(double)shift_of(m, p.c));
        t.m = m;
    };
    for (int q = first; q < end; q += kTileVecs * kBlock) {
        Tile tile = load_tile<DT, kW>(row, q, end);
        float all = kNegInf;
#pragma unroll
        for (int u = 0; u < kTileVecs; ++u) all = fmaxf(all, vec_max<DT>(tile.r[u]));
        if (__any(all > t.m)) raise_to(fmaxf(t.m, wave_max_f32(all)));
        t.s = 0.0f;
        add_vecs<DT, false>(tile.r, p.c, t);
        s = fma((double)t.s, down, s);
    }
    if (w.part == p.parts - 1 && wave_in_block() == 0) {
        const float z = tail_elem<DT, kW>(row, full, rem);
        if (__any(z > t.m)) raise_to(fmaxf(t.m, wave_max_f32(z)));
        s = fma((double)exp2_raw(power_of(z, t.m, p.c)), down, s);
    }
    __shared__ Sum part[kW];
    s = wave_sum_f64(s);
    if (lane_id() == 0) part[wave_in_block()] = Sum{t.m, s};
    __syncthreads();
    if (threadIdx.x == 0) {
        Sum a = part[0];
        for (int i = 1; i < kW; ++i) {
            Sum o = part[i];
            const double top = fmax(a.m, o.m);
            raise(a, top, p.inv_t);
            raise(o, top, p.inv_t);
            a.s += o.s;
        }
        p.part[w.i * p.parts + w.part] = a;
    }
}

// ----------------------------------------------------------------------------
// step 2

// Four sums over the wave: of s[n] in lane 16 n.  Halves, then quarters of the wave take a
// share of the sums each: 7 exchanges instead of 24.
__device__ __forceinline__ double wave_sums_f64(const double (&s)[4]) {
    const bool up = lane_id() & 32, odd = lane_id() & 16;
    double a = up ? s[2] : s[0], b = up ? s[3] : s[1];
    a += __shfl_xor(up ? s[0] : s[2], 32);
    b += __shfl_xor(up ? s[1] : s[3], 32);
    double v = odd ? b : a;
    v += __shfl_xor(odd ? a : b, 16);
#pragma unroll
    for (int o = 8; o >= 1; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

__device__ __forceinline__ double block_sum_f64(double v) {
    __shared__ double s[kBlock / kWave];
    v = wave_sum_f64(v);
    if (lane_id() == 0) s[wave_in_block()] = v;
    __syncthreads();
    v = (s[0] + s[1]) + (s[2] + s[3]);
    __syncthreads();
    return v;
}
static_assert(kBlock == 4 * kWave, "four waves");

// The exact sum of a row, by the block.
template <int DT>
__device__ double exact_sum(const Verify &p, const char *row, double m, const Powers &e) {
    constexpr int V = Elem<DT>::kVec;
    double s = 0.0;
    const int64_t whole = p.v / V;
    for (int64_t i = threadIdx.x; i < whole; i += kBlock) {
        float x[V];
        load_elems<DT, V>(row, i * V, x);
#pragma unroll
        for (int q = 0; q < V; ++q) s += e.exp((double)x[q], m, p.by);
    }
    const int64_t rest = whole * V + threadIdx.x;
    if (rest < p.v) s += e.exp((double)load1<DT>(row, rest), m, p.by);
    return block_sum_f64(s);
}

// Where sequence i stops, by one block.
template <int DT>
__device__ __forceinline__ Choice choose(const Verify &p, int64_t i, const Powers &e) {
    __shared__ Sum st[PDB_MAX_DRAFT + 1], sq[PDB_MAX_DRAFT];
    __shared__ unsigned long long stops, nears;
    const int have = drafted(p, i), wave = wave_in_block(), j = lane_id();
    const int64_t targets = (int64_t)p.b * (p.k + 1);
    // what the decision looks at, asked for before the sums are joined
    int32_t x = -1;
    float z = 0.0f, y = 0.0f, u = 0.0f;
    if (wave == 0 && j < have) {
        x = read_token(p.tokens, p.index, i * p.k + j, p.v, nullptr);
        u = p.u[i * (p.k + 1) + j];
        z = load1<DT>(p.target, (i * (p.k + 1) + j) * p.ldt + x);
        if (p.draft) y = load1<DT>(p.draft, (i * p.k + j) * p.ldq + x);
    }
    // a row's parts to a group of lanes: the targets' rows, then the drafts'
    const int group = p.parts <= 8 ? 8 : kWave, of_wave = kWave / group, l = lane_id() & (group - 1);
    const int rows = have + 1 + (p.draft ? have : 0);
    for (int r0 = wave * of_wave; r0 < rows; r0 += of_wave * (kBlock / kWave)) {
        const int r = r0 + lane_id() / group;
        const int64_t row = r <= have ? i * (p.k + 1) + r : targets + i * p.k + (r - have - 1);
        Sum t = {-FLT_MAX, 0.0};
        if (r < rows && l < p.parts) t = p.part[row * p.parts + l];
        double m = t.m;
        for (int o = group / 2; o >= 1; o >>= 1) m = fmax(m, __shfl_xor(m, o));
        raise(t, m, p.inv_t);
        for (int o = group / 2; o >= 1; o >>= 1) t.s += __shfl_xor(t.s, o);
        if (r < rows && l == 0) (r <= have ? st[r] : sq[r - have - 1]) = Sum{m, t.s};
    }
    __syncthreads();
    // a position to a lane of the first wave: whether it is refused, and whether step 1's
    // sums leave that open
    auto decide = [&](bool exact) {
        bool stop = j >= have, near = false;
        if (!stop) {
            const double px = e.exp((double)z, st[j].m, p.by) / st[j].s;
            double qx = 1.0;
            if (p.draft) qx = sq[j].s == 0.0 ? 0.0 : e.exp((double)y, sq[j].m, p.by) / sq[j].s;
            const double bar = (double)u * qx;
            stop = !(bar < px);
            near = px > 0.0 && fabs(px - bar) <= kNear * px;
        }
        const unsigned long long s = __ballot(stop), n = __ballot(near);
        if (j == 0) {
            if (!exact) nears = n;
            stops = s;
        }
    };
    if (wave == 0) decide(false);
    __syncthreads();
    // those nearer than step 1 can tell, as far as they come before the first refused
    while (true) {
        const unsigned long long n = nears, before = stops ? (stops & -stops) * 2 - 1 : ~0ull;
        if (!(n & before)) break;
        const int r = __ffsll(n & before) - 1;
        const double s = exact_sum<DT>(p, elem_at<DT>(p.target, (i * (p.k + 1) + r) * p.ldt), st[r].m, e);
        const double d = p.draft ? exact_sum<DT>(p, elem_at<DT>(p.draft, (i * p.k + r) * p.ldq), sq[r].m, e)
                                 : 0.0;
        __syncthreads();
        if (threadIdx.x == 0) {
            st[r].s = s;
            if (p.draft) sq[r].s = d;
            nears = n & ~(1ull << r);
        }
        __syncthreads();
        if (wave == 0) decide(true);
        __syncthreads();
    }
    // (with k = 64 drafted tokens there is no lane behind the last)
    const int at = stops ? __ffsll(stops) - 1 : have;
    Choice c = {st[at].m, 0.0, 0.0, at, -1};
    if (at < have) {
        c.x = read_token(p.tokens, p.index, i * p.k + at, p.v, nullptr);
        if (p.draft) {
            c.mq = sq[at].m;
            c.r = sq[at].s == 0.0 ? 0.0 : st[at].s / sq[at].s;
        }
    }
    __syncthreads();
    return c;
}

// A thread's E logits from e0 on of the rows that a sequence stopped at, -inf behind
// the row's end and in y where there is no q.
template <int DT, int E>
__device__ __forceinline__ void load_each(const Verify &p, const Choice &c, int64_t i, int64_t e0,
                                          float *x, float *y) {
    static_assert(E % Elem<DT>::kVec == 0, "whole vectors");
    const char *zt = elem_at<DT>(p.target, (i * (p.k + 1) + c.at) * p.ldt);
    const bool has_q = c.x >= 0 && p.draft;
    const char *zq = has_q ? elem_at<DT>(p.draft, (i * p.k + c.at) * p.ldq) : nullptr;
    if (e0 + E <= p.v) {
        load_elems<DT, E>(zt, e0, x);
        if (has_q) load_elems<DT, E>(zq, e0, y);
    } else {
#pragma unroll
        for (int q = 0; q < E; ++q) {
            x[q] = e0 + q < p.v ? load1<DT>(zt, e0 + q) : kNegInf;
            if (has_q) y[q] = e0 + q < p.v ? load1<DT>(zq, e0 + q) : kNegInf;
        }
    }
    if (!has_q) {
#pragma unroll
        for (int q = 0; q < E; ++q) y[q] = kNegInf;
    }
}

template <int DT>
__global__ __launch_bounds__(kBlock) void k_verify_choose(Verify p) {
    __shared__ Powers e;
    e.fill();
    __syncthreads();
    const Choice c = choose<DT>(p, blockIdx.x, e);
    if (threadIdx.x == 0) p.choice[blockIdx.x] = c;
}

// FUSED: the blocks of a sequence each find where it stops; else k_verify_choose has.
template <int DT, int E, bool FUSED>
__global__ __launch_bounds__(kBlock) void k_verify_chunks(Verify p) {
    constexpr int kChunk = kBlock * E;
    __shared__ Powers e;
    __shared__ double nears[kBlock / kWave][4];
    __shared__ double sums[kBlock / kWave][4];
    __shared__ float tops[kBlock / kWave];
    const int64_t i = blockIdx.x / p.chunks, k = blockIdx.x - i * p.chunks;
    e.fill();
    __syncthreads();
    Choice c = {0.0, 0.0, 0.0, 0, -1};
    if (p.k > 0) {
        if constexpr (FUSED)
            c = choose<DT>(p, i, e);
        else
            c = p.choice[i];
    }
    const bool has_q = c.x >= 0 && p.draft;
    const int64_t e0 = k * kChunk + threadIdx.x * E;
    float x[E], y[E];
    load_each<DT, E>(p, c, i, e0, x, y);
    if (p.k == 0) {
        float top = -FLT_MAX;
#pragma unroll
        for (int q = 0; q < E; ++q) top = fmaxf(top, x[q]);
        top = wave_max_f32(top);
        if (lane_id() == 0) tops[wave_in_block()] = top;
        __syncthreads();
        c.mp = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    }
    if ((FUSED || p.k == 0) && k == 0 && threadIdx.x == 0) p.choice[i] = c;
    double s[4] = {0.0, 0.0, 0.0, 0.0};  // e_p, e_q, and of the entries that p has more of
    double near[4] = {0.0, 0.0, __builtin_inf(), -__builtin_inf()};
#pragma unroll
    for (int q = 0; q < E; ++q) {
        const double ep = e.exp((double)x[q], c.mp, p.by);
        s[0] += ep;
        if (has_q) {
            const double eq = e.exp((double)y[q], c.mq, p.by), bar = c.r * eq;
            s[1] += eq;
            if (bar > 0.0 && fabs(ep - bar) <= kNear * bar) {
                const double ratio = ep / eq;
                near[0] += ep, near[1] += eq;
                near[2] = fmin(near[2], ratio), near[3] = fmax(near[3], ratio);
            } else if (ep > bar) {
                s[2] += ep, s[3] += eq;
            }
        }
        // (all of them at once would not fit the registers)
        if (q % 4 == 3) __builtin_amdgcn_sched_barrier(0);
    }
    const bool any = __syncthreads_or(near[3] >= 0.0);
    if (any) {
#pragma unroll
        for (int n = 0; n < 2; ++n) near[n] = wave_sum_f64(near[n]);
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) {
            near[2] = fmin(near[2], __shfl_xor(near[2], o));
            near[3] = fmax(near[3], __shfl_xor(near[3], o));
        }
        if (lane_id() == 0)
            for (int n = 0; n < 4; ++n) nears[wave_in_block()][n] = near[n];
    }
    if (has_q) {
        const double v = wave_sums_f64(s);
        if (lane_id() % 16 == 0) sums[wave_in_block()][lane_id() / 16] = v;
    } else {
        s[0] = wave_sum_f64(s[0]);
        if (lane_id() < 4) sums[wave_in_block()][lane_id()] = lane_id() == 0 ? s[0] : 0.0;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        double t[4];
        for (int n = 0; n < 4; ++n)
            t[n] = (sums[0][n] + sums[1][n]) + (sums[2][n] + sums[3][n]);
        if (any) {
            for (int n = 0; n < 2; ++n)
                near[n] = (nears[0][n] + nears[1][n]) + (nears[2][n] + nears[3][n]);
            near[2] = fmin(fmin(nears[0][2], nears[1][2]), fmin(nears[2][2], nears[3][2]));
            near[3] = fmax(fmax(nears[0][3], nears[1][3]), fmax(nears[2][3], nears[3][3]));
        }
        p.chunk[i * p.chunks + k] = Chunk{c.mp, t[0], t[1], t[2], t[3], near[0], near[1], near[2], near[3]};
    }
}

// ----------------------------------------------------------------------------
// step 3

// The sum over the threads below this one, and over all.
__device__ __forceinline__ double block_before_f64(double v, double *all) {
    __shared__ double s[kBlock / kWave];
    const double before = wave_before_f64(v);
    if (lane_id() == kWave - 1) s[wave_in_block()] = before + v;
    __syncthreads();
    double base = 0.0, sum = 0.0;
#pragma unroll
    for (int w = 0; w < kBlock / kWave; ++w) {
        if (w == wave_in_block()) base = sum;
        sum += s[w];
    }
    __syncthreads();
    *all = sum;
    return base + before;
}
// The smallest of the threads' a and the largest of their b, in every thread.
__device__ __forceinline__ void block_ends_i64(int64_t &a, int64_t &b) {
    __shared__ int64_t s[2][kBlock / kWave];
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
        a = min(a, (int64_t)__shfl_xor((long long)a, o));
        b = max(b, (int64_t)__shfl_xor((long long)b, o));
    }
    if (lane_id() == 0) s[0][wave_in_block()] = a, s[1][wave_in_block()] = b;
    __syncthreads();
    a = min(min(s[0][0], s[0][1]), min(s[0][2], s[0][3]));
    b = max(max(s[1][0], s[1][1]), max(s[1][2], s[1][3]));
    __syncthreads();
}

// A thread's E weights from e0 on: of what the refused token leaves, or of p.
template <int DT, int E>
__device__ __forceinline__ void weights(const Verify &p, const Choice &c, int64_t i, int64_t e0, double m,
                                        double r, bool residual, const Powers &e, double *w) {
    float x[E], y[E];
    load_each<DT, E>(p, c, i, e0, x, y);
#pragma unroll
    for (int q = 0; q < E; ++q) {
        w[q] = e.exp((double)x[q], m, p.by);
        if (!residual) continue;
        if (p.draft)
            w[q] = fmax(w[q] - r * e.exp((double)y[q], c.mq, p.by), 0.0);
        else if (e0 + q == c.x)
            w[q] = 0.0;
    }
}

template <int DT, int E>
__global__ __launch_bounds__(kBlock) void k_verify_pick(Verify p) {
    constexpr int kChunk = kBlock * E;
    __shared__ Powers e;
    __shared__ int todo, list[kBlock];
    const int64_t i = blockIdx.x;
    Chunk *chunk = p.chunk + i * p.chunks;
    const int t = threadIdx.x;
    // Up to 64 chunks are a wave's, each wave going over all of them, which spares the
    // block's waits; else a stretch of them is a thread's.  Where that is one, it stays in
    // registers.
    const bool narrow = p.chunks <= kWave;
    const int id = narrow ? lane_id() : t, ids = narrow ? kWave : kBlock;
    const int64_t each = (p.chunks + ids - 1) / ids, k0 = min(id * each, p.chunks),
                  k1 = min(k0 + each, p.chunks);
    // all that is known from the start is asked for first
    __shared__ double redone[kBlock];
    const bool single = each == 1;
    Chunk own = {};
    if (single && k0 < k1) own = chunk[k0];
    const double number = (double)p.u[i * (p.k + 1) + p.k];
    const Choice c = p.k == 0 ? Choice{0.0, 0.0, 0.0, 0, -1} : p.choice[i];
    int32_t token = -1;
    if (t < p.k) token = read_token(p.tokens, p.index, i * p.k + t, p.v, nullptr);
    const int have = drafted(p, i);
    e.fill();
    __syncthreads();
    auto at = [&](int64_t k) { return single ? own : chunk[k]; };
    auto sum_of = [&](double v) { return narrow ? wave_sum_f64(v) : block_sum_f64(v); };
    auto before_of = [&](double v, double *all) {
        if (!narrow) return block_before_f64(v, all);
        const double b = wave_before_f64(v);
        *all = __shfl(b + v, kWave - 1);
        return b;
    };
    // the row's maximum, where chunks have their own
    double m = c.mp;
    if (p.k == 0) {
        __shared__ double tops[kBlock / kWave];
        m = -FLT_MAX;
        for (int64_t k = k0; k < k1; ++k) m = fmax(m, at(k).m);
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) m = fmax(m, __shfl_xor(m, o));
        if (!narrow) {
            if (lane_id() == 0) tops[wave_in_block()] = m;
            __syncthreads();
            m = fmax(fmax(tops[0], tops[1]), fmax(tops[2], tops[3]));
        }
    }
    auto mass_p = [&](const Chunk &h) { return p.k == 0 ? h.sp * e.exp(h.m, m, p.by) : h.sp; };
    double sum = 0.0, sq = 0.0, all = 0.0;
    for (int64_t k = k0; k < k1; ++k) sum += mass_p(at(k)), sq += at(k).sq;
    const double before_p = before_of(sum, &all);
    bool residual = c.x >= 0;
    double r = 0.0, before = before_p;
    const double all_p = all;
    if (residual) {
        if (p.draft) {
            sq = sum_of(sq);
            r = sq == 0.0 ? 0.0 : all_p / sq;
            if (!(sq >= 0.0)) residual = false;  // the draft's row has no distribution
        }
    }
    auto again = [&](int64_t k) {
        return p.draft ? at(k).lo < r && r < at(k).hi : c.x >= k * kChunk && c.x < (k + 1) * kChunk;
    };
    if (residual) {
        // the chunks that step 2 left open, and without q that of the token, a turn of them
        // at a time
        for (int64_t a = 0; a < each; ++a) {
            if (t == 0) todo = 0;
            __syncthreads();
            if (t < ids && k0 + a < k1 && again(k0 + a)) list[atomicAdd(&todo, 1)] = t;
            __syncthreads();
            for (int n = 0; n < todo; ++n) {
                const int64_t k = list[n] * each + a;
                double w[E], s = 0.0;
                weights<DT, E>(p, c, i, k * kChunk + t * E, m, r, true, e, w);
#pragma unroll
                for (int q = 0; q < E; ++q) s += w[q];
                s = block_sum_f64(s);
                if (t == 0) {
                    if (single)
                        redone[k] = s;
                    else
                        chunk[k].m = s;  // (read for k = 0 only)
                }
            }
            __syncthreads();
        }
    }
    auto mass = [&](int64_t k) -> double {
        const Chunk h = at(k);
        if (!residual) return mass_p(h);
        if (again(k)) return single ? redone[k] : h.m;
        if (!p.draft) return h.sp;
        const double near = r <= h.lo ? h.an - r * h.bn : 0.0;
        return fmax(h.a - r * h.b, 0.0) + fmax(near, 0.0);
    };
    if (residual) {
        double s = 0.0;
        for (int64_t k = k0; k < k1; ++k) s += mass(k);
        before = before_of(s, &all);
        if (!(all > 0.0)) {
            residual = false;
            before = before_p;
            all = all_p;
        }
    }
    const double bar = number * all;
    constexpr int64_t kNone = INT64_MAX;
    int64_t found = kNone, last = -1;
    double run = before, base = before;
    for (int64_t k = k0; k < k1; ++k) {
        const double w = mass(k);
        if (found == kNone && w > 0.0 && run + w > bar) found = k, base = run;
        run += w;
        if (w > 0.0) last = k;
    }
    int64_t chunk_found = found, chunk_last = last;
    if (narrow) {
        const unsigned long long f = __ballot(found != kNone), l = __ballot(last >= 0);
        chunk_found = f ? __ffsll(f) - 1 : kNone;
        chunk_last = l ? 63 - __clzll(l) : -1;
        base = __shfl(base, f ? (int)chunk_found : 0);
    } else {
        __shared__ double s_base;
        block_ends_i64(chunk_found, chunk_last);
        if (found == chunk_found && found != kNone) s_base = base;
        __syncthreads();
        base = s_base;
    }
    int64_t next = -1;
    if (chunk_last >= 0 && all_p >= 0.0) {  // (not of a row with a NaN)
        // a sum that none exceeds: the last weight above 0
        const int64_t k = chunk_found != kNone ? chunk_found : chunk_last;
        const double limit = chunk_found != kNone ? bar : __builtin_inf();
        double w[E], s = 0.0, total;
        const int64_t e0 = k * kChunk + t * E;
        weights<DT, E>(p, c, i, e0, m, r, residual, e, w);
#pragma unroll
        for (int q = 0; q < E; ++q) s += w[q];
        double sofar = (chunk_found != kNone ? base : 0.0) + block_before_f64(s, &total);
        int64_t hit = kNone, end = -1;
#pragma unroll
        for (int q = 0; q < E; ++q) {
            sofar += w[q];
            // (the sums before two threads differ in their last bits from one thread's
            // own: an entry of weight 0 may seem to pass the bar)
            if (hit == kNone && w[q] > 0.0 && sofar > limit) hit = e0 + q;
            if (w[q] > 0.0) end = e0 + q;
        }
        block_ends_i64(hit, end);
        // the chunk's sum and its entries' may differ in their last bits
        next = hit != kNone ? hit : end;
    }
    if (t <= p.k) p.out[i * (p.k + 1) + t] = t < c.at ? token : t == c.at ? (int32_t)next : -1;
    static_assert(PDB_MAX_DRAFT < kBlock, "a place to a thread");
    if (t == 0 && have < p.k) read_token(p.tokens, p.index, i * p.k + have, p.v, p.status);
    if (t == 0) p.accepted[i] = c.at;
}

// ----------------------------------------------------------------------------
// host side

// Step 1's blocks: enough for an even load, of a tile at least.
constexpr int64_t kWantParts = 4096;

struct Space {
    int64_t rows, chunks;
    size_t choice, chunk, total;  // offsets in the workspace
};
Space space_of(int64_t b, int32_t k, int64_t v) {
    Space s;
    // (rows are cut up to kWantParts parts in all, and a row has one at least)
    s.rows = b * (2 * k + 1);
    s.chunks = cdiv(std::max<int64_t>(v, 1), kBlock * each_of(k));
    s.choice = (size_t)align_up((s.rows + kWantParts) * (int64_t)sizeof(Sum));
    s.chunk = s.choice + (size_t)align_up(b * (int64_t)sizeof(Choice));
    s.total = s.chunk + (size_t)align_up(b * s.chunks * (int64_t)sizeof(Chunk));
    return s;
}

// The call for `count` of its sequences, from i on.
Verify from_sequence(Verify p, int dtype, int64_t i, int64_t count) {
    p.b = (int32_t)count;
    p.target = static_cast<const char *>(p.target) + i * (p.k + 1) * p.ldt * dtype_size(dtype);
    if (p.draft) p.draft = static_cast<const char *>(p.draft) + i * p.k * p.ldq * dtype_size(dtype);
    if (p.k > 0) p.tokens = static_cast<const char *>(p.tokens) + i * p.k * (p.index == PDB_I64 ? 8 : 4);
    p.u += i * (p.k + 1);
    p.out += i * (p.k + 1);
    p.accepted += i;
    return p;
}

template <int DT>
int run_verify(Verify p, hipStream_t stream) {
    if (p.k > 0) {
        const int64_t rows = (int64_t)p.b * (p.k + 1 + (p.draft ? p.k : 0));
        const int64_t tile = kTileVecs * kBlock;
        const int64_t tiles = std::max<int64_t>(cdiv(p.v / Elem<DT>::kVec, tile), 1);
        const int64_t parts = std::min(std::min(kWantParts / rows, tiles), kMostParts);
        const int64_t of_part = cdiv(tiles, std::max<int64_t>(parts, 1));
        p.parts = (int32_t)cdiv(tiles, of_part);
        p.vecs = (int32_t)std::min<int64_t>(of_part * tile, INT32_MAX / 2);
        k_verify_sums<DT><<<(unsigned)(rows * p.parts), kBlock, 0, stream>>>(p);
        PDB_LAUNCHED();
    }
    // Where a sequence stops is found by each block of its chunks while they are few,
    // which saves a launch (64 of them: 20 us against 22, 575: 28 against 30), else once
    // (2,048: 59 against 62; 4,096: 70 against 73).
    const unsigned blocks = (unsigned)(p.b * p.chunks), rows = (unsigned)p.b;
    if (p.k == 0) {
        constexpr int E = each_of(0);
        k_verify_chunks<DT, E, true><<<blocks, kBlock, 0, stream>>>(p);
        PDB_LAUNCHED();
        k_verify_pick<DT, E><<<rows, kBlock, 0, stream>>>(p);
    } else {
        constexpr int E = each_of(1);
        if (blocks <= 1024) {
            k_verify_chunks<DT, E, true><<<blocks, kBlock, 0, stream>>>(p);
        } else {
            k_verify_choose<DT><<<rows, kBlock, 0, stream>>>(p);
            PDB_LAUNCHED();
            k_verify_chunks<DT, E, false><<<blocks, kBlock, 0, stream>>>(p);
        }
        PDB_LAUNCHED();
        k_verify_pick<DT, E><<<rows, kBlock, 0, stream>>>(p);
    }
    PDB_LAUNCHED();
    return PDB_OK;
}

}  // namespace
}  // namespace pdbk

using namespace pdbk;

extern "C" int pdb_draft_verify_workspace_bytes(int64_t b, int32_t k, int64_t v, size_t *bytes) {
    if (!bytes || b < 0 || k < 0 || v < 0) return PDB_ERR_INVALID_ARG;
    if (k > PDB_MAX_DRAFT || v > INT32_MAX || b * (k + 1) > INT32_MAX || b > INT32_MAX)
        return PDB_ERR_UNSUPPORTED;
    *bytes = space_of(b, k, v).total;
    return PDB_OK;
}

extern "C" int pdb_draft_verify(const void *target, int64_t ldt, const void *draft, int64_t ldq,
                                int dtype, int64_t b, int32_t k, int64_t v, const void *tokens,
                                int index, const float *u, double temp, int32_t *out,
                                int32_t *accepted, int32_t *status, void *ws, size_t ws_bytes,
                                hipStream_t stream) {
    if (b < 0 || k < 0 || v <= 0 || !(temp > 0.0) || !good_temp((float)temp)) return PDB_ERR_INVALID_ARG;
    if (k > PDB_MAX_DRAFT || b > INT32_MAX || b * (k + 1) > INT32_MAX) return PDB_ERR_UNSUPPORTED;
    if (int e = check_matrix(target, dtype, ldt, b * (k + 1), v)) return e;
    if (draft)
        if (int e = check_matrix(draft, dtype, ldq, b * k, v)) return e;
    if (k > 0)
        if (int e = check_tokens(tokens, index, b * k)) return e;
    if (b == 0) return PDB_OK;
    if (!u || !out || !accepted || !aligned_to(u, 4) || !aligned_to(out, 4) || !aligned_to(accepted, 4))
        return PDB_ERR_INVALID_ARG;
    const Space sp = space_of(b, k, v);
    if (!ws || !aligned_to(ws, 8) || ws_bytes < sp.total) return PDB_ERR_WORKSPACE;
    if (b * sp.chunks > INT32_MAX) return PDB_ERR_UNSUPPORTED;
    Verify all = {};
    all.target = target, all.draft = k > 0 ? draft : nullptr, all.tokens = tokens, all.ldt = ldt, all.ldq = ldq;
    all.v = v, all.k = k, all.index = index, all.u = u, all.inv_t = 1.0 / temp;
    all.by = all.inv_t * 0x1.71547652b82fep+6;
    all.c = (float)(0x1.71547652b82fep+0 / temp);
    all.out = out, all.accepted = accepted, all.status = status, all.chunks = sp.chunks;
    char *at = static_cast<char *>(ws);
    all.part = reinterpret_cast<Sum *>(at);
    all.choice = reinterpret_cast<Choice *>(at + sp.choice);
    all.chunk = reinterpret_cast<Chunk *>(at + sp.chunk);
    // As many sequences at once as a launch has blocks for, one behind another in the same
    // workspace (their parts in step 1: kWantParts at most, or one a row).
    const int64_t at_once = (kMostBlocks - kWantParts) / std::max<int64_t>(sp.chunks, 2 * k + 1);
    return with_dtype(dtype, [&](auto dt) -> int {
        for (int64_t i = 0; i < b; i += at_once) {
            const Verify p = from_sequence(all, dtype, i, std::min(at_once, b - i));
            if (int e = run_verify<decltype(dt)::value>(p, stream)) return e;
        }
        return PDB_OK;
    });
}
