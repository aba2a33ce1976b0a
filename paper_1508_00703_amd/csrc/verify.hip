// Verification of drafted tokens against the target's probabilities, from given random
// numbers; with nothing drafted, the drawing of a token (gfx950, wave64).
//
// The answers are choices: whether u q(x) < p(x), and where a running sum over the
// vocabulary passes u R.  In binary32 a sum over 131,072 entries is off by 1e-6 and
// more, as much as many an entry has; so exponentials, probabilities and sums are in
// binary64, which gfx950's vector unit multiplies and adds at half the rate of binary32.
//
// Three launches: every row's maximum and sum (rows in parts where they are few); then,
// for the row at which each sequence stopped, the weights' sum of every chunk of
// kChunk entries; then the chunk and the entry in it that the random number picks.
#include "pdb_softmax.h"

namespace pdbk {
namespace {

constexpr int kEach = 16;               // consecutive entries of a thread
constexpr int kChunk = kBlock * kEach;  // 4096
constexpr double kLowest = -700.0;      // powers below this count as 0

// e^y for y <= 0 (0 below kLowest, NaN of NaN): 2^n 2^f by the series of e^(f ln 2)
// through f^12, |f| <= 1/2; what is left out is below 2e-16.
__device__ __forceinline__ double exp_f64(double y) {
    const double t = y * 0x1.71547652b82fep+0;
    const double n = __builtin_rint(t);
    const double f = t - n;
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
    r = fma(r, f, 1.0);
    return y < kLowest ? 0.0 : __builtin_amdgcn_ldexp(r, (int)n);
}

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
__device__ __forceinline__ double weight(float z, double m, double inv_t) {
    return exp_f64(((double)z - m) * inv_t);
}

struct Verify {
    const void *target, *draft, *tokens;
    int64_t ldt, ldq, v;
    int32_t b, k, index;
    const float *u;
    double inv_t;
    int32_t *out, *accepted, *status;
    Parts cut;
    int64_t chunks;
    Sum *part;       // [rows][parts]: the targets' rows, then the drafts'
    struct Choice *choice;  // [b]
    double2 *mass;   // [b][chunks]: of max(p - q, 0), and of p
};
struct Choice {
    double mp, ip, mq, iq;  // maximum and 1 / sum of the rows p and q
    int32_t at, x;          // where the sequence stopped; the refused token, -1 if none
};

// How many tokens a sequence has, the same in every lane.
__device__ __forceinline__ int drafted(const Verify &p, int64_t i) {
    bool bad = false;
    if (lane_id() < p.k)
        bad = read_token(p.tokens, p.index, i * p.k + lane_id(), p.v, nullptr) < 0;
    const unsigned long long none = __ballot(bad);
    return none ? __ffsll((unsigned long long)none) - 1 : p.k;
}

template <int DT>
__global__ __launch_bounds__(kBlock) void k_verify_sums(Verify p) {
    constexpr int V = Elem<DT>::kVec;
    const Work w(blockIdx.x, p.cut.parts);
    const int64_t targets = (int64_t)p.b * (p.k + 1);
    const bool of_draft = w.i >= targets;
    const int64_t r = of_draft ? w.i - targets : w.i;
    const int per = of_draft ? p.k : p.k + 1;
    const int64_t seq = r / per;
    const int have = drafted(p, seq), j = (int)(r - seq * per);
    if (of_draft ? j >= have : j > have) return;
    const char *row = of_draft ? elem_at<DT>(p.draft, r * p.ldq) : elem_at<DT>(p.target, r * p.ldt);
    const int full = (int)(p.v / V), rem = (int)(p.v - (int64_t)full * V);
    const int first = w.part * p.cut.vecs;
    const int end = std::min<int64_t>(full, (int64_t)first + p.cut.vecs);
    const bool last = w.part == p.cut.parts - 1;
    float m = -FLT_MAX;
    double s = 0.0;
    for (int q = first; q < end; q += kTileVecs * kBlock) {
        const Tile tile = load_tile<DT, kBlock / kWave>(row, q, end);
        float all = kNegInf;
#pragma unroll
        for (int u = 0; u < kTileVecs; ++u) all = fmaxf(all, vec_max<DT>(tile.r[u]));
        if (__any(all > m)) {
            const float up = fmaxf(m, wave_max_f32(all));
            s *= exp_f64(((double)m - (double)up) * p.inv_t);
            m = up;
        }
#pragma unroll
        for (int u = 0; u < kTileVecs; ++u) {
            float x[V];
            unpack<DT>(tile.r[u], x);
#pragma unroll
            for (int e = 0; e < V; ++e) s += weight(x[e], m, p.inv_t);
        }
    }
    if (last && wave_in_block() == 0) {
        const float z = tail_elem<DT, kBlock / kWave>(row, full, rem);
        if (__any(z > m)) {
            const float up = fmaxf(m, wave_max_f32(z));
            s *= exp_f64(((double)m - (double)up) * p.inv_t);
            m = up;
        }
        s += weight(z, m, p.inv_t);
    }
    __shared__ Sum part[kBlock / kWave];
    s = wave_sum_f64(s);
    if (lane_id() == 0) part[wave_in_block()] = Sum{m, s};
    __syncthreads();
    if (threadIdx.x == 0) {
        Sum t = part[0];
        for (int k = 1; k < kBlock / kWave; ++k) {
            Sum o = part[k];
            const double top = fmax(t.m, o.m);
            raise(t, top, p.inv_t);
            raise(o, top, p.inv_t);
            t.s += o.s;
        }
        p.part[w.i * p.cut.parts + w.part] = t;
    }
}

// A row's maximum and sum from its parts', the same in every lane.
__device__ __forceinline__ Sum join_sums(const Verify &p, int64_t row) {
    Sum t = {-FLT_MAX, 0.0};
    if (lane_id() < p.cut.parts) t = p.part[row * p.cut.parts + lane_id()];
    double m = t.m;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) m = fmax(m, __shfl_xor(m, o));
    raise(t, m, p.inv_t);
    return {m, wave_sum_f64(t.s)};
}

// Where sequence i stops, by one block.
template <int DT>
__device__ __forceinline__ Choice choose(const Verify &p, int64_t i) {
    __shared__ Sum st[PDB_MAX_DRAFT + 1], sq[PDB_MAX_DRAFT];
    __shared__ Choice c;
    const int have = drafted(p, i), wave = wave_in_block();
    const int64_t targets = (int64_t)p.b * (p.k + 1);
    for (int j = wave; j <= have; j += kBlock / kWave) {
        const Sum s = join_sums(p, i * (p.k + 1) + j);
        if (lane_id() == 0) st[j] = s;
        if (j < have && p.draft) {
            const Sum d = join_sums(p, targets + i * p.k + j);
            if (lane_id() == 0) sq[j] = d;
        }
    }
    __syncthreads();
    if (wave == 0) {
        const int j = lane_id();
        bool stop = j >= have;
        int32_t x = -1;
        if (!stop) {
            x = read_token(p.tokens, p.index, i * p.k + j, p.v, nullptr);
            const float z = load1<DT>(p.target, (i * (p.k + 1) + j) * p.ldt + x);
            const double px = weight(z, st[j].m, p.inv_t) / st[j].s;
            double qx = 1.0;
            if (p.draft) {
                const float zq = load1<DT>(p.draft, (i * p.k + j) * p.ldq + x);
                qx = sq[j].s == 0.0 ? 0.0 : weight(zq, sq[j].m, p.inv_t) / sq[j].s;
            }
            stop = !((double)p.u[i * (p.k + 1) + j] * qx < px);
        }
        const unsigned long long stops = __ballot(stop);
        const int at = stops ? __ffsll((unsigned long long)stops) - 1 : have;
        x = __shfl(x, at & (kWave - 1));
        if (j == 0) {
            c.at = at;
            c.x = at < have ? x : -1;
            const Sum s = st[at];
            c.mp = s.m;
            c.ip = s.s == 0.0 ? 0.0 : 1.0 / s.s;
            c.mq = c.iq = 0.0;
            if (at < have && p.draft) {
                c.mq = sq[at].m;
                c.iq = sq[at].s == 0.0 ? 0.0 : 1.0 / sq[at].s;
            }
        }
    }
    __syncthreads();
    return c;
}

// A thread's kEach entries from e0 on: p, and what a refused token leaves of it.
template <int DT>
__device__ __forceinline__ void weights(const Verify &p, const Choice &c, int64_t i, int64_t e0,
                                        double *wp, double *wr) {
    constexpr int V = Elem<DT>::kVec;
    const char *zt = elem_at<DT>(p.target, (i * (p.k + 1) + c.at) * p.ldt);
    const bool has_q = c.x >= 0 && p.draft;
    const char *zq = has_q ? elem_at<DT>(p.draft, (i * p.k + c.at) * p.ldq) : nullptr;
    float x[kEach], y[kEach];
    if (e0 + kEach <= p.v) {
        load_elems<DT, kEach>(zt, e0, x);
        if (has_q) load_elems<DT, kEach>(zq, e0, y);
    } else {
#pragma unroll
        for (int q = 0; q < kEach; ++q) {
            x[q] = e0 + q < p.v ? load1<DT>(zt, e0 + q) : kNegInf;
            y[q] = has_q && e0 + q < p.v ? load1<DT>(zq, e0 + q) : kNegInf;
        }
    }
    static_assert(kEach % V == 0, "whole vectors");
#pragma unroll
    for (int q = 0; q < kEach; ++q) {
        // (a row of nothing but -inf: 1 / sum is 0, and no weight is above 0)
        wp[q] = weight(x[q], c.mp, p.inv_t) * c.ip;
        double r = 0.0;
        if (c.x >= 0) {
            r = has_q ? wp[q] - weight(y[q], c.mq, p.inv_t) * c.iq : (e0 + q == c.x ? 0.0 : wp[q]);
            r = r > 0.0 ? r : 0.0;
        }
        wr[q] = r;
    }
}

template <int DT>
__global__ __launch_bounds__(kBlock) void k_verify_mass(Verify p) {
    const int64_t i = blockIdx.x / p.chunks, k = blockIdx.x - i * p.chunks;
    const Choice c = choose<DT>(p, i);
    if (k == 0 && threadIdx.x == 0) p.choice[i] = c;
    double wp[kEach], wr[kEach], sp = 0.0, sr = 0.0;
    weights<DT>(p, c, i, k * kChunk + threadIdx.x * kEach, wp, wr);
#pragma unroll
    for (int q = 0; q < kEach; ++q) sp += wp[q], sr += wr[q];
    sp = wave_sum_f64(sp);
    sr = wave_sum_f64(sr);
    __shared__ double2 s[kBlock / kWave];
    if (lane_id() == 0) s[wave_in_block()] = double2{sr, sp};
    __syncthreads();
    if (threadIdx.x == 0) {
        double2 t = s[0];
        for (int w = 1; w < kBlock / kWave; ++w) t.x += s[w].x, t.y += s[w].y;
        p.mass[i * p.chunks + k] = t;
    }
}

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
__device__ __forceinline__ int64_t block_min_i64(int64_t v) {
    __shared__ int64_t s[kBlock / kWave];
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v = min(v, (int64_t)__shfl_xor((long long)v, o));
    if (lane_id() == 0) s[wave_in_block()] = v;
    __syncthreads();
    v = min(min(s[0], s[1]), min(s[2], s[3]));
    __syncthreads();
    return v;
}
static_assert(kBlock == 4 * kWave, "four waves");

template <int DT>
__global__ __launch_bounds__(kBlock) void k_verify_pick(Verify p) {
    const int64_t i = blockIdx.x;
    const Choice c = p.choice[i];
    const double2 *mass = p.mass + i * p.chunks;
    const int t = threadIdx.x;
    // the residual, unless it is 0 throughout; a stretch of chunks to a thread
    const int64_t each = (p.chunks + kBlock - 1) / kBlock, k0 = min(t * each, p.chunks),
                  k1 = min(k0 + each, p.chunks);
    double all = 0.0, before = 0.0;
    bool residual = c.x >= 0;
    if (residual) {
        double s = 0.0;
        for (int64_t k = k0; k < k1; ++k) s += mass[k].x;
        before = block_before_f64(s, &all);
        residual = all > 0.0;
    }
    if (!residual) {
        double s = 0.0;
        for (int64_t k = k0; k < k1; ++k) s += mass[k].y;
        before = block_before_f64(s, &all);
    }
    const double bar = (double)p.u[i * (p.k + 1) + p.k] * all;
    constexpr int64_t kNone = INT64_MAX;
    int64_t found = kNone, last = -1;
    double run = before, base = before;
    for (int64_t k = k0; k < k1; ++k) {
        const double m = residual ? mass[k].x : mass[k].y;
        if (found == kNone && m > 0.0 && run + m > bar) found = k, base = run;
        run += m;
        if (m > 0.0) last = k;
    }
    const int64_t chunk_found = block_min_i64(found);
    const int64_t chunk_last = -block_min_i64(-last);
    __shared__ double s_base;
    if (found == chunk_found && found != kNone) s_base = base;
    __syncthreads();
    int64_t next = -1;
    if (chunk_last >= 0) {
        // a sum that none exceeds: the last weight above 0
        const int64_t k = chunk_found != kNone ? chunk_found : chunk_last;
        const double limit = chunk_found != kNone ? bar : __builtin_inf();
        double wp[kEach], wr[kEach], s = 0.0, sum;
        const int64_t e0 = k * kChunk + t * kEach;
        weights<DT>(p, c, i, e0, wp, wr);
#pragma unroll
        for (int q = 0; q < kEach; ++q) {
            if (residual) wp[q] = wr[q];
            s += wp[q];
        }
        double sofar = (chunk_found != kNone ? s_base : 0.0) + block_before_f64(s, &sum);
        int64_t hit = kNone, end = -1;
#pragma unroll
        for (int q = 0; q < kEach; ++q) {
            sofar += wp[q];
            // (the sums before two threads differ in their last bits from one thread's
            // own: an entry of weight 0 may seem to pass the bar)
            if (hit == kNone && wp[q] > 0.0 && sofar > limit) hit = e0 + q;
            if (wp[q] > 0.0) end = e0 + q;
        }
        const int64_t a = block_min_i64(hit), z = -block_min_i64(-end);
        // the chunk's sum and its entries' may differ in their last bits
        next = a != kNone ? a : z;
    }
    for (int j = t; j <= p.k; j += kBlock) {
        int32_t o = -1;
        if (j < c.at) o = read_token(p.tokens, p.index, i * p.k + j, p.v, nullptr);
        if (j == c.at) o = (int32_t)next;
        p.out[i * (p.k + 1) + j] = o;
    }
    const int have = drafted(p, i);
    if (t == 0 && have < p.k) read_token(p.tokens, p.index, i * p.k + have, p.v, p.status);
    if (t == 0) p.accepted[i] = c.at;
}

struct Space {
    Parts cut;
    int64_t rows, chunks;
    size_t parts, choice, total;  // offsets in the workspace
};
Space space_of(int64_t b, int32_t k, int64_t v) {
    Space s;
    // rows are cut only up to kWantBlocks parts in all
    s.rows = b * (2 * k + 1);
    s.chunks = cdiv(std::max<int64_t>(v, 1), kChunk);
    s.parts = (size_t)align_up(std::max(s.rows, kWantBlocks) * (int64_t)sizeof(Sum));
    s.choice = s.parts + (size_t)align_up(b * (int64_t)sizeof(Choice));
    s.total = s.choice + (size_t)align_up(b * s.chunks * (int64_t)sizeof(double2));
    return s;
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
                                int index, const float *u, float temp, int32_t *out,
                                int32_t *accepted, int32_t *status, void *ws, size_t ws_bytes,
                                hipStream_t stream) {
    if (b < 0 || k < 0 || v <= 0 || !good_temp(temp)) return PDB_ERR_INVALID_ARG;
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
    if (!ws || ws_bytes < sp.total) return PDB_ERR_WORKSPACE;
    if (b * sp.chunks > INT32_MAX) return PDB_ERR_UNSUPPORTED;
    Verify p = {};
    p.target = target, p.draft = k > 0 ? draft : nullptr, p.tokens = tokens, p.ldt = ldt, p.ldq = ldq;
    p.v = v, p.b = (int32_t)b, p.k = k, p.index = index, p.u = u, p.inv_t = 1.0 / (double)temp;
    p.out = out, p.accepted = accepted, p.status = status, p.chunks = sp.chunks;
    char *at = static_cast<char *>(ws);
    p.part = reinterpret_cast<Sum *>(at);
    p.choice = reinterpret_cast<Choice *>(at + sp.parts);
    p.mass = reinterpret_cast<double2 *>(at + sp.choice);
    return with_dtype(dtype, [&](auto dt) -> int {
        constexpr int DT = decltype(dt)::value;
        const int64_t rows = b * (k + 1) + (p.draft ? b * k : 0);
        p.cut = cut_rows(rows, v, Elem<DT>::kVec, kMostParts);
        if (rows * p.cut.parts > INT32_MAX) return PDB_ERR_UNSUPPORTED;
        k_verify_sums<DT><<<(unsigned)(rows * p.cut.parts), kBlock, 0, stream>>>(p);
        k_verify_mass<DT><<<(unsigned)(b * p.chunks), kBlock, 0, stream>>>(p);
        k_verify_pick<DT><<<(unsigned)b, kBlock, 0, stream>>>(p);
        PDB_LAUNCHED();
        return PDB_OK;
    });
}
