// Distillation from a teacher's top logits (gfx950, wave64): the loss of every row
// and its gradient by the row's logits.
//
//   loss = w sum_j p_j (log p_j - log q_{id_j}),  dz = (w / T) (q - p at the ids)
//
// The gradient needs the row's sum before its first element, so the logits are read
// twice -- unless a row stays on chip.  It does in registers: 16 vectors a thread, as
// they are stored, with one to sixteen waves to a row, which holds rows of up to
// 131,072 16-bit logits and leaves 16 waves on every compute unit.  The floor is then
// one read and one write (4,096 rows of 131,072 bf16: 436 us, 4.9 TB/s).  Longer rows,
// and rows too few to fill the card, go the other way: a kernel for the statistics of
// their parts and one for the gradient (1,024 rows of 151,936 bf16: 210 us, 94 and 114,
// where one read and one write would be 121; of 262,144: 337; 64 rows of 131,072: 20).
#include "pdb_softmax.h"

namespace pdbk {
namespace {

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

// A row's teacher: ids, log probabilities and the student's logits there.
template <int K>
struct TeacherLds {
    int32_t id[K];
    float lp[K], z[K];
    int some;  // whether the teacher has a distribution
};

__device__ __forceinline__ float load_teacher(const DistillArgs &p, int64_t at) {
    if (p.teacher_dtype == PDB_F32) return load1<PDB_F32>(p.teacher, at);
    return p.teacher_dtype == PDB_BF16 ? load1<PDB_BF16>(p.teacher, at)
                                       : load1<PDB_F16>(p.teacher, at);
}

// One wave fills L; the others see it after the team's next barrier.  An id out of range
// is noted unless the row's weight is 0: such rows come here too where others' loads are
// under way (to leave them out took 38.2 -> 39.6 us for 4,200 rows of 8,000 bf16).
template <int DT, int K>
__device__ __forceinline__ void teacher_row(const DistillArgs &p, int64_t i, const char *row,
                                            TeacherLds<K> &L) {
    Stat t = empty_stat();
    float top = kNegInf;
    for (int j = lane_id(); j < p.k; j += kWave) {
        int32_t id = p.ids[i * p.k + j];
        if (id >= p.v) {
            if (p.status && row_weight(p, i) != 0.0f) *p.status = PDB_ERR_INVALID_ARG;
            id = -1;
        }
        const float y = id < 0 ? kNegInf : load_teacher(p, i * p.k + j);
        L.id[j] = id < 0 ? -1 : id;
        L.lp[j] = y;
        L.z[j] = id < 0 ? 0.0f : load1<DT>(row, id);
        top = fmaxf(top, y);
    }
    t.m = fmaxf(t.m, wave_max_f32(top));
    for (int j = lane_id(); j < p.k; j += kWave) t.s += exp2_raw(power_of(L.lp[j], t.m, p.c));
    t = team_stat<1>(t, p.c);
    const float ls = log_sum(t, p.c);
    for (int j = lane_id(); j < p.k; j += kWave) L.lp[j] = (L.lp[j] - t.m) * p.inv_t - ls;
    if (lane_id() == 0) L.some = t.s != 0.0f;  // (NaN: one that is NaN)
}

// The row's loss, by one wave.
template <int K>
__device__ __forceinline__ void put_loss(const DistillArgs &p, int64_t i, float wt, float m,
                                         float ls, const TeacherLds<K> &L) {
    float sum = 0.0f;
    for (int j = lane_id(); j < p.k; j += kWave) {
        const float lp = L.lp[j], q = exp2_raw(lp * kLog2e);
        if (q != 0.0f) sum = __builtin_fmaf(q, lp - log_prob(L.z[j], m, ls, p.inv_t), sum);
    }
    sum = wave_sum64(sum);
    if (lane_id() == 0) p.loss[i] = wt * sum;
}

// g q of a logit, q by its root twice: the product reaches the subnormals, which the
// instruction's own results do not.
struct Gradient {
    float m, half_c, half_l;  // c / 2, log2 S / 2 (0 in a row that holds only -inf)
    __device__ __forceinline__ Gradient(float m, float ls, float c)
        : m(m), half_c(0.5f * c), half_l(ls == kNegInf ? 0.0f : 0.5f * kLog2e * ls) {}
    __device__ __forceinline__ float operator()(float g, float z) const {
        const float r = exp2_raw(__builtin_fmaf(z - m, half_c, -half_l));
        return r * (r * g);
    }
};

// The teacher's entries among the vectors [first, last) of a row: once per id, with the
// sum of its probabilities.  After the team's own stores to those places.
template <int DT, int W, int K>
__device__ __forceinline__ void put_entries(const DistillArgs &p, char *out, int first, int last,
                                            float g, const Gradient &gradient,
                                            const TeacherLds<K> &L) {
    constexpr int kV = Elem<DT>::kVec;
    for (int j = Team<W>::thread(); j < p.k; j += Team<W>::kThreads) {
        const int32_t id = L.id[j];
        if (id < 0 || id / kV < first || id / kV >= last) continue;
        float sum = 0.0f;
        bool seen = false;
        for (int q = 0; q < p.k; ++q)
            if (L.id[q] == id) {
                seen |= q < j;
                sum += exp2_raw(L.lp[q] * kLog2e);
            }
        if (!seen) store1<DT>(out, id, g * (gradient(1.0f, L.z[j]) - sum));
    }
}

// ----------------------------------------------------------------------------
// a row in its team's registers

// The teacher's entries that a team has room for, three rows' of them in LDS: fewer
// where many teams share a compute unit.
template <int W>
constexpr int kTeacherRoom = W == 1 ? 128 : W == 2 ? 256 : W == 4 ? 512 : PDB_MAX_TEACHER;

constexpr int kGroup = 4;  // vectors that go into the statistics together

// A copy of a vector that the compiler does not know to be one: what is unpacked of it
// is not kept to be used again where the vector is (the registers are full).
template <int DT>
__device__ __forceinline__ u32x4 apart(u32x4 r) {
    if constexpr (DT != PDB_F32) asm volatile("" : "+v"(r));
    return r;
}

// R vectors a thread.  A team takes every so many-th row, with one barrier a row that
// leaves loads and stores under way.  A vector's gradient leaves its registers to the
// next row's, whose sums follow four vectors at a time while later ones of this row
// are still to be written; the teacher's entries of a row, which go over its own
// stores, are written behind the next row's barrier: a wave's accesses return in
// order, so its stores are done when it has the next row.
template <int DT, int W, int R, bool GRAD>
__global__ __launch_bounds__(W == 1 ? kBlock : W * kWave, R > 4 ? 4 : 8)
void k_distill_row(DistillArgs p) {
    constexpr int kV = Elem<DT>::kVec, kT = Team<W>::kThreads, kGroups = R / kGroup;
    constexpr int kAhead = kGroups / 2;  // of the next row's groups, summed within this row
    static_assert(R % kGroup == 0, "whole groups");
    __shared__ TeacherLds<kTeacherRoom<W>> s_teacher[Team<W>::kPerBlock][3];
    __shared__ float s_m[2][W], s_s[2][W];
    auto &teacher = s_teacher[Team<W>::here()];
    const int thread = Team<W>::thread();
    const int full = (int)(p.v / kV), rem = (int)(p.v % kV);
    const int64_t step = (int64_t)gridDim.x * Team<W>::kPerBlock;
    int64_t i = (int64_t)blockIdx.x * Team<W>::kPerBlock + Team<W>::here();
    if (i >= p.n) return;
    u32x4 r[R];
    float tail;
    // Every load is made, past the row's end of its last vector: under a condition it
    // would go through other registers, and be waited for there.  Its offset is formed
    // anew each time: kept, they would not fit the registers.
    auto load = [&](int u, const char *row, int end) {
        int lane = thread;
        asm volatile("" : "+v"(lane));
        r[u] = load16(row + (uint32_t)(min(lane + u * kT, end - 1) * 16));
    };
    auto load_tail = [&](const char *row) {
        tail = load1<DT>(row, min((int64_t)full * kV + thread, p.v - 1));
    };
    // Of the row in r, as far as it is summed.  Here y is c (z - m) throughout: one
    // subtraction more, but no second form of the loops for rows out of range.
    Stat t = empty_stat();
    auto raise = [&](float top) {
        if (__any(top > t.m)) {
            const float m = fmaxf(t.m, wave_max_f32(top));
            t.s *= exp2_raw((t.m - m) * p.c);
            t.m = m;
        }
    };
    auto sum_group = [&](int q) {
        if (q * kGroup * kT >= full) return;
        float all = kNegInf;
#pragma unroll
        for (int u = q * kGroup; u < (q + 1) * kGroup; ++u) {
            const float top = vec_max<DT>(apart<DT>(r[u]));
            all = thread + u * kT < full ? fmaxf(all, top) : all;
        }
        raise(all);
        const float m = wave_uniform(t.m);
#pragma unroll
        for (int u = q * kGroup; u < (q + 1) * kGroup; ++u) {
            float x[kV], s = 0.0f;
            unpack<DT>(r[u], x);
#pragma unroll
            for (int e = 0; e < kV; ++e) s += exp2_raw((x[e] - m) * p.c);
            t.s += thread + u * kT < full ? s : 0.0f;
            __builtin_amdgcn_sched_barrier(0);
        }
        asm volatile("" : "+v"(t.s));
    };
    const char *row = elem_at<DT>(p.z, i * p.ldz);
#pragma unroll
    for (int u = 0; u < R; ++u) load(u, row, full);
    load_tail(row);
    if (Team<W>::wave() == 0) teacher_row<DT>(p, i, row, teacher[0]);
#pragma unroll
    for (int q = 0; q < kAhead; ++q) sum_group(q);
    char *last_out = nullptr;     // of the row before: where its entries go, and its factors
    float last_g = 0.0f;
    Gradient last(0.0f, 0.0f, 0.0f);
    for (int turn = 0, slot = 0; i < p.n; i += step, turn ^= 1, slot = slot == 2 ? 0 : slot + 1) {
        auto &L = teacher[slot], &L_next = teacher[slot == 2 ? 0 : slot + 1];
        auto &L_last = teacher[slot == 0 ? 2 : slot - 1];
        // the team's next row (behind its last: that one's first vector, for nobody)
        const bool more = i + step < p.n;
        const int64_t i_next = more ? i + step : i;
        const char *next = elem_at<DT>(p.z, i_next * p.ldz);
        const int end = more ? full : 1;
        char *out = elem_at<DT>(p.dz, i * p.ldd);
        const float wt = row_weight(p, i);
#pragma unroll
        for (int q = kAhead; q < kGroups; ++q) sum_group(q);
        if (thread >= rem) tail = kNegInf;
        raise(tail);
        t.s = wave_sum64(t.s + exp2_raw((tail - t.m) * p.c));
        if constexpr (W > 1) {
            if (lane_id() == 0) {
                s_m[turn][wave_in_block()] = t.m;
                s_s[turn][wave_in_block()] = t.s;
            }
            Team<W>::sync_lds();
            // every lane its share of the waves, then all lanes the sum (W <= 64)
            const bool has = lane_id() < W;
            const float wm = has ? s_m[turn][lane_id() & (W - 1)] : -FLT_MAX;
            const float ws = has ? s_s[turn][lane_id() & (W - 1)] : 0.0f;
            t.m = wave_max_f32(wm);
            t.s = wave_sum64(ws * exp2_raw((wm - t.m) * p.c));
        } else {
            Team<W>::sync();
        }
        if (GRAD && last_out)
            put_entries<DT, W>(p, last_out, 0, full + 1, last_g, last, L_last);
        last_out = nullptr;
        const float ls = t.s == 0.0f ? kNegInf : __builtin_amdgcn_logf(t.s) * kLn2;
        const float m = t.s == 0.0f ? 0.0f : t.m;
        t = empty_stat();
        const bool some = wt != 0.0f && L.some;
        if (Team<W>::wave() == 0) {
            if (some)
                put_loss(p, i, wt, m, ls, L);
            else if (lane_id() == 0)
                p.loss[i] = 0.0f;
        }
        const float g = wt * p.inv_t;
        const Gradient gradient(m, ls, p.c);
        if (GRAD && thread < rem)
            store1<DT>(out, (int64_t)full * kV + thread, some ? gradient(g, tail) : 0.0f);
        load_tail(next);
#pragma unroll
        for (int u = 0; u < R; ++u) {
            if (GRAD && thread + u * kT < full) {
                u32x4 d = {0, 0, 0, 0};
                if (some) {
                    float x[kV];
                    unpack<DT>(apart<DT>(r[u]), x);
#pragma unroll
                    for (int e = 0; e < kV; ++e) x[e] = gradient(g, x[e]);
                    d = pack<DT>(x);
                }
                store16(vec_at<W>(out, u * kT), d);
            }
            load(u, next, end);
            __builtin_amdgcn_sched_barrier(0);
            // the next row's first groups, R / 2 vectors behind their loads
            if (kAhead > 0 && u >= R / 2 && (u + 1) % kGroup == 0)
                sum_group((u + 1 - R / 2) / kGroup - 1);
        }
        if (GRAD && some) {
            last_out = out;
            last_g = g;
            last = gradient;
        }
        if (more) {
            if (Team<W>::wave() == 0) teacher_row<DT>(p, i_next, next, L_next);
        } else if (GRAD && last_out) {  // the team's last row
            __builtin_amdgcn_s_waitcnt(0);
            Team<W>::sync();
            put_entries<DT, W>(p, out, 0, full + 1, last_g, last, L);
        }
    }
}

// ----------------------------------------------------------------------------
// rows in parts

constexpr int kPartWaves = kBlock / kWave;

template <int DT>
__global__ __launch_bounds__(kBlock) void k_distill_stat(DistillArgs p) {
    constexpr int kV = Elem<DT>::kVec, W = kPartWaves;
    const int full = (int)(p.v / kV), rest = (int)(p.v % kV), thread = threadIdx.x;
    for (int64_t w = blockIdx.x; w < p.n * p.parts; w += gridDim.x) {
        const auto [i, part] = Work(w, p.parts);
        if (row_weight(p, i) == 0.0f) continue;
        const int first = part * p.part_vecs, end = min(full, first + p.part_vecs);
        const int rem = end == full ? rest : 0;  // the tail is the last part's
        const char *row = elem_at<DT>(p.z, i * p.ldz);
        Stat t = empty_stat();
        for (int j = first; j < end; j += kTileVecs * kBlock) {
            float lm[kTileVecs];
            add_tile<DT, false>(load_tile<DT, W>(row, j, end), p.c, t, lm);
        }
        if (rem > 0) add_elem<false>(tail_elem<DT, W>(row, full, rem), p.c, t);
        t = team_stat<W>(t, p.c);
        if (thread == 0) put_part(p.part_stat, w, t);
    }
}

template <int DT, bool GRAD>
__global__ __launch_bounds__(kBlock) void k_distill_part(DistillArgs p) {
    constexpr int kV = Elem<DT>::kVec, W = kPartWaves;
    __shared__ TeacherLds<PDB_MAX_TEACHER> L;
    const int full = (int)(p.v / kV), rest = (int)(p.v % kV), thread = threadIdx.x;
    for (int64_t w = blockIdx.x; w < p.n * p.parts; w += gridDim.x) {
        const auto [i, part] = Work(w, p.parts);
        const int first = part * p.part_vecs, end = min(full, first + p.part_vecs);
        const int rem = end == full ? rest : 0;  // the tail is the last part's
        const char *row = elem_at<DT>(p.z, i * p.ldz);
        char *out = elem_at<DT>(p.dz, i * p.ldd);
        const float wt = row_weight(p, i);
        __syncthreads();  // the row before is done with L
        if (wt != 0.0f && wave_in_block() == 0) teacher_row<DT>(p, i, row, L);
        __syncthreads();
        if (wt == 0.0f || !L.some) {
            if (part == 0 && thread == 0 && p.loss) p.loss[i] = 0.0f;
            if (GRAD) zero_row<DT, W>(out, first, end, full, rem);
            continue;
        }
        const Stat t = join_parts(p.part_stat, i, p.stat_parts, p.c);
        const float ls = log_sum(t, p.c), m = t.s == 0.0f ? 0.0f : t.m;
        if (part == 0 && p.loss && wave_in_block() == 0) put_loss(p, i, wt, m, ls, L);
        if constexpr (GRAD) {
            const float g = wt * p.inv_t;
            const Gradient gradient(m, ls, p.c);
            const float tail = tail_elem<DT, W>(row, full, rem);
            map_row<DT, W>(row, out, first, end, [&](int, float *x) {
#pragma unroll
                for (int e = 0; e < kV; ++e) x[e] = gradient(g, x[e]);
            });
            if (thread < rem) store1<DT>(out, (int64_t)full * kV + thread, gradient(g, tail));
            __syncthreads();
            put_entries<DT, W>(p, out, first, rem > 0 ? full + 1 : end, g, gradient, L);
        }
    }
}

// Rows from which the card is full with a team each (on fewer, parts keep more compute
// units at work).
constexpr int64_t kFullRows = 256;

template <int DT, int W, int R>
int distill_rows(const DistillArgs &p, hipStream_t s) {
    constexpr int kThreads = W == 1 ? kBlock : W * kWave;
    // as many teams as stay resident, each with every so many-th row
    const int64_t resident = 256 * (R > 4 ? 1024 : 2048) / kThreads;
    const unsigned blocks =
        (unsigned)std::min<int64_t>(blocks_for(p.n, Team<W>::kPerBlock), resident);
    if (p.dz)
        k_distill_row<DT, W, R, true><<<blocks, kThreads, 0, s>>>(p);
    else
        k_distill_row<DT, W, R, false><<<blocks, kThreads, 0, s>>>(p);
    PDB_LAUNCHED();
    return PDB_OK;
}

template <int DT>
int distill_parts(DistillArgs p, const Parts &cut, hipStream_t s) {
    p.part_vecs = cut.vecs;
    p.parts = p.stat_parts = cut.parts;
    const unsigned blocks = blocks_for(p.n * cut.parts);
    k_distill_stat<DT><<<blocks, kBlock, 0, s>>>(p);
    PDB_LAUNCHED();
    // the loss reads the logits of every id: in place, before any part of a row is
    // overwritten
    if (!p.dz || (p.dz == p.z && cut.parts > 1)) {
        p.parts = 1;
        k_distill_part<DT, false><<<blocks_for(p.n), kBlock, 0, s>>>(p);
        PDB_LAUNCHED();
        p.parts = cut.parts;
        p.loss = nullptr;
    }
    if (p.dz) {
        k_distill_part<DT, true><<<blocks, kBlock, 0, s>>>(p);
        PDB_LAUNCHED();
    }
    return PDB_OK;
}

}  // namespace
}  // namespace pdbk

using namespace pdbk;

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
        const DistillArgs p = {logits, ldz, n, v, ids, teacher, teacher_dtype, k, 1.0f / temp,
                               kLog2e / temp, weight, loss, dlogits, ldd, status, 0, 1, 1,
                               static_cast<float *>(ws)};
        const Parts cut = cut_rows(n, v, Elem<DT>::kVec, kMostParts);
        // the fewest waves whose registers hold a row, and whose LDS the teacher's entries
        const int64_t full = v / Elem<DT>::kVec, lanes = cdiv(full, 16);
        auto fits = [&](int w, int room) { return lanes <= w * kWave && k <= room; };
        if (full < 1 || lanes > 16 * kWave || (cut.parts > 1 && n < kFullRows))
            return distill_parts<DT>(p, cut, s);
        if (full <= 4 * kWave && k <= kTeacherRoom<1>) return distill_rows<DT, 1, 4>(p, s);
        if (fits(1, kTeacherRoom<1>)) return distill_rows<DT, 1, 16>(p, s);
        if (fits(2, kTeacherRoom<2>)) return distill_rows<DT, 2, 16>(p, s);
        if (fits(4, kTeacherRoom<4>)) return distill_rows<DT, 4, 16>(p, s);
        if (fits(8, kTeacherRoom<8>)) return distill_rows<DT, 8, 16>(p, s);
        return distill_rows<DT, 16, 16>(p, s);
    });
}
