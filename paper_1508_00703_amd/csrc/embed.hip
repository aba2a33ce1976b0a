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
// tile order by a second kernel.  No atomics: the order of every sum follows
// from the sizes.
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
// gradient

// tokens to sort keys: padding goes behind every row of the table
__global__ __launch_bounds__(kBlock) void k_embed_keys(const void *__restrict__ tokens, int index,
                                                       int64_t n, int64_t v,
                                                       uint32_t *__restrict__ keys,
                                                       int32_t *status) {
    for (int64_t i = blockIdx.x * (int64_t)kBlock + threadIdx.x; i < n;
         i += (int64_t)gridDim.x * kBlock) {
        const int32_t t = read_token(tokens, index, i, v, status);
        keys[i] = t < 0 ? (uint32_t)v : (uint32_t)t;
    }
}

// grad[t] at columns c.. from a finished sum
template <int GT, int E>
__device__ __forceinline__ void put_row(void *grad, int64_t ldg, uint32_t t, int64_t c, int64_t d,
                                        float scale, bool accumulate, const float *sum) {
    float x[E];
    if (accumulate) {
        load_cols<GT, E>(grad, (int64_t)t * ldg, c, d, x);
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = __builtin_fmaf(scale, sum[e], x[e]);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = scale * sum[e];
    }
    store_cols<GT, E>(grad, (int64_t)t * ldg, c, d, x);
}

constexpr int kAhead = 4;  // rows a lane has in flight

// One tile of R sorted entries per group.  part: [tiles][2][d], slot 0 what the
// tile adds to a token that began before it, slot 1 to one that goes on after it.
template <int DT, int GT>
__global__ __launch_bounds__(kBlock) void k_embed_tiles(
    const void *__restrict__ dy, int64_t ldy, const uint32_t *__restrict__ keys,
    const uint32_t *__restrict__ vals, int64_t n, int64_t d, int64_t v, int R, int lg, float scale,
    int accumulate, void *__restrict__ grad, int64_t ldg, float *__restrict__ part) {
    constexpr int kE = Pair<DT, GT>::kE;
    const int lane = threadIdx.x & ((1 << lg) - 1);
    const int64_t tile = (int64_t)blockIdx.x * (kBlock >> lg) + (threadIdx.x >> lg);
    const int64_t c = ((int64_t)blockIdx.y << lg | lane) * kE;
    const int64_t e0 = tile * R, e1 = min(n, e0 + R);
    if (e0 >= n || c >= d) return;
    float sum[kE];
#pragma unroll
    for (int e = 0; e < kE; ++e) sum[e] = 0.0f;
    uint32_t cur = keys[e0];
    bool began = e0 > 0 && keys[e0 - 1] == cur;  // cur's first entry lies in an earlier tile
    for (int64_t e = e0; e < e1; e += kAhead) {
        uint32_t t[kAhead];
        float x[kAhead][kE];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int64_t at = min(e + k, e1 - 1);
            t[k] = keys[at];
            if (t[k] < (uint32_t)v) load_cols<DT, kE>(dy, (int64_t)vals[at] * ldy, c, d, x[k]);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (e + k >= e1 || cur == (uint32_t)v) break;  // padding comes last
            if (t[k] != cur) {
                if (began)
                    store_cols<PDB_F32, kE>(part, (tile * 2) * d, c, d, sum);
                else
                    put_row<GT, kE>(grad, ldg, cur, c, d, scale, accumulate, sum);
                began = false;
                cur = t[k];
                if (cur == (uint32_t)v) break;
#pragma unroll
                for (int q = 0; q < kE; ++q) sum[q] = 0.0f;
            }
#pragma unroll
            for (int q = 0; q < kE; ++q) sum[q] += x[k][q];
        }
    }
    if (cur == (uint32_t)v) return;
    const bool goes_on = e1 < n && keys[e1] == cur;
    if (began)
        store_cols<PDB_F32, kE>(part, (tile * 2) * d, c, d, sum);
    else if (goes_on)
        store_cols<PDB_F32, kE>(part, (tile * 2 + 1) * d, c, d, sum);
    else
        put_row<GT, kE>(grad, ldg, cur, c, d, scale, accumulate, sum);
}

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

// Tokens that cross tiles: the group of the tile where one begins adds the
// later tiles' slots to its own, in tile order.  A run of more than kOwn tiles is
// added by the whole block: every group takes each G-th tile, then the groups'
// sums are added in order.
constexpr int kOwn = 16;
template <int GT, int E>
__global__ __launch_bounds__(kBlock) void k_embed_join(const uint32_t *__restrict__ keys, int64_t n,
                                                       int64_t d, int64_t v, int64_t tiles, int R,
                                                       int lg, float scale, int accumulate,
                                                       void *__restrict__ grad, int64_t ldg,
                                                       const float *__restrict__ part) {
    __shared__ float s_sum[kBlock * E];
    __shared__ int64_t s_last[kBlock];
    const int L = 1 << lg, lane = threadIdx.x & (L - 1);
    const int groups = kBlock >> lg, g = threadIdx.x >> lg;
    const int64_t tile0 = (int64_t)blockIdx.x * groups;
    const int64_t c = ((int64_t)blockIdx.y << lg | lane) * E;
    auto add_slots = [&](float *sum, int64_t from, int64_t to, int64_t step) {
        for (int64_t q = from; q <= to; q += step * kAhead) {
            float x[kAhead][E];
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                if (q + k * step <= to)
                    load_cols<PDB_F32, E>(part, (q + k * step) * 2 * d, c, d, x[k]);
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                if (q + k * step > to) break;
#pragma unroll
                for (int e = 0; e < E; ++e) sum[e] += x[k][e];
            }
        }
    };
    // the last tile of the token that begins in this group's tile and goes on; -1 none
    const int64_t tile = tile0 + g;
    int64_t last = -1;
    uint32_t t = 0;
    if (tile < tiles - 1) {
        const int64_t e0 = tile * R, e1 = e0 + R;
        t = keys[e1 - 1];
        const bool whole = e0 > 0 && keys[e0 - 1] == t;  // it began before this tile
        if (t < (uint32_t)v && keys[e1] == t && !whole)
            last = (lower_bound_key(keys, e1, n, t + 1) - 1) / R;
    }
    const bool mine = last >= 0 && last - tile <= kOwn;
    if (mine && c < d) {
        float sum[E];
        load_cols<PDB_F32, E>(part, (tile * 2 + 1) * d, c, d, sum);
        add_slots(sum, tile + 1, last, 1);
        put_row<GT, E>(grad, ldg, t, c, d, scale, accumulate, sum);
    }
    if (lane == 0) s_last[g] = last >= 0 && !mine ? last : -1;
    __syncthreads();
    for (int k = 0; k < groups; ++k) {
        const int64_t to = s_last[k];
        if (to < 0) continue;
        const int64_t from = tile0 + k;
        float sum[E];
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] = 0.0f;
        if (c < d) {
            if (g == 0) load_cols<PDB_F32, E>(part, (from * 2 + 1) * d, c, d, sum);
            add_slots(sum, from + 1 + g, to, groups);
        }
#pragma unroll
        for (int e = 0; e < E; ++e) s_sum[threadIdx.x * E + e] = sum[e];
        __syncthreads();
        if (g == 0 && c < d) {
            for (int q = 1; q < groups; ++q)
#pragma unroll
                for (int e = 0; e < E; ++e) sum[e] += s_sum[(q * L + lane) * E + e];
            put_row<GT, E>(grad, ldg, keys[from * R + R - 1], c, d, scale, accumulate, sum);
        }
        __syncthreads();
    }
}

// zeros in the rows of the table that no token picked, 64 rows per block
template <int GT>
__global__ __launch_bounds__(kBlock) void k_embed_zero(const uint32_t *__restrict__ keys, int64_t n,
                                                       int64_t d, int64_t v, int lg,
                                                       void *__restrict__ grad, int64_t ldg) {
    constexpr int kE = Elem<GT>::kVec;
    __shared__ unsigned long long s_free;
    const float zero[kE] = {};
    const int lane = threadIdx.x & ((1 << lg) - 1);
    for (int64_t r0 = (int64_t)blockIdx.x * kWave; r0 < v; r0 += (int64_t)gridDim.x * kWave) {
        if (wave_in_block() == 0) {
            const int64_t r = r0 + lane_id();
            bool free = false;
            if (r < v) {
                const int64_t at = lower_bound_key(keys, 0, n, (uint32_t)r);
                free = at >= n || keys[at] != (uint32_t)r;
            }
            const unsigned long long m = __ballot(free);
            if (lane_id() == 0) s_free = m;
        }
        __syncthreads();
        const unsigned long long m = s_free;
        for (int q = threadIdx.x >> lg; q < kWave; q += kBlock >> lg)
            if ((m >> q) & 1ull)
                for (int64_t c = (int64_t)lane * kE; c < d; c += (int64_t)kE << lg)
                    store_cols<GT, kE>(grad, (r0 + q) * ldg, c, d, zero);
        __syncthreads();
    }
}

// ----------------------------------------------------------------------------

// Entries per tile.  Enough tiles that n d / R elements, about 2^22, fill the
// card's lanes with one vector each; not fewer than 8, so that few partials are
// written, nor more than 256.
inline int tile_rows(int64_t n, int64_t d) {
    const int64_t r = (n * d) >> 22;
    return (int)std::min<int64_t>(std::max<int64_t>(r, 8), 256);
}

struct GradWs {
    uint32_t *keys, *kA, *vA, *kB, *vB, *hist, *scan_tmp;
    float *part;
    size_t total;
};
GradWs grad_ws_layout(void *base, int64_t n, int64_t d) {
    GradWs w;
    char *p = static_cast<char *>(base);
    size_t off = 0;
    auto take = [&](int64_t bytes) {
        char *at = p + off;
        off += (size_t)align_up(bytes);
        return at;
    };
    const int64_t st = cdiv(std::max<int64_t>(n, 1), kTile), R = tile_rows(n, d);
    w.keys = reinterpret_cast<uint32_t *>(take(4 * n));
    w.kA = reinterpret_cast<uint32_t *>(take(4 * n));
    w.vA = reinterpret_cast<uint32_t *>(take(4 * n));
    w.kB = reinterpret_cast<uint32_t *>(take(4 * n));
    w.vB = reinterpret_cast<uint32_t *>(take(4 * n));
    w.hist = reinterpret_cast<uint32_t *>(take(4 * 256 * st));
    w.scan_tmp = reinterpret_cast<uint32_t *>(take(4 * (int64_t)scan_tmp_elems(256 * st)));
    w.part = reinterpret_cast<float *>(take(cdiv(n, R) * 2 * d * 4));
    w.total = off;
    return w;
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
    if (w.total > 0 && (!ws || ws_bytes < w.total)) return PDB_ERR_WORKSPACE;
    uint32_t *keys = nullptr, *vals = nullptr;
    if (n > 0) {
        k_embed_keys<<<grid_for(n, kBlock, 4096), kBlock, 0, s>>>(tokens, index, n, v, w.keys,
                                                                  status);
        PDB_LAUNCHED();
        int bits = 1;
        while (((int64_t)1 << bits) <= v) ++bits;
        PDB_HIP(radix_sort_pairs(w.keys, nullptr, n, bits, w.kA, w.vA, w.kB, w.vB, w.hist,
                                 w.scan_tmp, &keys, &vals, s));
    }
    const int R = tile_rows(n, d);
    const int64_t tiles = cdiv(n, R);
    return with_dtype(grad_dtype, [&](auto gt) -> int {
        constexpr int GT = decltype(gt)::value;
        if (!accumulate) {
            const int lg = lanes_log2(cdiv(d, Elem<GT>::kVec));
            k_embed_zero<GT><<<grid_for(v, kWave, 1 << 16), kBlock, 0, s>>>(keys, n, d, v, lg, grad,
                                                                            ldg);
            PDB_LAUNCHED();
        }
        if (n == 0) return PDB_OK;
        return with_dtype(dtype, [&](auto dt) -> int {
            constexpr int DT = decltype(dt)::value, kE = Pair<DT, GT>::kE;
            const int64_t vectors = cdiv(d, kE);
            const int lg = lanes_log2(vectors);
            const int64_t slices = cdiv(vectors, 1 << lg);
            if (slices > 65535) return PDB_ERR_UNSUPPORTED;
            const dim3 grid((unsigned)cdiv(tiles, kBlock >> lg), (unsigned)slices);
            k_embed_tiles<DT, GT><<<grid, kBlock, 0, s>>>(dy, ldy, keys, vals, n, d, v, R, lg, scale,
                                                          accumulate, grad, ldg, w.part);
            PDB_LAUNCHED();
            k_embed_join<GT, kE><<<grid, kBlock, 0, s>>>(keys, n, d, v, tiles, R, lg, scale,
                                                         accumulate, grad, ldg, w.part);
            PDB_LAUNCHED();
            return PDB_OK;
        });
    });
}
