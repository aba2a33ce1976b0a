// The norm of many tensors together, and the clipped gradients or the clipped step by
// it (gfx950, wave64).
//
// norm = |s| sqrt(sum g^2).  The tensors are cut into chunks; descriptions of up to
// kMostTensors (without gaps: kMostDense) travel in a launch's arguments, so nothing is
// copied to the device.
// Squares and sums are in binary64 (a square in binary32 passes its range from 1.8e19
// on, and falls out of it below 1e-23); each block leaves one sum, and whoever needs
// the norm adds the blocks' sums in the same order: no atomics.  Bound: the bytes (400 MB in
// one list 71 us, 5.7 TB/s).
// Clipping cannot begin before the last gradient is read: a second pass, from the last
// chunk to the first, so that it meets first what the cache still holds.
#include <math.h>
#include <stdlib.h>

#include <algorithm>
#include <type_traits>

#include "pdb_vec.h"
#include "../../include/pdb_layers.h"

namespace pdbk {
namespace {

// Tensors of a launch: 3.5 KB of arguments.  A launch has an end of its own, where blocks
// run out of chunks: 200 tensors of 400 MB in four took 86 us, in two 80.
constexpr int kMostTensors = 64, kMostDense = 112;
// Elements of a chunk.  (4,096: the same tensors 89 us, since each chunk's description is
// looked up; 16,384: ends of launches, 61 strided matrices 118 us against 107.)
constexpr int kChunk = 8192;
constexpr int kSums = 2048;  // blocks that the card holds, a sum of each

struct Item {
    const char *g;
    char *o;
    int64_t cols, ld, ldo;
    int32_t rows;
    uint32_t first;  // the tensor's first chunk in the launch
    int16_t dt, odt;
    int32_t rows_at_once;  // rows of a chunk; 1 where a row has several chunks
};
struct DenseItem {  // of one row
    const char *g;
    char *o;
    int64_t cols;
    uint32_t first;
    int16_t dt, odt;
};
template <typename ITEM>
struct List {
    static constexpr int kMost = std::is_same<ITEM, Item>::value ? kMostTensors : kMostDense;
    ITEM item[kMost];
    int32_t count;
    uint32_t chunks;
};

// The tensor of a chunk, by a wave.
template <typename ITEM>
__device__ __forceinline__ int item_of(const List<ITEM> &list, uint32_t w) {
    int i = -1;
#pragma unroll
    for (int l0 = 0; l0 < List<ITEM>::kMost; l0 += kWave) {
        const int l = l0 + lane_id();
        i += __popcll(__ballot(l < list.count && list.item[l].first <= w));
    }
    return __builtin_amdgcn_readfirstlane(i);
}

// A chunk: rows [row, row + rows) x columns [col, col + cols) of a tensor.
struct Chunk {
    int64_t row, col;
    int32_t rows, cols;
};
__device__ __forceinline__ Chunk chunk_of(const Item &t, uint32_t w) {
    const uint32_t k = w - t.first;
    if (t.cols > kChunk) {
        const uint32_t of_row = (uint32_t)((t.cols + kChunk - 1) / kChunk);
        const uint32_t row = k / of_row;
        const int64_t col = (int64_t)(k - row * of_row) * kChunk;
        return {(int64_t)row, col, 1, (int32_t)min((int64_t)kChunk, t.cols - col)};
    }
    const int64_t row = (int64_t)k * t.rows_at_once;
    return {row, 0, (int32_t)min((int64_t)t.rows_at_once, t.rows - row), (int32_t)t.cols};
}
__device__ __forceinline__ Chunk chunk_of(const DenseItem &t, uint32_t w) {
    const int64_t col = (int64_t)(w - t.first) * kChunk;
    return {0, col, 1, (int32_t)min((int64_t)kChunk, t.cols - col)};
}
__device__ __forceinline__ int64_t row_of(const Item &t) { return t.ld; }
__device__ __forceinline__ int64_t row_of(const DenseItem &t) { return 0; }
__device__ __forceinline__ int64_t out_row_of(const Item &t) { return t.ldo; }
__device__ __forceinline__ int64_t out_row_of(const DenseItem &t) { return 0; }

// Calls f(offset in g, offset in o, elements) for a thread's vectors of a chunk: whole
// ones (elements = V), and what is left of rows.
template <int V, typename ITEM, typename F>
__device__ __forceinline__ void for_vectors(const ITEM &t, const Chunk &c, F f) {
    const int64_t ld = row_of(t), ldo = out_row_of(t);
    const int64_t g0 = c.row * ld + c.col, o0 = c.row * ldo + c.col;
    const int whole = c.cols / V, rem = c.cols - whole * V;
    if (std::is_same<ITEM, DenseItem>::value || c.rows == 1) {
#pragma unroll 4
        for (int v = threadIdx.x; v < whole; v += kBlock) f(g0 + v * V, o0 + v * V, V);
        if ((int)threadIdx.x < rem)
            f(g0 + whole * V + threadIdx.x, o0 + whole * V + threadIdx.x, 1);
        return;
    }
    const uint32_t of_row = (uint32_t)(whole + (rem ? 1 : 0)), all = of_row * (uint32_t)c.rows;
    for (uint32_t v = threadIdx.x; v < all; v += kBlock) {
        const uint32_t r = v / of_row, q = (v - r * of_row) * V;
        f(g0 + r * ld + q, o0 + r * ldo + q, min(V, c.cols - (int)q));
    }
}

__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
// the sum over the block, the same in every thread
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

template <int DT, typename ITEM>
__device__ __forceinline__ double chunk_squares(const ITEM &t, const Chunk &c) {
    constexpr int V = Elem<DT>::kVec;
    double s[2] = {0.0, 0.0};
    for_vectors<V>(t, c, [&](int64_t g, int64_t, int k) {
        if (k == V) {
            float x[V];
            unpack<DT>(load16(elem_at<DT>(t.g, g)), x);
#pragma unroll
            for (int q = 0; q < V; ++q) s[q & 1] = fma((double)x[q], (double)x[q], s[q & 1]);
        } else {
            for (int q = 0; q < k; ++q) {
                const double x = load1<DT>(t.g, g + q);
                s[0] = fma(x, x, s[0]);
            }
        }
    });
    return s[0] + s[1];
}

// sums[block] (+)= the squares of the block's chunks
template <typename ITEM>
__global__ __launch_bounds__(kBlock) void k_grad_squares(List<ITEM> list, double *sums, int add) {
    double s = 0.0;
    for (uint32_t w = blockIdx.x; w < list.chunks; w += gridDim.x) {
        const ITEM &t = list.item[item_of(list, w)];
        const Chunk c = chunk_of(t, w);
        if (t.dt == PDB_F32) s += chunk_squares<PDB_F32>(t, c);
        if (t.dt == PDB_F16) s += chunk_squares<PDB_F16>(t, c);
        if (t.dt == PDB_BF16) s += chunk_squares<PDB_BF16>(t, c);
    }
    s = block_sum_f64(s);
    if (threadIdx.x == 0) sums[blockIdx.x] = add ? sums[blockIdx.x] + s : s;
}

__device__ __forceinline__ double norm_of(const double *sums, int count, double scale) {
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < kSums / kBlock; ++i) {
        const int at = i * kBlock + threadIdx.x;
        s += at < count ? sums[at] : 0.0;
    }
    return fabs(scale) * sqrt(block_sum_f64(s));
}

__global__ __launch_bounds__(kBlock) void k_grad_norm(const double *sums, int count, double scale,
                                                      float *norm) {
    const double n = norm_of(sums, count, scale);
    if (threadIdx.x == 0) *norm = (float)n;
}

// Four or eight elements at element i, in one access of 8 or 16 bytes.  What is written,
// and what it is added to, is used once: it leaves the cache to the gradients, which are
// read twice (48 tensors, 240 MB of 16 bits in and out: 75 us without, 62 with).
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));
template <int DT, int V>
__device__ __forceinline__ u32x4 load_few(const char *p, int64_t i, bool once) {
    static_assert(V * Elem<DT>::kSize == 16 || V * Elem<DT>::kSize == 8, "one access");
    if constexpr (V * Elem<DT>::kSize == 16) {
        const auto *at = reinterpret_cast<const u32x4_any *>(elem_at<DT>(p, i));
        return once ? __builtin_nontemporal_load(at) : *at;
    } else {
        const auto *at = reinterpret_cast<const u32x2_any *>(elem_at<DT>(p, i));
        const u32x2 r = once ? __builtin_nontemporal_load(at) : *at;
        return u32x4{r[0], r[1], 0, 0};
    }
}
template <int DT, int V>
__device__ __forceinline__ void store_few(char *p, int64_t i, u32x4 r) {
    if constexpr (V * Elem<DT>::kSize == 16) {
        __builtin_nontemporal_store(r, reinterpret_cast<u32x4_any *>(elem_at<DT>(p, i)));
    } else {
        __builtin_nontemporal_store(u32x2{r[0], r[1]}, reinterpret_cast<u32x2_any *>(elem_at<DT>(p, i)));
    }
}

template <int DT, int OT, typename ITEM>
__device__ __forceinline__ void chunk_step(const ITEM &t, const Chunk &c, float by, bool acc) {
    // 16 bytes of the wider type: whole lines to a store of either (16 bits into 32: 82 us
    // for 60M elements, 110 with eight to a thread).  One vector at a time: the card's
    // waves hide it (four at a time: 93 us, more registers and fewer waves).
    constexpr int V = std::min(Elem<DT>::kVec, Elem<OT>::kVec);
    for_vectors<V>(t, c, [&](int64_t g, int64_t o, int k) {
        if (k == V) {
            float x[8], y[8];
            unpack<DT>(load_few<DT, V>(t.g, g, false), x);
            if (acc) unpack<OT>(load_few<OT, V>(t.o, o, true), y);
#pragma unroll
            for (int q = 0; q < V; ++q) y[q] = acc ? __builtin_fmaf(by, x[q], y[q]) : by * x[q];
            store_few<OT, V>(t.o, o, pack<OT>(y));
        } else {
            for (int q = 0; q < k; ++q) {
                const float x = load1<DT>(t.g, g + q);
                const float y = acc ? __builtin_fmaf(by, x, load1<OT>(t.o, o + q)) : by * x;
                store1<OT>(t.o, o + q, y);
            }
        }
    });
}

template <typename ITEM>
__global__ __launch_bounds__(kBlock) void k_grad_clip(List<ITEM> list, const double *sums, int count,
                                                      double scale, double most, double step,
                                                      int acc, float *norm) {
    const double n = norm_of(sums, count, scale);
    const float nf = (float)n;
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = nf;
    if (!(fabsf(nf) < __builtin_inff())) return;
    const float by = (float)(step * (n > most ? most / n : 1.0) * scale);
    for (uint32_t i = blockIdx.x; i < list.chunks; i += gridDim.x) {
        const uint32_t w = list.chunks - 1 - i;
        const ITEM &t = list.item[item_of(list, w)];
        const Chunk c = chunk_of(t, w);
        if (!acc && by == 1.0f && t.g == t.o) continue;
        auto to = [&](auto dt) {
            constexpr int DT = decltype(dt)::value;
            if (t.odt == PDB_F32) chunk_step<DT, PDB_F32>(t, c, by, acc);
            if (t.odt == PDB_F16) chunk_step<DT, PDB_F16>(t, c, by, acc);
            if (t.odt == PDB_BF16) chunk_step<DT, PDB_BF16>(t, c, by, acc);
        };
        if (t.dt == PDB_F32) to(DtypeTag<PDB_F32>());
        if (t.dt == PDB_F16) to(DtypeTag<PDB_F16>());
        if (t.dt == PDB_BF16) to(DtypeTag<PDB_BF16>());
    }
}

// ----------------------------------------------------------------------------
// host side

constexpr int64_t kMostElements = (int64_t)1 << 40;  // of a tensor: at most 2^28 chunks
constexpr int64_t kMostAll = (int64_t)1 << 43;       // at most 2^31 chunks
constexpr int64_t kMostChunks = (int64_t)1 << 30;    // a list is closed from here on
constexpr int kMostLists = (1 << 20) / kMostTensors + 4;

int check_tensor(const pdb_tensor &t) {
    if (!is_dtype(t.dtype) || t.rows < 0 || t.cols < 0) return PDB_ERR_INVALID_ARG;
    if (t.rows == 0 || t.cols == 0) return PDB_OK;
    if (t.rows > INT32_MAX || t.cols >= kMostElements || t.rows >= kMostElements / t.cols ||
        t.ld > kMostElements)
        return PDB_ERR_UNSUPPORTED;
    if (t.rows > 1 && t.ld < t.cols) return PDB_ERR_INVALID_ARG;
    if (!t.data || !aligned_to(t.data, dtype_size(t.dtype))) return PDB_ERR_INVALID_ARG;
    return PDB_OK;
}

int check_tensors(const pdb_tensor *grads, int64_t count, const pdb_tensor *outs) {
    if (count < 0 || (count > 0 && !grads)) return PDB_ERR_INVALID_ARG;
    if (count >= 1 << 20) return PDB_ERR_UNSUPPORTED;
    int64_t all = 0;
    for (int64_t i = 0; i < count; ++i) {
        if (int e = check_tensor(grads[i])) return e;
        all += grads[i].rows * grads[i].cols;
        if (all >= kMostAll) return PDB_ERR_UNSUPPORTED;
        if (!outs) continue;
        if (int e = check_tensor(outs[i])) return e;
        if (outs[i].rows != grads[i].rows || outs[i].cols != grads[i].cols) return PDB_ERR_INVALID_ARG;
        const bool some = grads[i].rows > 0 && grads[i].cols > 0;
        if (some && outs[i].data == grads[i].data &&
            (outs[i].dtype != grads[i].dtype || (outs[i].rows > 1 && outs[i].ld != grads[i].ld)))
            return PDB_ERR_INVALID_ARG;
    }
    return PDB_OK;
}

bool no_gaps(const pdb_tensor &t) { return t.rows <= 1 || t.ld == t.cols; }
bool no_gaps(const pdb_tensor *grads, const pdb_tensor *outs, int64_t i) {
    return no_gaps(grads[i]) && (!outs || no_gaps(outs[i]));
}

// Memory that the call reads or writes: a tensor without gaps, or the first row of one
// with (rows of several tensors may lie between one another).
struct Span {
    uintptr_t at, end;
    bool written;
};
// What the tensors lie in: an output that is its own gradient once.
int64_t spans_of(const pdb_tensor *grads, const pdb_tensor *outs, int64_t count, Span *spans) {
    int64_t n = 0;
    auto add = [&](const pdb_tensor &t, bool written) {
        const uintptr_t at = (uintptr_t)t.data;
        const int64_t cells = no_gaps(t) ? t.rows * t.cols : t.cols;
        spans[n++] = {at, at + (uintptr_t)cells * (uintptr_t)dtype_size(t.dtype), written};
    };
    for (int64_t i = 0; i < count; ++i) {
        if (grads[i].rows == 0 || grads[i].cols == 0) continue;
        add(outs[i], true);
        if (grads[i].data != outs[i].data) add(grads[i], false);
    }
    return n;
}
// Whether an output shares memory with another output or with a gradient that is not its
// own: the blocks of a launch, and launches one after another, read the gradients while
// outputs are written, in no order that a caller knows.
int check_apart(const pdb_tensor *grads, const pdb_tensor *outs, int64_t count) {
    constexpr int64_t kHere = 256;  // spans that need no memory of their own
    Span here[kHere];
    Span *spans = 2 * count <= kHere ? here : static_cast<Span *>(malloc(2 * count * sizeof(Span)));
    if (!spans) return PDB_ERR_UNSUPPORTED;
    const int64_t n = spans_of(grads, outs, count, spans);
    std::sort(spans, spans + n, [](const Span &a, const Span &b) { return a.at < b.at; });
    uintptr_t read = 0, written = 0;  // how far what was met reaches
    bool apart = true;
    for (int64_t i = 0; i < n && apart; ++i) {
        const Span &s = spans[i];
        apart = s.at >= written && (!s.written || s.at >= read);
        (s.written ? written : read) = std::max(s.written ? written : read, s.end);
    }
    if (spans != here) free(spans);
    return apart ? PDB_OK : PDB_ERR_INVALID_ARG;
}

inline void put(Item &t, const pdb_tensor &g, const pdb_tensor *o, int64_t *chunks) {
    t.rows = (int32_t)g.rows, t.cols = g.cols, t.ld = g.ld, t.ldo = o ? o->ld : 0;
    t.rows_at_once = t.cols >= kChunk ? 1 : (int32_t)(kChunk / t.cols);
    *chunks = t.cols > kChunk ? t.rows * cdiv(t.cols, kChunk) : cdiv(t.rows, t.rows_at_once);
}
inline void put(DenseItem &t, const pdb_tensor &g, const pdb_tensor *, int64_t *chunks) {
    t.cols = g.rows * g.cols;
    *chunks = cdiv(t.cols, kChunk);
}

// A list of the tensors of [from, count) without gaps (DenseItem) or with (Item); the
// first that no longer went into it.
template <typename ITEM>
int64_t fill_list(const pdb_tensor *grads, const pdb_tensor *outs, int64_t from, int64_t count,
                  List<ITEM> *list) {
    list->count = 0;
    list->chunks = 0;
    int64_t i = from;
    for (; i < count && list->count < List<ITEM>::kMost && list->chunks < kMostChunks; ++i) {
        const pdb_tensor &g = grads[i];
        if (g.rows == 0 || g.cols == 0) continue;
        if (no_gaps(grads, outs, i) != std::is_same<ITEM, DenseItem>::value) continue;
        ITEM &t = list->item[list->count++];
        t.g = static_cast<const char *>(g.data);
        t.o = outs ? static_cast<char *>(outs[i].data) : nullptr;
        t.dt = (int16_t)g.dtype;
        t.odt = outs ? (int16_t)outs[i].dtype : 0;
        t.first = list->chunks;
        int64_t chunks = 0;
        put(t, g, outs ? &outs[i] : nullptr, &chunks);
        list->chunks += (uint32_t)chunks;
    }
    return i;
}

// Calls f for the lists of one kind, from the first tensor on.
template <typename ITEM, typename F>
int for_lists(const pdb_tensor *grads, const pdb_tensor *outs, int64_t count, F f) {
    List<ITEM> list;
    for (int64_t i = 0; i < count;) {
        i = fill_list(grads, outs, i, count, &list);
        if (list.count > 0)
            if (int e = f(list)) return e;
    }
    return PDB_OK;
}

// The same from the last list to the first.
template <typename ITEM, typename F>
int for_lists_back(const pdb_tensor *grads, const pdb_tensor *outs, int64_t count, F f) {
    List<ITEM> list;
    int32_t starts[kMostLists];
    int lists = 0;
    for (int64_t i = 0; i < count && lists < kMostLists; ++lists) {
        starts[lists] = (int32_t)i;
        i = fill_list(grads, outs, i, count, &list);
    }
    while (lists-- > 0) {
        fill_list(grads, outs, starts[lists], count, &list);
        if (list.count > 0)
            if (int e = f(list)) return e;
    }
    return PDB_OK;
}

unsigned blocks_of(uint32_t chunks) { return std::max(std::min<uint32_t>(chunks, kSums), 1u); }

// The sums of squares of all tensors; how many sums there are.
int sum_squares(const pdb_tensor *grads, int64_t count, double *sums, int *blocks,
                hipStream_t stream) {
    unsigned most = 1;
    auto widest = [&](const auto &list) -> int {
        most = std::max(most, blocks_of(list.chunks));
        return PDB_OK;
    };
    for_lists<Item>(grads, nullptr, count, widest);
    for_lists<DenseItem>(grads, nullptr, count, widest);
    *blocks = (int)most;
    bool add = false;
    // (the first launch gives every sum a value)
    auto squares = [&](const auto &list) -> int {
        k_grad_squares<<<add ? blocks_of(list.chunks) : most, kBlock, 0, stream>>>(list, sums, add);
        PDB_LAUNCHED();
        add = true;
        return PDB_OK;
    };
    if (int e = for_lists<Item>(grads, nullptr, count, squares)) return e;
    if (int e = for_lists<DenseItem>(grads, nullptr, count, squares)) return e;
    if (!add) {
        List<DenseItem> none;
        none.count = 0;
        none.chunks = 0;
        return squares(none);
    }
    return PDB_OK;
}

constexpr size_t kGradWs = kSums * sizeof(double);

}  // namespace
}  // namespace pdbk

using namespace pdbk;

extern "C" int pdb_grad_workspace_bytes(size_t *bytes) {
    if (!bytes) return PDB_ERR_INVALID_ARG;
    *bytes = kGradWs;
    return PDB_OK;
}

extern "C" int pdb_grad_norm(const pdb_tensor *grads, int64_t count, float scale, float *norm,
                             void *ws, size_t ws_bytes, hipStream_t stream) {
    if (int e = check_tensors(grads, count, nullptr)) return e;
    if (!isfinite(scale) || !norm || !aligned_to(norm, 4)) return PDB_ERR_INVALID_ARG;
    if (!ws || !aligned_to(ws, 8) || ws_bytes < kGradWs) return PDB_ERR_WORKSPACE;
    double *sums = static_cast<double *>(ws);
    int blocks = 0;
    if (int e = sum_squares(grads, count, sums, &blocks, stream)) return e;
    k_grad_norm<<<1, kBlock, 0, stream>>>(sums, blocks, scale, norm);
    PDB_LAUNCHED();
    return PDB_OK;
}

extern "C" int pdb_grad_clip(const pdb_tensor *grads, int64_t count, float scale, float max_norm,
                             float step, int accumulate, const pdb_tensor *outs, float *norm,
                             void *ws, size_t ws_bytes, hipStream_t stream) {
    if (count > 0 && !outs) return PDB_ERR_INVALID_ARG;
    if (int e = check_tensors(grads, count, outs)) return e;
    if (int e = check_apart(grads, outs, count)) return e;
    if (!isfinite(scale) || !isfinite(step) || !(max_norm >= 0.0f) || !norm || !aligned_to(norm, 4) ||
        (accumulate != 0 && accumulate != 1))
        return PDB_ERR_INVALID_ARG;
    if (!ws || !aligned_to(ws, 8) || ws_bytes < kGradWs) return PDB_ERR_WORKSPACE;
    double *sums = static_cast<double *>(ws);
    int blocks = 0;
    if (int e = sum_squares(grads, count, sums, &blocks, stream)) return e;
    // what was read last first
    bool first = true;
    auto clip = [&](const auto &list) -> int {
        k_grad_clip<<<blocks_of(list.chunks), kBlock, 0, stream>>>(list, sums, blocks, scale, max_norm,
                                                                  step, accumulate, first ? norm : nullptr);
        PDB_LAUNCHED();
        first = false;
        return PDB_OK;
    };
    if (int e = for_lists_back<DenseItem>(grads, outs, count, clip)) return e;
    if (int e = for_lists_back<Item>(grads, outs, count, clip)) return e;
    if (first) {
        List<DenseItem> none;
        none.count = 0;
        none.chunks = 0;
        return clip(none);
    }
    return PDB_OK;
}
