// Typed 16-byte vectors of the token operators (gfx950, wave64): unpacking to
// binary32, packing with one rounding, rows at any element alignment.
// Internal header, not installed.
#pragma once

#include "../../include/pdb_tokens.h"
#include "pdb_internal.h"

namespace pdbk {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// Rows of an odd stride start at any element: the 16-byte accesses go through
// types of element alignment (global memory takes them unaligned), so one
// path serves every base and stride.
typedef u32x4 u32x4_any __attribute__((aligned(2)));

__host__ __device__ constexpr int dtype_size(int dt) { return dt == PDB_F32 ? 4 : 2; }

template <int DT>
struct Elem {
    static constexpr int kSize = dtype_size(DT);
    static constexpr int kVec = 16 / kSize;  // elements of a 16-byte vector
};

__device__ __forceinline__ u32x4 load16(const void *p) {
    return *static_cast<const u32x4_any *>(p);
}
__device__ __forceinline__ void store16(void *p, u32x4 v) { *static_cast<u32x4_any *>(p) = v; }

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

template <int DT>
__device__ __forceinline__ void unpack(u32x4 r, float *x) {
    if constexpr (DT == PDB_F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(r[i]);
    } else if constexpr (DT == PDB_BF16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(r[i] << 16);
            x[2 * i + 1] = __uint_as_float(r[i] & 0xFFFF0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            // a copy first: a bit cast of the vector's element takes the first one
            const uint32_t w = r[i];
            const f16x2 h = __builtin_bit_cast(f16x2, w);
            x[2 * i] = (float)h[0];
            x[2 * i + 1] = (float)h[1];
        }
    }
}

template <int DT>
__device__ __forceinline__ u32x4 pack(const float *x) {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (DT == PDB_F32) {
            r[i] = __float_as_uint(x[i]);
        } else {
            const f32x2 f = {x[2 * i], x[2 * i + 1]};
            if constexpr (DT == PDB_BF16)
                r[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
            else
                r[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f, f16x2));
        }
    }
    return r;
}

template <int DT>
__device__ __forceinline__ float load1(const void *p, int64_t i) {
    if constexpr (DT == PDB_F32) return static_cast<const float *>(p)[i];
    if constexpr (DT == PDB_BF16)
        return __uint_as_float((uint32_t) static_cast<const uint16_t *>(p)[i] << 16);
    if constexpr (DT == PDB_F16) return (float)static_cast<const _Float16 *>(p)[i];
}

template <int DT>
__device__ __forceinline__ void store1(void *p, int64_t i, float x) {
    if constexpr (DT == PDB_F32) static_cast<float *>(p)[i] = x;
    if constexpr (DT == PDB_BF16) static_cast<__bf16 *>(p)[i] = (__bf16)x;
    if constexpr (DT == PDB_F16) static_cast<_Float16 *>(p)[i] = (_Float16)x;
}

template <int DT>
__device__ __forceinline__ const char *elem_at(const void *p, int64_t i) {
    return static_cast<const char *>(p) + i * Elem<DT>::kSize;
}
template <int DT>
__device__ __forceinline__ char *elem_at(void *p, int64_t i) {
    return static_cast<char *>(p) + i * Elem<DT>::kSize;
}

// E elements (a multiple of the type's vector) at element i
template <int DT, int E>
__device__ __forceinline__ void load_elems(const void *p, int64_t i, float *x) {
    constexpr int kV = Elem<DT>::kVec;
    static_assert(E % kV == 0, "whole vectors");
#pragma unroll
    for (int k = 0; k < E / kV; ++k) unpack<DT>(load16(elem_at<DT>(p, i + k * kV)), x + k * kV);
}
template <int DT, int E>
__device__ __forceinline__ void store_elems(void *p, int64_t i, const float *x) {
    constexpr int kV = Elem<DT>::kVec;
#pragma unroll
    for (int k = 0; k < E / kV; ++k) store16(elem_at<DT>(p, i + k * kV), pack<DT>(x + k * kV));
}

// A token as int32: -1 for padding and, noted in *status, for one >= v.
template <typename I>
__device__ __forceinline__ int32_t read_token(const I *tokens, int64_t i, int64_t v,
                                              int32_t *status) {
    const I t = tokens[i];
    if (t >= 0 && (int64_t)t >= v) {
        if (status) *status = PDB_ERR_INVALID_ARG;
        return -1;
    }
    return t < 0 ? -1 : (int32_t)t;
}
__device__ __forceinline__ int32_t read_token(const void *tokens, int index, int64_t i, int64_t v,
                                              int32_t *status) {
    return index == PDB_I64 ? read_token(static_cast<const int64_t *>(tokens), i, v, status)
                            : read_token(static_cast<const int32_t *>(tokens), i, v, status);
}

// ----------------------------------------------------------------------------
// host-side checks
inline bool is_dtype(int dt) { return dt == PDB_F32 || dt == PDB_F16 || dt == PDB_BF16; }
inline bool is_index(int ix) { return ix == PDB_I32 || ix == PDB_I64; }
inline bool aligned_to(const void *p, int size) { return (uintptr_t)p % (size_t)size == 0; }
// a matrix of `rows` x `cols` at p: PDB_OK, or why it cannot be used
inline int check_matrix(const void *p, int dt, int64_t ld, int64_t rows, int64_t cols) {
    if (!is_dtype(dt) || rows < 0 || cols < 0) return PDB_ERR_INVALID_ARG;
    if (rows > INT32_MAX || cols > INT32_MAX || ld > ((int64_t)1 << 40)) return PDB_ERR_UNSUPPORTED;
    if (rows > 1 && ld < cols) return PDB_ERR_INVALID_ARG;
    if (rows > 0 && cols > 0 && (!p || !aligned_to(p, dtype_size(dt)))) return PDB_ERR_INVALID_ARG;
    return PDB_OK;
}
inline int check_tokens(const void *t, int index, int64_t n) {
    if (!is_index(index) || n < 0) return PDB_ERR_INVALID_ARG;
    if (n > INT32_MAX) return PDB_ERR_UNSUPPORTED;
    if (n > 0 && (!t || !aligned_to(t, index == PDB_I64 ? 8 : 4))) return PDB_ERR_INVALID_ARG;
    return PDB_OK;
}

// Calls f with the dtype as a compile-time constant.
template <int DT>
struct DtypeTag {
    static constexpr int value = DT;
};
template <typename F>
inline int with_dtype(int dt, F f) {
    switch (dt) {
    case PDB_F32: return f(DtypeTag<PDB_F32>());
    case PDB_F16: return f(DtypeTag<PDB_F16>());
    case PDB_BF16: return f(DtypeTag<PDB_BF16>());
    }
    return PDB_ERR_INVALID_ARG;
}

}  // namespace pdbk
