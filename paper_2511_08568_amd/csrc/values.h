// Vectors of table and gradient values: loads that widen to fp32, stores that
// round once (to nearest, ties to even).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/recmg.h"

namespace recmg {

template <int DT> struct Elem;
template <> struct Elem<RECMG_F32> { typedef float type; };
template <> struct Elem<RECMG_F16> { typedef _Float16 type; };
template <> struct Elem<RECMG_BF16> { typedef __bf16 type; };
template <int DT> using elem_t = typename Elem<DT>::type;

static inline int elem_size(int32_t dtype) { return dtype == RECMG_F32 ? 4 : 2; }

// V values from the address of one of them on.  Rows of any width and stride
// start anywhere, so only an element's own alignment is assumed; the hardware
// takes 16-byte accesses at any such address.
template <typename T, int V> struct Vec {
    typedef T raw __attribute__((ext_vector_type(V)));
    typedef raw type __attribute__((aligned(sizeof(T))));
};

template <typename T, int V> __device__ __forceinline__ void load_whole(const T *p, float (&x)[V]) {
    const typename Vec<T, V>::raw v = *reinterpret_cast<const typename Vec<T, V>::type *>(p);
#pragma unroll
    for (int k = 0; k < V; ++k) x[k] = (float)v[k];
}

// One row's values of `left` columns from p on (left >= 1); what lies behind them is 0.
template <typename T, int V>
__device__ __forceinline__ void load_vec(const T *p, int32_t left, float (&x)[V]) {
    if (left >= V) {
        load_whole<T, V>(p, x);
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k) x[k] = k < left ? (float)p[k] : 0.f;
    }
}

// N vectors from the addresses at(0), ... on, of `left` columns each: in flight together.  `whole` is the same in all
// lanes: every vector is V columns or none (left <= 0; x is then of no use), and the loads have no branches between them,
// which would make the compiler wait for each (norm of 800 MB of 290 tensors: 150 us, 188 with branches).
template <typename T, int V, int N, typename At>
__device__ __forceinline__ void load_vecs(bool whole, int32_t left, At at, float (&x)[N][V]) {
    if (whole) {
        if (left > 0)
#pragma unroll
            for (int k = 0; k < N; ++k) load_whole<T, V>(at(k), x[k]);
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) load_vec<T, V>(at(k), left, x[k]);
    }
}

// A value rounded to T.  The empty statement keeps a product apart from its rounding to fp16: the instruction that
// does both adds +0, which takes the sign of a product of -0.
template <typename T> __device__ __forceinline__ T rounded(float x) {
    if constexpr (__is_same(T, _Float16)) asm("" : "+v"(x));
    return (T)x;
}

// CACHED stores, or STREAM: past the caches, for what no kernel reads soon.
enum { CACHED = 0, STREAM = 1 };
template <typename T, int V, int HOW = CACHED>
__device__ __forceinline__ void store_vec(T *p, int32_t left, const float (&x)[V]) {
    if (left >= V) {
        typename Vec<T, V>::raw v;
#pragma unroll
        for (int k = 0; k < V; ++k) v[k] = rounded<T>(x[k]);
        if constexpr (HOW == STREAM) __builtin_nontemporal_store(v, reinterpret_cast<typename Vec<T, V>::type *>(p));
        else *reinterpret_cast<typename Vec<T, V>::type *>(p) = v;
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (k < left) p[k] = rounded<T>(x[k]);
    }
}

// A token id of either width.
__device__ __forceinline__ int64_t load_id(const void *ids, int32_t index_type, int64_t i) {
    return index_type == RECMG_I32 ? (int64_t) reinterpret_cast<const int32_t *>(ids)[i]
                                   : reinterpret_cast<const int64_t *>(ids)[i];
}

// The row of the table that a token id names, or -1 if it lies outside the table's part of the ids.
__device__ __forceinline__ int64_t local_row(int64_t id, int64_t first_row, int64_t rows) {
    // unsigned: an id far below first_row must not wrap into the table
    const uint64_t r = (uint64_t)id - (uint64_t)first_row;
    return id >= first_row && r < (uint64_t)rows ? (int64_t)r : -1;
}

}  // namespace recmg
