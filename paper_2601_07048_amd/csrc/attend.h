// Attention beside the index: argument records and launchers (host), element types and 8-element loads (device).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "../../include/jx.h"

namespace jx {

// ---- launchers: arguments have been checked by the entry points ------------------------------------------------------
struct KvPlanArgs {
    const int32_t *len, *add;
    int n_req, page_shift;
    int32_t* table;
    int table_pages;
    const int32_t *free_pages, *n_free;
    int n_pages;
    int32_t *n_free_out, *q_start, *kv_len, *pos;
    int64_t* slot;
    long long n_tokens;
};
hipError_t launch_kv_plan(const KvPlanArgs& a, hipStream_t st);
hipError_t launch_kv_release(const int32_t* first, const int32_t* end, int n_req, int32_t* table, int table_pages, int32_t* free_pages,
                             int32_t* n_free, int n_pages, hipStream_t st);
hipError_t launch_qk_norm_rope(const jx_rope_args& a, hipStream_t st);
int64_t paged_attention_bytes(const jx_attend_args& a);
hipError_t launch_paged_attention(const jx_attend_args& a, uint8_t* work, hipStream_t st);
hipError_t launch_found_attention(const jx_found_args& a, hipStream_t st);

// the smallest power of two of 8-element chunks that holds a row, 8..32
inline int row_lanes(int head_dim) { return head_dim <= 64 ? 8 : head_dim <= 128 ? 16 : 32; }
inline int log2_of(int power) { return 31 - __builtin_clz((unsigned)power); }

// Threads of a launch, in all; it has to be less than 2^32.  Norm and rotation: a group of lanes takes a head of a token, or four from as
// many heads on as the card holds lanes at a time
inline bool rope_many(const jx_rope_args& a) { return a.n_tokens * (a.n_heads + 2ll * a.n_kv_heads) * row_lanes(a.head_dim) > 256 * 2048; }
inline int64_t rope_threads(const jx_rope_args& a) {
    const int64_t rows = a.n_heads + 2ll * a.n_kv_heads;
    return (a.n_tokens * (rope_many(a) ? (rows + 3) / 4 : rows) * row_lanes(a.head_dim) + 255) / 256 * 256;
}
inline int64_t found_threads(const jx_found_args& a) { return (a.n_tokens * a.n_heads + 3) / 4 * 256; }

// ---- device ----------------------------------------------------------------------------------------------------------
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

template <typename T>
struct Vec;
template <>
struct Vec<__bf16> {
    typedef __bf16 x8 __attribute__((ext_vector_type(8)));
    typedef __bf16 x4 __attribute__((ext_vector_type(4)));
    typedef __bf16 x2 __attribute__((ext_vector_type(2)));
};
template <>
struct Vec<_Float16> {
    typedef _Float16 x8 __attribute__((ext_vector_type(8)));
    typedef _Float16 x4 __attribute__((ext_vector_type(4)));
    typedef _Float16 x2 __attribute__((ext_vector_type(2)));
};

template <typename T>
__device__ __forceinline__ f32x8 load8(const T* p) {
    return __builtin_convertvector(*reinterpret_cast<const typename Vec<T>::x8*>(p), f32x8);
}
// rounds to nearest even
template <typename T>
__device__ __forceinline__ void store8(T* p, f32x8 v) {
    *reinterpret_cast<typename Vec<T>::x8*>(p) = __builtin_convertvector(v, typename Vec<T>::x8);
}

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

}  // namespace jx
