// Rows of fp32, fp16 or bf16 in vectors of 16 bytes, and what the calls on them have in common.
#pragma once

#include "dgq_internal.h"

namespace dgq {

template <class T>
constexpr int kVec = 16 / (int)sizeof(T);

// Memory operations of gfx950 need no alignment beyond the element's, so odd widths and strides take the same loads.
template <class T, int N>
using loose [[gnu::aligned(alignof(T))]] = T __attribute__((ext_vector_type(N)));

// The first `have` of a vector's elements, the others 0.
template <class T, int V>
__device__ inline void load_vector(const T *from, int have, float (&f)[V]) {
    if (have >= V) {
        const loose<T, V> x = *reinterpret_cast<const loose<T, V> *>(from);
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = (float)x[i];
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = i < have ? (float)from[i] : 0.f;
    }
}
template <class T, int V>
__device__ inline void store_vector(T *to, int have, const float (&f)[V]) {
    if (have >= V) {
        loose<T, V> x;
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = (T)f[i];
        *reinterpret_cast<loose<T, V> *>(to) = x;
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < have) to[i] = (T)f[i];
    }
}

// The same for what no cache need keep (nontemporal): whole vectors.
template <class V>
__device__ inline V load_past(const V *from) {
    return __builtin_nontemporal_load(from);
}
template <class T, int V>
__device__ inline void store_past(T *to, int have, const float (&f)[V]) {
    if (have < V) return store_vector(to, have, f);
    loose<T, V> x;
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = (T)f[i];
    __builtin_nontemporal_store(x, reinterpret_cast<loose<T, V> *>(to));
}

// t / (1 + exp(-t)) with the hardware's 2^x and 1 / x, good to one unit in the last place each; the exponent's own rounding adds
// |t| 2^-24.  Below -87.3, where 1 / x would be below 2^-126, it may be 0 for what is there up to 10^-36.
__device__ inline float silu(float t) {
    return t * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(t * -1.44269504088896341f));
}

// f with a value of the C type of a dgq_dtype; of an output's, which is x's own type or fp32.
template <class F>
void by_dtype(int32_t t, F f) {
    t == DGQ_F32 ? f(float{}) : t == DGQ_F16 ? f(_Float16{}) : f(__bf16{});
}
template <class T, class F>
void by_output(int32_t t, F f) {
    if constexpr (sizeof(T) == 4) f(float{});
    else if (t == DGQ_F32) f(float{});
    else f(T{});
}

}  // namespace dgq
