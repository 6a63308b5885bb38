// What the kernels on [tokens, channels] rows share: element types, the sequences that the rows belong to, and the activations.
#pragma once
#include "chela_internal.h"

namespace chela {

typedef __bf16 bf16;
typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned u32x2;

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(bf16 x) { return (float)x; }
template <typename IO> __device__ __forceinline__ IO from_f(float x) { return (IO)x; }      // (round to nearest even)

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// exp(x) for an argument that is already in units of ln 2
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float sigmoid_(float x) { return __builtin_amdgcn_rcpf(1.f + exp2_(-kLog2e * x)); }
// log(1 + exp(x)) = max(x, 0) + log(1 + e), e = exp(-|x|).  With w = 1 + e as rounded and r = e - (w - 1) what the rounding lost (exact, e
// being no larger than 1), log(1 + e) = log(w) + r / w, and 2 - w does for 1 / w: r is below 2^-24 and 2 - w off by (w - 1)^2.
// (log(w) alone loses all digits of a step size of 1e-6.)
__device__ __forceinline__ float softplus_(float x)
{
    const float e = exp2_(-kLog2e * fabsf(x)), w = 1.f + e;
    return fmaxf(x, 0.f) + fmaf(2.f - w, e - (w - 1.f), __builtin_amdgcn_logf(w) * kLn2);
}

// The sequences as the kernels see them (chela_internal.h: Rows).  Offsets out of [0, T] are taken for the nearest in it, so that whatever
// `cu` holds no row out of [0, T) is touched.
__device__ __forceinline__ int seq_begin(const Rows& r, int s)
{
    if (r.cu == nullptr) return s * r.L;
    const int b = r.cu[s];
    return b < 0 ? 0 : b > r.T ? r.T : b;
}
__device__ __forceinline__ int seq_end(const Rows& r, int s)
{
    return r.cu == nullptr ? (s + 1) * r.L : seq_begin(r, s + 1);
}
// The sequence that row t is in: -1 in front of the first one, n_seq behind the last one.
__device__ __forceinline__ int seq_of(const Rows& r, int t)
{
    if (r.cu == nullptr) return r.L > 0 ? t / r.L : r.n_seq;
    int lo = 0, hi = r.n_seq + 1;              // the first offset that is above t
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (r.cu[mid] > t) hi = mid; else lo = mid + 1;
    }
    return lo - 1;
}
// Where sequence s keeps its state, or -1: it has none.
__device__ __forceinline__ int slot_of(const Rows& r, int s)
{
    const int k = r.slots == nullptr ? s : r.slots[s];
    return k >= 0 && k < r.n_slots ? k : -1;
}

}  // namespace chela
