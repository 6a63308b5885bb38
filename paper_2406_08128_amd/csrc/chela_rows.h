// What the kernels on [tokens, channels] rows share: element types, the sequences that the rows belong to, and the activations.
#pragma once
#include "chela_internal.h"

namespace chela {

typedef __bf16 bf16;
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
    return __builtin_amdgcn_fmed3f(x, 0.f, __builtin_inff()) + fmaf(2.f - w, e - (w - 1.f), __builtin_amdgcn_logf(w) * kLn2);
}
// ... and its slope, 1 / (1 + exp(-x))
__device__ __forceinline__ float softplus_(float x, float* slope)
{
    const float e = exp2_(-kLog2e * fabsf(x)), w = 1.f + e, r = __builtin_amdgcn_rcpf(w);
    *slope = x < 0.f ? e * r : r;
    return __builtin_amdgcn_fmed3f(x, 0.f, __builtin_inff()) + fmaf(2.f - w, e - (w - 1.f), __builtin_amdgcn_logf(w) * kLn2);
}

// A lane's element of a row whose address all lanes share: scalar base, 32-bit offset in bytes.  (The empty instructions keep the base in
// scalar registers and the offset in 32 bits where it is used: the compiler adds lane and base first otherwise, or widens the offset in
// front of the loop, and a 64-bit vector addition per row and tensor remains.)
#define CHELA_GLOBAL __attribute__((address_space(1)))
template <typename T> __device__ __forceinline__ T row_load(const T* row, unsigned off)
{
    const CHELA_GLOBAL char* p = (const CHELA_GLOBAL char*)row;
    asm("" : "+s"(p), "+v"(off));
    return *(const CHELA_GLOBAL T*)(p + off);
}
template <typename T> __device__ __forceinline__ void row_store(T* row, unsigned off, T x)
{
    CHELA_GLOBAL char* p = (CHELA_GLOBAL char*)row;
    asm("" : "+s"(p), "+v"(off));
    *(CHELA_GLOBAL T*)(p + off) = x;
}
// Rows one after the other, the last one again behind it: where the next one is, and how far it is to the one after.
template <typename T>
struct RowWalk {
    const char* p;
    unsigned step;
    __device__ __forceinline__ void start(const void* base, long ld, int row) { p = (const char*)((const T*)base + (long)row * ld); step = (unsigned)ld * sizeof(T); }
    __device__ __forceinline__ T get(unsigned off) const { return row_load((const T*)p, off); }
    __device__ __forceinline__ void next(bool on) { p += on ? step : 0u; }
    __device__ __forceinline__ void back(bool on) { p -= on ? step : 0u; }
};

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
// The same, by all 64 lanes of a wave together: 64 offsets at a time, so that the wave waits once for up to 64 offsets and twice up to 4096.
// (One by one, 11 sequences took four waits in a row, two of the 50 us that a wave of 48 rows has in all.)
__device__ __forceinline__ int seq_of_wave(const Rows& r, int t, int lane)
{
    if (r.cu == nullptr) return r.L > 0 ? t / r.L : r.n_seq;
    int first = 0, n = r.n_seq + 1;            // the offsets in question
    while (n > 64) {
        const int step = (n + 63) / 64;
        const int i = lane * step;
        const int below = __popcll(__ballot(i < n && r.cu[first + min(i, n - 1)] <= t));
        if (below == 0) return first - 1;
        const int skip = min((below - 1) * step, n - 1);
        first += skip;
        n = min(step, n - skip);
    }
    return first - 1 + __popcll(__ballot(lane < n && r.cu[first + min(lane, n - 1)] <= t));
}
// Where sequence s keeps its state, or -1: it has none.
__device__ __forceinline__ int slot_of(const Rows& r, int s)
{
    const int k = r.slots == nullptr ? s : r.slots[s];
    return k >= 0 && k < r.n_slots ? k : -1;
}

}  // namespace chela
