// What the norms share: a row in the registers of the threads that have it, and sums over them.
#pragma once
#include "chela_rows.h"

namespace chela {

// A thread's share of a row: NV pieces of four elements, 8 bytes (bf16) or 16 (fp32) at a time.  VEC: rows begin on a whole piece.  Otherwise
// they begin on an element (loads and stores of global memory need no more), and the up to three elements behind the last whole piece go to
// the row's first threads, one each: all loads stay on their way until they are needed.  (Element by element, the threads' next to each other,
// both directions took 489, 2522, 1820 us at 40 million elements in bf16 rows of 941, 4506, 8191; so they take 227, 385, 330, and those
// of 1000, 4096, 8192 200, 204, 222.)  Raw holds what was read as it lies in memory.
template <typename T, int TPR, int NV, bool VEC>
struct RowPart {
    static constexpr int E = NV * 4 + !VEC;
    typedef unsigned Piece __attribute__((ext_vector_type(sizeof(T))));          // (words: single elements would take a register each)
    struct __attribute__((packed, aligned(sizeof(T)))) Loose { Piece p; };
    struct Elements { T e[4]; };
    struct Raw { Piece p[NV]; T last; };
    static __device__ __forceinline__ void load(const T* row, int D, int tid, Raw& x)
    {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int k = (v * TPR + tid) * 4;
            x.p[v] = Piece(0);
            if (VEC) {
                if (k < D) x.p[v] = *reinterpret_cast<const Piece*>(row + k);
            } else {
                if (k + 4 <= D) x.p[v] = reinterpret_cast<const Loose*>(row + k)->p;
            }
        }
        if (!VEC) x.last = tid < D % 4 ? row[D / 4 * 4 + tid] : (T)0.f;
    }
    static __device__ __forceinline__ void widen(const Raw& x, float (&to)[E])
    {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const Elements t = __builtin_bit_cast(Elements, x.p[v]);
#pragma unroll
            for (int j = 0; j < 4; ++j) to[4 * v + j] = to_f(t.e[j]);
        }
        if (!VEC) to[E - 1] = to_f(x.last);
    }
    static __device__ __forceinline__ void load(const T* row, int D, int tid, float (&x)[E])
    {
        Raw r;
        load(row, D, tid, r);
        widen(r, x);
    }
    static __device__ __forceinline__ void store(T* row, int D, int tid, const float (&x)[E])
    {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int k = (v * TPR + tid) * 4;
            Elements t;
#pragma unroll
            for (int j = 0; j < 4; ++j) t.e[j] = from_f<T>(x[4 * v + j]);
            if (VEC) {
                if (k < D) *reinterpret_cast<Piece*>(row + k) = __builtin_bit_cast(Piece, t);
            } else {
                if (k + 4 <= D) reinterpret_cast<Loose*>(row + k)->p = __builtin_bit_cast(Piece, t);
            }
        }
        if (!VEC && tid < D % 4) row[D / 4 * 4 + tid] = from_f<T>(x[E - 1]);
    }
};

template <int CTRL>
__device__ __forceinline__ float plus_dpp(float x)
{
    return x + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float wave_sum(float x)
{
    x = plus_dpp<0xB1>(x);           // lanes that differ in bit 0, in bit 1, the other half of 8, of 16
    x = plus_dpp<0x4E>(x);
    x = plus_dpp<0x141>(x);
    x = plus_dpp<0x140>(x);
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

// Sums of K values over a row's threads; every thread returns with them.  s: room for K values per wave, not in use by the call before.
template <int TPR, int K>
__device__ __forceinline__ void row_sums(float (&x)[K], float (*s)[K])
{
#pragma unroll
    for (int k = 0; k < K; ++k) x[k] = wave_sum(x[k]);
    if (TPR == 64) return;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int k = 0; k < K; ++k) s[threadIdx.x >> 6][k] = x[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) x[k] = 0.f;
#pragma unroll
    for (int i = 0; i < TPR / 64; ++i)
#pragma unroll
        for (int k = 0; k < K; ++k) x[k] += s[i][k];
}

}  // namespace chela
