// Gated delta rule, gradient, gfx950.  Names as in the forward's file; S is the state in front of a chunk, dS_next the gradient of the one behind.
//
//     dU = P^T dO + K~ dS_next,   dR = T^T dU,   dV = beta dR,
//     X = scale D o (dO U^T) for s <= t,   Y = D o (dR U^T) for s < t,
//     dQ = scale e^gamma dO S^T + X K,   read = -beta (e^gamma dR S^T + Y K),   carry = e^(gamma_C - gamma) U dS_next^T,
//     write = carry + X^T Q - (beta Y)^T K,   dK = read + write,
//     dbeta_t = dR_t . v_t - k_t . (e^gamma_t S dR_t) - sum_s Y_ts k_t . k_s,
//     dg_t = e^gamma_C <S, dS_next> + sum_{u >= t} near_u + sum_{s < t} k_s . carry_s + sum_{s < t <= u} W_us,
//         near_u = q_u . (scale e^gamma dO S^T)_u - beta_u k_u . (e^gamma dR S^T)_u,   W_us = X_us q_u . k_s - beta_u Y_us k_u . k_s.
// (The same dg_t is a sum over all tokens from t on of q . dQ, and so on, in which pairs on one side of t cancel but for roundings.  Of those that t divides,
// each has the factor e^g_t: where little is let through little is added up, and nothing where nothing is.)
//     dS = w dS_next - N^T dS_next + Z' (w and N as forward),   Z' = scale (e^gamma Q)^T dO - (beta e^gamma K)^T T^T P^T dO.
// Three launches, as forward: N^T and Z' of all chunks, the walk from the last chunk to the first, all gradients.
#include "chela_delta.h"

namespace chela {

// ---- a chunk's N^T and Z'.  32768 tokens in 8 sequences, 12 heads of 64 and 128 (4 key heads): 120 us, 440 MB at 3.7 TB/s.
// P's transpose and T are in the same place one after the other, P^T dO in registers meanwhile.
template <typename E, int DK, int DV, int P>
__global__ __launch_bounds__(256, 2) void delta_bwd_prep_kernel(DeltaArgs a)
{
    constexpr int C = DeltaChunk<E>::C, NB = C / 16, KC = C / 32, KS = DK / 32, LK = DK + kPad<E>, LV = DV + kPad<E>, LT = C + kPad<E>;
    __shared__ __align__(16) E sQ[C * LK], sK[C * LK], sO[C * LV], sT[kScores<E>];         // (P's transpose, then T)
    __shared__ ChunkSteps<C> st;
    __shared__ __align__(16) float s_qu[C];                        // scale e^gamma
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), q = lane >> 4, c = lane & 15;
    const int place = blockIdx.x / a.H, h = blockIdx.x - place * a.H, hk = h / (a.H / a.Hk);
    const Chunk ch = chunk_at(a.rows, C, place, lane);
    if (ch.n <= 0) return;
    const size_t at = (size_t)place * a.H + h;
    PackedT<E, C, 256> m;
    {
        Tile<E, C, DK> y, k;
        Tile<E, C, DV> o;
        const Steps s = fetch_steps((const E*)a.g, a.ldg, (const E*)a.beta, a.ldb, ch.row, h, ch.n, lane);
        y.fetch((const E*)a.Q + hk * DK, a.ldq, ch.row, ch.n, tid);
        k.fetch((const E*)a.K + hk * DK, a.ldk, ch.row, ch.n, tid);
        o.fetch((const E*)a.dO + h * DV, a.lddo, ch.row, ch.n, tid);
        m.fetch((const E*)a.T + at * (C * C), tid);
        put_steps(st, s, ch.n, tid);
        y.put(sQ, LK, ch.n, tid);
        k.put(sK, LK, ch.n, tid);
        o.put(sO, LV, ch.n, tid);
    }
    __syncthreads();
    if (tid == 0) a.whole[at] = no_growth(st.whole);
    const float grown = st.whole - no_growth(st.whole);
    const Planes<E, 2> T{sT, LT, C * LT};
    if (w < NB) {                                                  // P's transpose, sixteen of its rows to a wave
        const int s = 16 * w + c;
        for (int tb = w & ~1; tb < NB; ++tb) {
            f32x4 x = zero4();
            if (tb >= w) {
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) x = mma(rows_op(sQ, LK, 16 * tb, 32 * ks, lane), rows_op(sK, LK, 16 * w, 32 * ks, lane), x);
                x *= splat4(a.scale) * st.decays_to(16 * tb + 4 * q, s);
                if (tb == w)
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[i] = c <= 4 * q + i ? x[i] : 0.f;
            }
            T.put4(s, 16 * tb, q, x);
        }
    }
    if (tid < C) s_qu[tid] = a.scale * st.up[tid];
    __syncthreads();
    f32x4 po[DV / 64][NB];                                         // P^T dO of the wave's value columns, sixteen of every 64
#pragma unroll
    for (int i = 0; i < DV / 64; ++i) {
        read_afresh();
#pragma unroll
        for (int b = 0; b < NB; ++b) po[i][b] = zero4();
#pragma unroll
        for (int ks = 0; ks < KC; ++ks) {
            const Op<E, 1> o = cols_op(sO, LV, 32 * ks, 64 * i + 16 * w, lane);
#pragma unroll
            for (int b = 0; b <= 2 * ks + 1; ++b) po[i][b] = mma(T.rows(16 * b, 32 * ks, lane), o, po[i][b]);
        }
    }
    __syncthreads();
    m.put(T, tid);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < (DK + DV) / 64; ++i) {
        const int p = 4 * i + w;
        read_afresh();
        f32x4 x[NB];
        Op<E, 2> xo[KC];
        if (i < DV / 64) {
            Op<E, 2> qo[KC];
#pragma unroll
            for (int ks = 0; ks < KC; ++ks) {
                qo[ks] = scaled<E, 2>(cols_op(sO, LV, 32 * ks, 16 * p, lane), s_qu, 32 * ks, lane);
                xo[ks] = operand<E, 2>(po[i < DV / 64 ? i : 0][2 * ks], po[i < DV / 64 ? i : 0][2 * ks + 1]);
            }
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                x[b] = zero4();
#pragma unroll
                for (int ks = b / 2; ks < KC; ++ks) x[b] = mma(T.cols(32 * ks, 16 * b, lane), xo[ks], x[b]);
                x[b] *= *(const f32x4*)(st.bu + 16 * b + 4 * q);
            }
#pragma unroll
            for (int ks = 0; ks < KC; ++ks) xo[ks] = operand<E, 2>(x[2 * ks], x[2 * ks + 1]);
#pragma unroll
            for (int n = 0; n < DK / 16; ++n) {
                f32x4 z = zero4();
#pragma unroll
                for (int ks = 0; ks < KC; ++ks) {
                    z = mma(cols_op(sK, LK, 32 * ks, 16 * n, lane), xo[ks], z);
                    z = mma(cols_op(sQ, LK, 32 * ks, 16 * n, lane), qo[ks], z);
                }
                *(f32x4*)(a.Z + at * (DK * DV) + (size_t)(p * (DK / 16) + n) * 256 + 4 * lane) = z;
            }
        } else {
            const int g = p - DV / 16;
#pragma unroll
            for (int b = 0; b < NB; ++b) x[b] = zero4();
#pragma unroll
            for (int ks = 0; ks < KC; ++ks) {
                const Op<E, 2> k = scaled<E, 2>(cols_op(sK, LK, 32 * ks, 16 * g, lane), st.bu, 32 * ks, lane);
#pragma unroll
                for (int b = 2 * ks; b < NB; ++b) x[b] = mma(T.rows(16 * b, 32 * ks, lane), k, x[b]);
            }
#pragma unroll
            for (int b = 0; b < NB; ++b) x[b] *= *(const f32x4*)(st.down + 16 * b + 4 * q);
#pragma unroll
            for (int ks = 0; ks < KC; ++ks) xo[ks] = operand<E, 2>(x[2 * ks], x[2 * ks + 1]);
#pragma unroll
            for (int n = 0; n < KS; ++n) {
                f32x4 r0 = zero4(), r1 = zero4();
                if (n == g / 2) {
                    if (g % 2 == 0) r0 = plus_diagonal(r0, grown, lane);
                    else r1 = plus_diagonal(r1, grown, lane);
                }
#pragma unroll
                for (int ks = 0; ks < KC; ++ks) {
                    r0 = mma(cols_op(sK, LK, 32 * ks, 32 * n, lane), xo[ks], r0);
                    r1 = mma(cols_op(sK, LK, 32 * ks, 32 * n + 16, lane), xo[ks], r1);
                }
                store_op<E, P>((E*)a.N + (at * (DK / 16 * KS) + g * KS + n) * kOpElems<E, P>, operand<E, P>(r0, r1), lane);
            }
        }
    }
}

// ---- the same for a run of chunks, from its last to its first: one N^T and one Z' for all of them.  What a chunk makes of a state's gradient,
//     dS <- e^gamma dS + scale (e^gamma Q)^T dO - (beta e^gamma K)^T T^T (P^T dO + K~ dS),
// with Z' beside what is left of the identity (X = M^T - w, as forward, without the terms in dO), thirty-two columns to a wave.  65536 tokens in 4
// sequences, 12 heads of 64: 149 us, 400 MB at 2.7 TB/s: instruction issue, vector instructions 70 % of the time, matrix 30, with three waves to a SIMD
// (154 registers; heads of 128 up to 197, two waves).
template <typename E, int DK, int DV, int P>
__global__ __launch_bounds__((DK + DV) * 2) void delta_bwd_prep_run_kernel(DeltaArgs a)
{
    constexpr int C = DeltaChunk<E>::C, NB = C / 16, KC = C / 32, KS = DK / 32, LK = DK + kPad<E>, LV = DV + kPad<E>, LT = C + kPad<E>;
    constexpr int NT = (DK + DV) * 2, NW = NT / 64;
    __shared__ __align__(16) E sQ[C * LK], sK[C * LK], sO[C * LV], sT[kScores<E>];         // (P's transpose, then T)
    __shared__ ChunkSteps<C> st;
    const int tid0 = threadIdx.x, lane0 = tid0 & 63, w = __builtin_amdgcn_readfirstlane(tid0 >> 6);
    const int place = blockIdx.x / a.H, h = blockIdx.x - place * a.H, hk = h / (a.H / a.Hk);
    const Chunk ch = chunk_at(a.rows, C * a.run, place, lane0);
    if (ch.n <= 0) return;
    const size_t at = (size_t)place * a.H + h;
    const int chunk0 = chunk_place(a.rows, C, ch, a.run, 0), n_chunks = (ch.n + C - 1) / C;
    const bool of_k = w < DK / 32;
    const int col = 32 * (of_k ? w : w - DK / 32);
    Tile<E, C, DK, NT> tq, tk;
    Tile<E, C, DV, NT> to;
    PackedT<E, C, NT> tt;
    Steps ts;
    auto fetch = [&](int r, int tid, int lane) {
        const int row = ch.row + r * C, n = min(C, ch.n - r * C);
        ts = fetch_steps((const E*)a.g, a.ldg, (const E*)a.beta, a.ldb, row, h, n, lane);
        tq.fetch((const E*)a.Q + hk * DK, a.ldq, row, n, tid);
        tk.fetch((const E*)a.K + hk * DK, a.ldk, row, n, tid);
        to.fetch((const E*)a.dO + h * DV, a.lddo, row, n, tid);
    };
    fetch(n_chunks - 1, tid0, lane0);
    const Planes<E, 2> T{sT, LT, C * LT};
    f32x4 X[DK / 16][2];
#pragma unroll
    for (int d = 0; d < DK / 16; ++d) X[d][0] = X[d][1] = zero4();
    float before = 1.f;
    for (int r = n_chunks - 1; r >= 0; --r) {
        const int n = min(C, ch.n - r * C);
        const bool first = r == n_chunks - 1;
        int lane = lane0;
        asm volatile("" : "+v"(lane));             // (addresses are worked out where they are used)
        const int tid = 64 * w + lane, q = lane >> 4, c = lane & 15;
        if (!first) __syncthreads();
        put_steps(st, ts, n, tid);
        tq.put(sQ, LK, n, tid);
        tk.put(sK, LK, n, tid);
        to.put(sO, LV, n, tid);
        tt.fetch((const E*)a.T + ((size_t)(chunk0 + r) * a.H + h) * (C * C), tid);
        __syncthreads();
        {
            constexpr int GI = NW / NB > 0 ? NW / NB : 1;
            const int tw = w % NB, gi = w / NB, s = 16 * tw + c;
            if (gi < GI)
                for (int tb = (tw & ~1) + gi; tb < NB; tb += GI) {     // P's transpose, sixteen of its rows to a wave
                    f32x4 x = zero4();
                    if (tb >= tw) {
#pragma unroll
                        for (int ks = 0; ks < KS; ++ks) x = mma(rows_op(sQ, LK, 16 * tb, 32 * ks, lane), rows_op(sK, LK, 16 * tw, 32 * ks, lane), x);
                        x *= splat4(a.scale) * st.decays_to(16 * tb + 4 * q, s);
                        if (tb == tw)
#pragma unroll
                            for (int i = 0; i < 4; ++i) x[i] = c <= 4 * q + i ? x[i] : 0.f;
                    }
                    T.put4(s, 16 * tb, q, x);
                }
        }
        f32x4 y[NB][2];
#pragma unroll
        for (int b = 0; b < NB; ++b) y[b][0] = y[b][1] = zero4();
        if (of_k)
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int g = 0; g < 2; ++g) y[b][g] = splat4(before) * tile_of(sK, LK, 16 * b, col + 16 * g, lane);
        if (!first)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                read_afresh();
                const Op<E, 2> x0 = operand<E, 2>(X[2 * ks][0], X[2 * ks + 1][0]), x1 = operand<E, 2>(X[2 * ks][1], X[2 * ks + 1][1]);
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    const Op<E, 1> k = rows_op(sK, LK, 16 * b, 32 * ks, lane);
                    y[b][0] = mma(k, x0, y[b][0]);
                    y[b][1] = mma(k, x1, y[b][1]);
                }
            }
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const f32x4 d = *(const f32x4*)(st.down + 16 * b + 4 * q);
            y[b][0] *= d;
            y[b][1] *= d;
        }
        __syncthreads();
        if (!of_k)
#pragma unroll
            for (int ks = 0; ks < KC; ++ks) {
                const Op<E, 1> o0 = cols_op(sO, LV, 32 * ks, col, lane), o1 = cols_op(sO, LV, 32 * ks, col + 16, lane);
#pragma unroll
                for (int b = 0; b <= 2 * ks + 1; ++b) {
                    const Op<E, 2> m = T.rows(16 * b, 32 * ks, lane);
                    y[b][0] = mma(m, o0, y[b][0]);
                    y[b][1] = mma(m, o1, y[b][1]);
                }
            }
        __syncthreads();
        tt.put(T, tid);
        if (r > 0) fetch(r - 1, tid, lane);
        __syncthreads();
        Op<E, 2> yo[KC][2];
#pragma unroll
        for (int ks = 0; ks < KC; ++ks)
#pragma unroll
            for (int g = 0; g < 2; ++g) yo[ks][g] = operand<E, 2>(y[2 * ks][g], y[2 * ks + 1][g]);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            y[b][0] = y[b][1] = zero4();
#pragma unroll
            for (int ks = b / 2; ks < KC; ++ks) {
                const Op<E, 2> m = T.cols(32 * ks, 16 * b, lane);
                y[b][0] = mma(m, yo[ks][0], y[b][0]);
                y[b][1] = mma(m, yo[ks][1], y[b][1]);
            }
            const f32x4 f = *(const f32x4*)(st.bu + 16 * b + 4 * q);
            y[b][0] *= f;
            y[b][1] *= f;
        }
#pragma unroll
        for (int ks = 0; ks < KC; ++ks)
#pragma unroll
            for (int g = 0; g < 2; ++g) yo[ks][g] = operand<E, 2>(y[2 * ks][g], y[2 * ks + 1][g]);
        const float whole = st.whole, after = no_growth(before * whole), grown = before * whole - after;
#pragma unroll
        for (int d = 0; d < DK / 16; ++d) {
            if (d % 2 == 0) read_afresh();
            X[d][0] *= splat4(whole);
            X[d][1] *= splat4(whole);
            if (d / 2 == w) X[d][d % 2] = plus_diagonal(X[d][d % 2], grown, lane);        // (only of X, whose waves come first)
#pragma unroll
            for (int ks = 0; ks < KC; ++ks) {
                const Op<E, 1> k = cols_op(sK, LK, 32 * ks, 16 * d, lane);
                X[d][0] = mma(k, yo[ks][0], X[d][0]);
                X[d][1] = mma(k, yo[ks][1], X[d][1]);
            }
        }
        if (!of_k) {
            Op<E, 2> qo[KC][2];
#pragma unroll
            for (int ks = 0; ks < KC; ++ks)
#pragma unroll
                for (int g = 0; g < 2; ++g) qo[ks][g] = scaled<E, 2>(cols_op(sO, LV, 32 * ks, col + 16 * g, lane), st.up, 32 * ks, lane, a.scale);
#pragma unroll
            for (int d = 0; d < DK / 16; ++d) {
                if (d % 2 == 0) read_afresh();
#pragma unroll
                for (int ks = 0; ks < KC; ++ks) {
                    const Op<E, 1> k = cols_op(sQ, LK, 32 * ks, 16 * d, lane);
                    X[d][0] = mma(k, qo[ks][0], X[d][0]);
                    X[d][1] = mma(k, qo[ks][1], X[d][1]);
                }
            }
        }
        before = after;
    }
    if (of_k) {
        // as it is read, the columns of X down the rows of a tile: by products with the identity
        const int q = lane0 >> 4, c = lane0 & 15;
#pragma unroll
        for (int n = 0; n < DK / 16; n += 2) {
            const Op<E, 2> x0 = operand<E, 2>(X[n][0], X[n + 1][0]), x1 = operand<E, 2>(X[n][1], X[n + 1][1]);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                f32x4 lo = zero4(), hi = zero4();
#pragma unroll
                for (int j = 0; j < 4; ++j) lo[j] = 4 * q + j == c ? 1.f : 0.f;
                const Op<E, 1> one = i == 0 ? operand<E, 1>(lo, hi) : operand<E, 1>(hi, lo);
                store_op<E, P>((E*)a.N + (at * (DK / 16 * KS) + (n + i) * KS + w) * kOpElems<E, P>,
                               operand<E, P>(mma(x0, one, zero4()), mma(x1, one, zero4())), lane0);
            }
        }
    } else {
#pragma unroll
        for (int d = 0; d < DK / 16; ++d)
#pragma unroll
            for (int g = 0; g < 2; ++g) *(f32x4*)(a.Z + at * (DK * DV) + (size_t)((col / 16 + g) * (DK / 16) + d) * 256 + 4 * lane0) = X[d][g];
    }
    if (tid0 == 0) a.whole[at] = before;
}

__device__ __forceinline__ float dot4(f32x4 a, f32x4 b) { return fmaf(a[0], b[0], fmaf(a[1], b[1], fmaf(a[2], b[2], a[3] * b[3]))); }
template <typename E> __device__ __forceinline__ f32x4 wide4(const E* p) { return __builtin_convertvector(*(const Vec4<E>*)p, f32x4); }
// over the four lanes that have a column of a tile
__device__ __forceinline__ float column_sum(float x)
{
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}
// A workgroup has a chunk and a key head, and goes over that one's value heads: the sums of dQ and dK over them stay in registers.  RUN: a run of chunks
// and a head, from the last chunk to the first with the gradient of the state behind each in registers, sixteen value columns to a wave.  Sixteen value
// columns to a wave for U and dR; then sixteen tokens, as queries and as keys, and a part of the key columns.  X and Y are worked out twice, by the wave
// of the query's tokens and by that of the key's: as the operands of its own products they then lie in a wave's registers as they are.
// 65536 tokens in 4 sequences, 12 heads of 64: 377 us, 900 MB at 2.4 TB/s; 32768 in 8, 12 heads of 64 and 128 with 4 key heads: 316.  Two waves to a SIMD
// wait for LDS and each other half the time (eight barriers to a chunk, ten with 128 key columns; vector instructions 45 % of the time, LDS 40, matrix
// instructions 18).  Registers (199 to 256 in bf16) and LDS (76 KB with heads of 64, twice that where there are 128 value columns) each allow two; with 128 key and
// 64 value columns 92 KB and 256 registers, more of them for accumulators, allow one.  (dg by the pairs that a token divides, of that, where there are decays: 25 and 16;
// both parts of P and T 20 and 10.)
template <typename E, int DK, int DV, bool RUN>
__global__ __launch_bounds__(DV * 4, 2) void delta_grad_kernel(DeltaArgs a)
{
    constexpr int C = DeltaChunk<E>::C, NB = C / 16, KC = C / 32, KS = DK / 32, VS = DV / 32, LK = DK + kPad<E>, LV = DV + kPad<E>;
    // Key columns of S and dS_next at a time, and tiles of them to a wave.  (fp32, 64 value columns: with 64 of them two workgroups would not fit in a compute
    // unit's LDS: 3000 tokens, 6 heads of 64, 74 us, with 32 69.  Rows without padding where 160 KB are too few otherwise.)
    constexpr int NW = DV / 16, NT = DV * 4, GI = NW / NB, CW = sizeof(E) == 4 && DV == 64 ? 32 : 64, DT = CW / 16 / GI;
    constexpr int LT = C + kPad<E>, LS = CW + (sizeof(E) == 4 && DK + DV == 256 ? 0 : kPad<E>);
    constexpr bool SHARED = 2 * DV * LS <= kScores<E>;          // (the states' operands fit where P's transpose and then T were)
    __shared__ __align__(16) E sQ[C * LK], sK[C * LK], sV[C * LV], sO[C * LV], sU[C * LV], sT[kScores<E>], sS[SHARED ? 8 : 2 * DV * LS];
    __shared__ ChunkSteps<C> st;
    __shared__ float s_db[NW][C], s_db2[GI][C], s_near[GI][C], s_far[GI][C], s_pairs[NB][C], s_ss[NW];
    E *const sS0 = SHARED ? sT : sS, *const sdS = sS0 + DV * LS;
    const int tid0 = threadIdx.x, lane0 = tid0 & 63, w = __builtin_amdgcn_readfirstlane(tid0 >> 6), tw = w % NB, gi = w / NB;
    const int place = blockIdx.x / a.Hk, hk = blockIdx.x - place * a.Hk, share = RUN ? 1 : a.H / a.Hk;
    if (place >= a.places) {
        const int b = blockIdx.x - a.places * a.Hk;
        clear_rows(a.rows, b, (E*)a.dQ, a.Hk * DK);
        clear_rows(a.rows, b, (E*)a.dK, a.Hk * DK);
        clear_rows(a.rows, b, (E*)a.dV, a.H * DV);
        clear_rows(a.rows, b, (E*)a.dg, a.H);
        clear_rows(a.rows, b, (E*)a.dbeta, a.H);
        return;
    }
    const Chunk run = chunk_at(a.rows, C * a.run, place, lane0);
    if (run.n <= 0) return;
    const int chunk0 = chunk_place(a.rows, C, run, a.run, 0), n_chunks = RUN ? (run.n + C - 1) / C : 1;
    Chunk ch = run;
    // What the next head needs, or (NEXT) the next chunk, on its way during this one, where there are registers for it: 12 heads of 64, 16 sequences of
    // 2048 tokens, the gradient 332 us without, 324 with; 16 heads of 64 and 128, 8 of 2048, 415 and 422; of 128 and 128, 1083 and 1105.
    constexpr bool AHEAD = DV == 128, NEXT = RUN && DK + DV == 128 && DK == CW;
    Tile<E, C, DV, NT> tv, to;
    PackedT<E, C, NT> tt;
    Steps ts;
    Op<E, 1> so[KS], bo[KS];                                    // the states' operands, of the wave's value columns
    auto fetch = [&](int h, int chunk, int row, int n, int tid, int lane) {
        const size_t at = (size_t)chunk * a.H + h;
        ts = fetch_steps((const E*)a.g, a.ldg, (const E*)a.beta, a.ldb, row, h, n, lane);
        tv.fetch((const E*)a.V + h * DV, a.ldv, row, n, tid);
        to.fetch((const E*)a.dO + h * DV, a.lddo, row, n, tid);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            so[ks] = load_op<E, 1>((const E*)a.S0c + at * (DK * DV) + (w * KS + ks) * 512, lane);
            if (!RUN) bo[ks] = load_op<E, 1>((const E*)a.dS + at * (DK * DV) + (w * KS + ks) * 512, lane);
        }
    };
    f32x4 B[RUN ? DK / 16 : 1];
    if (RUN) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            bo[ks] = load_op<E, 1>((const E*)a.dS + ((size_t)place * a.H + hk) * (DK * DV) + (w * KS + ks) * 512, lane0);
            f32x8 v;
            if constexpr (sizeof(E) == 4) v = bo[ks].v;
            else v = __builtin_convertvector(bo[ks].h, f32x8);
            B[2 * ks] = __builtin_shufflevector(v, v, 0, 1, 2, 3);
            B[2 * ks + 1] = __builtin_shufflevector(v, v, 4, 5, 6, 7);
        }
    }
    for (int rc = n_chunks - 1; rc >= 0; --rc) {
    if (RUN) {
        if (rc < n_chunks - 1) __syncthreads();
        ch.row = run.row + rc * C;
        ch.n = min(C, run.n - rc * C);
    }
    {
        Tile<E, C, DK, NT> ty, tk;
        ty.fetch((const E*)a.Q + hk * DK, a.ldq, ch.row, ch.n, tid0);
        tk.fetch((const E*)a.K + hk * DK, a.ldk, ch.row, ch.n, tid0);
        if (AHEAD) fetch(hk * share, chunk0 + rc, ch.row, ch.n, tid0, lane0);
        ty.put(sQ, LK, ch.n, tid0);
        tk.put(sK, LK, ch.n, tid0);
    }
    const Planes<E, 2> Tm{sT, LT, C * LT};
    const Planes<E, 1> Um{sU, LV, 0}, Rm{sV, LV, 0};
    f32x4 sumQ[DK / CW * DT], sumK[DK / CW * DT];
#pragma unroll
    for (int d = 0; d < DK / CW * DT; ++d) sumQ[d] = sumK[d] = zero4();
    for (int hh = 0; hh < share; ++hh) {
        const int h = hk * share + hh;
        int lane = lane0;
        asm volatile("" : "+v"(lane));             // (addresses are worked out where they are used: kept over the heads, they fill the registers)
        const int tid = 64 * w + lane, q = lane >> 4, c = lane & 15, t = 16 * tw + c;
        if (NEXT ? rc == n_chunks - 1 : !AHEAD) fetch(h, chunk0 + rc, ch.row, ch.n, tid, lane);
        if (hh > 0) __syncthreads();
        put_steps(st, ts, ch.n, tid);
        tv.put(sV, LV, ch.n, tid);
        to.put(sO, LV, ch.n, tid);
        tt.fetch((const E*)a.T + ((size_t)(chunk0 + rc) * a.H + h) * (C * C), tid);
        __syncthreads();
        // P's transpose, sixteen of its rows to a wave
        for (int tb = (tw & ~1) + gi; tb < NB; tb += GI) {
            f32x4 x = zero4();
            if (tb >= tw) {
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) x = mma(rows_op(sQ, LK, 16 * tb, 32 * ks, lane), rows_op(sK, LK, 16 * tw, 32 * ks, lane), x);
                x *= splat4(a.scale) * st.decays_to(16 * tb + 4 * q, t);
                if (tb == tw)
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[i] = c <= 4 * q + i ? x[i] : 0.f;
            }
            Tm.put4(t, 16 * tb, q, x);
        }
        // U and dR, sixteen value columns to a wave
        float ss = 0.f;
        f32x4 x[NB], y[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) x[b] = y[b] = zero4();
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            f32x8 sf, df;
            if constexpr (sizeof(E) == 4) { sf = so[ks].v; df = bo[ks].v; }
            else { sf = __builtin_convertvector(so[ks].h, f32x8); df = __builtin_convertvector(bo[ks].h, f32x8); }
#pragma unroll
            for (int j = 0; j < 8; ++j) ss = fmaf(sf[j], df[j], ss);
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const Op<E, 1> k = rows_op(sK, LK, 16 * b, 32 * ks, lane);
                x[b] = mma(k, so[ks], x[b]);
                y[b] = mma(k, bo[ks], y[b]);
            }
        }
        Op<E, 2> ro[KC];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            x[b] = x[b] * *(const f32x4*)(st.bu + 16 * b + 4 * q) + *(const f32x4*)(st.beta + 16 * b + 4 * q) * tile_of(sV, LV, 16 * b, 16 * w, lane);
            y[b] *= *(const f32x4*)(st.down + 16 * b + 4 * q);
        }
#pragma unroll
        for (int d = 1; d < 64; d *= 2) ss += __shfl_xor(ss, d);
        if (lane == 0) s_ss[w] = ss;
        __syncthreads();                                               // (P is there)
#pragma unroll
        for (int ks = 0; ks < KC; ++ks) {
            const Op<E, 1> o = cols_op(sO, LV, 32 * ks, 16 * w, lane);
#pragma unroll
            for (int b = 0; b <= 2 * ks + 1; ++b) y[b] = mma(Tm.rows(16 * b, 32 * ks, lane), o, y[b]);
        }
        __syncthreads();
        tt.put(Tm, tid);
        __syncthreads();
#pragma unroll
        for (int ks = 0; ks < KC; ++ks) ro[ks] = operand<E, 2>(x[2 * ks], x[2 * ks + 1]);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            f32x4 u = zero4();
#pragma unroll
            for (int ks = 0; ks <= b / 2; ++ks) u = mma(ro[ks], Tm.rows(16 * b, 32 * ks, lane), u);
            Um.put4(16 * b + c, 16 * w, q, u);
        }
#pragma unroll
        for (int ks = 0; ks < KC; ++ks) ro[ks] = operand<E, 2>(y[2 * ks], y[2 * ks + 1]);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const int r0 = 16 * b + c;
            f32x4 r = zero4();
#pragma unroll
            for (int ks = b / 2; ks < KC; ++ks) r = mma(ro[ks], Tm.cols(32 * ks, 16 * b, lane), r);
            const float db = column_sum(dot4(r, wide4(sV + r0 * LV + four_of<E>(16 * w, q))));
            if (q == 0) s_db[w][r0] = db;
            Rm.put4(r0, 16 * w, q, r);                            // (dR where the value was: no other lane reads that one)
            if (r0 < ch.n)
                *(Vec4<E>*)((E*)a.dV + (size_t)(ch.row + r0) * (a.H * DV) + h * DV + 16 * w + 4 * q) =
                    __builtin_convertvector(r * splat4(st.beta[r0]), Vec4<E>);
        }
        __syncthreads();
        // S and dS_next so that their rows are summed over, CW columns of them; what the next head needs is on its way
        auto put = [&](int half) {
#pragma unroll
            for (int i = 0; i < CW / 32; ++i) {
                E *const p = sS0 + (16 * w + c) * LS + 32 * i, *const r = sdS + (16 * w + c) * LS + 32 * i;
                if constexpr (sizeof(E) == 4) {
                    const f32x8 s = so[CW / 32 * half + i].v, b = bo[CW / 32 * half + i].v;
                    *(f32x4*)(p + 4 * q) = __builtin_shufflevector(s, s, 0, 1, 2, 3);
                    *(f32x4*)(p + 16 + 4 * q) = __builtin_shufflevector(s, s, 4, 5, 6, 7);
                    *(f32x4*)(r + 4 * q) = __builtin_shufflevector(b, b, 0, 1, 2, 3);
                    *(f32x4*)(r + 16 + 4 * q) = __builtin_shufflevector(b, b, 4, 5, 6, 7);
                } else {
                    *(bf16x8*)(p + 8 * q) = so[CW / 32 * half + i].h;
                    *(bf16x8*)(r + 8 * q) = bo[CW / 32 * half + i].h;
                }
            }
        };
        put(0);
        if (AHEAD && DK == CW && hh + 1 < share) fetch(h + 1, chunk0, ch.row, ch.n, tid, lane);
        if (NEXT && rc > 0) fetch(h, chunk0 + rc - 1, ch.row - C, C, tid, lane);
        // X and beta Y of the wave's tokens as queries, then as keys
        float dbeta = 0.f, near = 0.f, far = 0.f;
        Op<E, 1> xq[KC], yq[KC], xk[KC], yk[KC];
        {
            Op<E, 1> o[VS], r[VS], u[VS];
#pragma unroll
            for (int ks = 0; ks < VS; ++ks) {
                o[ks] = rows_op(sO, LV, 16 * tw, 32 * ks, lane);
                r[ks] = rows_op(sV, LV, 16 * tw, 32 * ks, lane);
            }
            f32x4 rest = zero4();                                      // of W, the sums over the keys of the blocks in front, u down the rows, in all columns
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                x[b] = y[b] = zero4();
                read_afresh();
                if (b <= tw) {                                         // keys b
                    f32x4 g = zero4();
#pragma unroll
                    for (int ks = 0; ks < VS; ++ks) {
                        const Op<E, 1> m = rows_op(sU, LV, 16 * b, 32 * ks, lane);
                        x[b] = mma(m, o[ks], x[b]);
                        y[b] = mma(m, r[ks], y[b]);
                    }
                    if (gi == 0)
#pragma unroll
                        for (int ks = 0; ks < KS; ++ks) g = mma(rows_op(sK, LK, 16 * b, 32 * ks, lane), rows_op(sK, LK, 16 * tw, 32 * ks, lane), g);
                    const f32x4 d = st.decays_from(t, 16 * b + 4 * q);
                    x[b] *= splat4(a.scale) * d;
                    y[b] *= d;
                    if (b == tw)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            x[b][i] = 4 * q + i <= c ? x[b][i] : 0.f;
                            y[b][i] = 4 * q + i < c ? y[b][i] : 0.f;
                        }
                    dbeta -= dot4(y[b], g);
                    y[b] *= splat4(st.beta[t]);
                    if (gi == 0 && a.g != nullptr) {
                        f32x4 p = zero4();
#pragma unroll
                        for (int ks = 0; ks < KS; ++ks) p = mma(rows_op(sK, LK, 16 * b, 32 * ks, lane), rows_op(sQ, LK, 16 * tw, 32 * ks, lane), p);
                        // sum of W_us over s < t for the t of the keys' block, by a product with ones below the diagonal; then over the wave's u, u >= t
                        const f32x4 W = x[b] * p - y[b] * g;
                        f32x4 v = rest;
#pragma unroll
                        for (int j = 0; j < 4; ++j) v = __builtin_amdgcn_mfma_f32_16x16x4f32(W[j], 4 * q + j < c ? 1.f : 0.f, v, 0, 0, 0);
                        if (b == tw)
#pragma unroll
                            for (int i = 0; i < 4; ++i) v[i] = 4 * q + i >= c ? v[i] : 0.f;
                        else
#pragma unroll
                            for (int j = 0; j < 4; ++j) rest = __builtin_amdgcn_mfma_f32_16x16x4f32(W[j], 1.f, rest, 0, 0, 0);
                        const float sum = column_sum((v[0] + v[1]) + (v[2] + v[3]));
                        if (q == 0) s_pairs[tw][16 * b + c] = sum;
                    }
                }
            }
#pragma unroll
            for (int ks = 0; ks < KC; ++ks) {
                xq[ks] = operand<E, 1>(x[2 * ks], x[2 * ks + 1]);
                yq[ks] = operand<E, 1>(y[2 * ks], y[2 * ks + 1]);
            }
#pragma unroll
            for (int ks = 0; ks < VS; ++ks) u[ks] = rows_op(sU, LV, 16 * tw, 32 * ks, lane);
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                x[b] = y[b] = zero4();
                read_afresh();
                if (b >= tw) {                                         // queries b
#pragma unroll
                    for (int ks = 0; ks < VS; ++ks) {
                        x[b] = mma(rows_op(sO, LV, 16 * b, 32 * ks, lane), u[ks], x[b]);
                        y[b] = mma(rows_op(sV, LV, 16 * b, 32 * ks, lane), u[ks], y[b]);
                    }
                    const f32x4 d = st.decays_to(16 * b + 4 * q, t);
                    x[b] *= splat4(a.scale) * d;
                    y[b] *= d;
                    if (b == tw)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            x[b][i] = c <= 4 * q + i ? x[b][i] : 0.f;
                            y[b][i] = c < 4 * q + i ? y[b][i] : 0.f;
                        }
                    y[b] *= *(const f32x4*)(st.beta + 16 * b + 4 * q);
                }
            }
#pragma unroll
            for (int ks = 0; ks < KC; ++ks) {
                xk[ks] = operand<E, 1>(x[2 * ks], x[2 * ks + 1]);
                yk[ks] = operand<E, 1>(y[2 * ks], y[2 * ks + 1]);
            }
        }
        // the gradients of queries and keys
#pragma unroll
        for (int half = 0; half < DK / CW; ++half) {
            if (half > 0) {
                __syncthreads();
                put(half);
                if (AHEAD && half + 1 == DK / CW && hh + 1 < share) fetch(h + 1, chunk0, ch.row, ch.n, tid, lane);
            }
            __syncthreads();
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                const int n = DT * gi + d, col = CW * half + 16 * n;
                read_afresh();
                f32x4 xx = zero4(), yy = zero4(), zz = zero4();
#pragma unroll
                for (int ks = 0; ks < VS; ++ks) {
                    const Op<E, 1> s = cols_op(sS0, LS, 32 * ks, 16 * n, lane);
                    xx = mma(s, rows_op(sO, LV, 16 * tw, 32 * ks, lane), xx);
                    yy = mma(s, rows_op(sV, LV, 16 * tw, 32 * ks, lane), yy);
                    zz = mma(cols_op(sdS, LS, 32 * ks, 16 * n, lane), rows_op(sU, LV, 16 * tw, 32 * ks, lane), zz);
                }
                const f32x4 k4 = wide4(sK + t * LK + four_of<E>(col, q)), q4 = wide4(sQ + t * LK + four_of<E>(col, q));
                xx *= splat4(a.scale * st.up[t]);
                yy *= splat4(st.up[t]);
                zz *= splat4(st.down[t]);
                const float read = dot4(yy, k4);
                dbeta -= read;
                near += fmaf(-st.beta[t], read, dot4(xx, q4));
                far += dot4(zz, k4);
                yy *= splat4(st.beta[t]);
                f32x4 vv = zero4();
#pragma unroll
                for (int ks = 0; ks < KC; ++ks) {
                    const Op<E, 1> k = cols_op(sK, LK, 32 * ks, col, lane);
                    if (ks <= tw / 2) {
                        xx = mma(k, xq[ks], xx);
                        yy = mma(k, yq[ks], yy);
                    }
                    if (ks >= tw / 2) {
                        zz = mma(cols_op(sQ, LK, 32 * ks, col, lane), xk[ks], zz);
                        vv = mma(k, yk[ks], vv);
                    }
                }
                zz -= vv;
                sumQ[DT * half + d] += xx;
                sumK[DT * half + d] += zz - yy;
            }
        }
        dbeta = column_sum(dbeta);
        near = column_sum(near);
        far = column_sum(far);
        if (q == 0) {
            s_db2[gi][t] = dbeta;
            s_near[gi][t] = near;
            s_far[gi][t] = far;
        }
        __syncthreads();
        if (tid < 64) {
            float b = 0.f, behind = 0.f, front = 0.f, pairs = 0.f, ends = 0.f;
            if (tid < C) {
#pragma unroll
                for (int i = 0; i < GI; ++i) { b += s_db2[i][tid]; behind += s_near[i][tid]; front += s_far[i][tid]; }
#pragma unroll
                for (int i = 0; i < NB; ++i) pairs += i >= tid / 16 ? s_pairs[i][tid] : 0.f;
#pragma unroll
                for (int i = 0; i < NW; ++i) b += s_db[i][tid];
                if (tid < ch.n) ((E*)a.dbeta)[(size_t)(ch.row + tid) * a.H + h] = from_f<E>(b);
            }
#pragma unroll
            for (int i = 0; i < NW; ++i) ends += s_ss[i];
            front = __shfl_up(front, 1);                                 // (of the tokens in front, t itself not among them)
            if (tid == 0) front = 0.f;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const float x = __shfl_down(behind, d), y1 = __shfl_up(front, d);
                if (tid + d < 64) behind += x;
                if (tid >= d) front += y1;
            }
            if (a.g != nullptr && tid < ch.n) ((E*)a.dg)[(size_t)(ch.row + tid) * a.H + h] = from_f<E>(st.whole * ends + behind + front + pairs);
        }
    }
    if (RUN && rc > 0) {
        // the gradient of the state in front: dS <- e^gamma dS + scale (e^gamma Q)^T dO - (beta e^gamma K)^T dR
        int lane = lane0;
        asm volatile("" : "+v"(lane));
        Op<E, 2> qo[KC], ro[KC];
#pragma unroll
        for (int ks = 0; ks < KC; ++ks) {
            qo[ks] = scaled<E, 2>(cols_op(sO, LV, 32 * ks, 16 * w, lane), st.up, 32 * ks, lane, a.scale);
            ro[ks] = scaled<E, 2>(cols_op(sV, LV, 32 * ks, 16 * w, lane), st.bu, 32 * ks, lane);
        }
#pragma unroll
        for (int d = 0; d < DK / 16; ++d) {
            if (d % 2 == 0) read_afresh();
            B[d] *= splat4(st.whole);
#pragma unroll
            for (int ks = 0; ks < KC; ++ks) {
                B[d] = mma(cols_op(sQ, LK, 32 * ks, 16 * d, lane), qo[ks], B[d]);
                B[d] = mma(cols_op(sK, LK, 32 * ks, 16 * d, lane), ro[ks], B[d]);
            }
        }
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) bo[ks] = operand<E, 1>(B[2 * ks], B[2 * ks + 1]);
    }
    const int q = lane0 >> 4, t = 16 * tw + (lane0 & 15);
    if (t < ch.n) {
        E* dq = (E*)a.dQ + (size_t)(ch.row + t) * (a.Hk * DK) + hk * DK + 4 * q;
        E* dk = (E*)a.dK + (size_t)(ch.row + t) * (a.Hk * DK) + hk * DK + 4 * q;
#pragma unroll
        for (int i = 0; i < DK / CW * DT; ++i) {
            const int col = CW * (i / DT) + 16 * (DT * gi + i % DT);
            *(Vec4<E>*)(dq + col) = __builtin_convertvector(sumQ[i], Vec4<E>);
            *(Vec4<E>*)(dk + col) = __builtin_convertvector(sumK[i], Vec4<E>);
        }
    }
    }
}

// -------------------------------------------------------------------------------------------------------------------- host
hipError_t launch_delta_bwd(DeltaArgs a, const DeltaPlan& p, char* ws, char* saved, bool has_saved, int dk, int dv, int dtype, hipStream_t st)
{
    ProfScope prof(KID_DELTA_BWD, st);
    hipError_t e = hipSuccess;
    if (!has_saved) saved = ws + p.saved_at;
    a.N = ws + p.N;
    a.Z = (float*)(ws + p.Z);
    a.whole = (float*)(ws + p.whole);
    a.T = saved + p.T;
    a.S0 = a.S0c = saved + p.S0c;
    if (!has_saved) {
        a.places = p.chunks;
        a.run = 1;
        if ((e = launch_delta_states(a, p, dk, dv, dtype, st)) != hipSuccess) return e;
    }
    a.places = p.places;
    a.run = p.run;
    a.dS = ws + p.dS;
    if (p.places > 0) {
        const dim3 grid((unsigned)((size_t)p.places * a.H));
#define CHELA_RUN(E, DK, DV)                                                                                          \
    do {                                                                                                              \
        constexpr int P2 = sizeof(E) == 2 ? 2 : 1;                                                                    \
        const dim3 threads(p.run > 1 ? (DK + DV) * 2 : 256);                                                          \
        if (p.run > 1 && p.parts == 2) hipLaunchKernelGGL((delta_bwd_prep_run_kernel<E, DK, DV, P2>), grid, threads, 0, st, a); \
        else if (p.run > 1) hipLaunchKernelGGL((delta_bwd_prep_run_kernel<E, DK, DV, 1>), grid, threads, 0, st, a);    \
        else if (p.parts == 2) hipLaunchKernelGGL((delta_bwd_prep_kernel<E, DK, DV, P2>), grid, threads, 0, st, a);    \
        else hipLaunchKernelGGL((delta_bwd_prep_kernel<E, DK, DV, 1>), grid, threads, 0, st, a);                      \
    } while (0)
        CHELA_DELTA(CHELA_RUN)
#undef CHELA_RUN
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if ((e = launch_delta_walk(a, true, p.parts, dk, dv, dtype, st)) != hipSuccess) return e;
    const bool clear = a.rows.clear && a.rows.cu != nullptr;
    const size_t blocks = (size_t)p.places * a.Hk + (clear ? (a.rows.T + 63) / 64 : 0);
    if (blocks == 0) return hipSuccess;
    const dim3 grid((unsigned)blocks);
#define CHELA_RUN(E, DK, DV)                                                                                          \
    do {                                                                                                              \
        if (p.run > 1) hipLaunchKernelGGL((delta_grad_kernel<E, DK, DV, true>), grid, dim3(DV * 4), 0, st, a);        \
        else hipLaunchKernelGGL((delta_grad_kernel<E, DK, DV, false>), grid, dim3(DV * 4), 0, st, a);                 \
    } while (0)
    CHELA_DELTA(CHELA_RUN)
#undef CHELA_RUN
    return hipGetLastError();
}

}  // namespace chela
