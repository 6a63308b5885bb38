// Gated delta rule, gradient, gfx950.  Names as in the forward's file; S is the state in front of a chunk, dS_next the gradient of the one behind.
//
//     dU = P^T dO + K~ dS_next,   dR = T^T dU,   dV = beta dR,
//     X = scale D o (dO U^T) for s <= t,   Y = D o (dR U^T) for s < t,
//     dQ = scale e^gamma dO S^T + X K,   read = -beta (e^gamma dR S^T + Y K),   carry = e^(gamma_C - gamma) U dS_next^T,
//     write = carry + X^T Q - (beta Y)^T K,   dK = read + write,
//     dbeta_t = dR_t . v_t - k_t . (e^gamma_t S dR_t) - sum_s Y_ts k_t . k_s,
//     dgamma_t = q_t . dQ_t + k_t . read_t - k_t . write_t, at the chunk's last token + e^gamma_C <S, dS_next> + sum_s k_s . carry_s,
//     dg_t = sum of dgamma from t to the chunk's end   (every pair of tokens on one side of t cancels: both take it from the same X, Y),
//     dS = e^gamma_C dS_next - N^T dS_next + Z',   Z' = scale (e^gamma Q)^T dO - (beta e^gamma K)^T T^T P^T dO.
// Three launches, as forward: N^T and Z' of all chunks, the walk from the last chunk to the first, all gradients.
#include "chela_delta.h"

namespace chela {

template <typename E, int DK, int DV, int P>
__global__ __launch_bounds__(256, 2) void delta_bwd_prep_kernel(DeltaArgs a)
{
    constexpr int C = DeltaChunk<E>::C, NB = C / 16, KC = C / 32, KS = DK / 32, LK = DK + kPad<E>, LV = DV + kPad<E>, LT = C + kPad<E>;
    __shared__ __align__(16) E sQ[C * LK], sK[C * LK], sO[C * LV], sT[P * C * LT], sP[P * C * LT];
    __shared__ __align__(16) float s_inv[P == 2 ? C * (C + 4) + C * 20 : 1];
    __shared__ ChunkSteps<C> st;
    __shared__ __align__(16) float s_qu[C];                        // scale e^gamma
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, q = lane >> 4, c = lane & 15;
    const int place = blockIdx.x / a.H, h = blockIdx.x - place * a.H, hk = h / (a.H / a.Hk);
    const Chunk ch = chunk_at(a.rows, C, place, lane);
    if (ch.n <= 0) return;
    const size_t at = (size_t)place * a.H + h;
    {
        Tile<E, C, DK> y, k;
        Tile<E, C, DV> o;
        Tile<E, C, C> m;
        const Steps s = fetch_steps((const E*)a.g, a.ldg, (const E*)a.beta, a.ldb, ch.row, h, ch.n, lane);
        y.fetch((const E*)a.Q + hk * DK, a.ldq, ch.row, ch.n, tid);
        k.fetch((const E*)a.K + hk * DK, a.ldk, ch.row, ch.n, tid);
        o.fetch((const E*)a.dO + h * DV, a.lddo, ch.row, ch.n, tid);
        if (P == 1) m.fetch((const E*)a.T + at * (C * C), C, 0, C, tid);
        put_steps(st, s, ch.n, tid);
        y.put(sQ, LK, ch.n, tid);
        k.put(sK, LK, ch.n, tid);
        o.put(sO, LV, ch.n, tid);
        if (P == 1) m.put(sT, LT, C, tid);
    }
    __syncthreads();
    const Planes<E, P> T{sT, LT, C * LT}, Pt{sP, LT, C * LT};
    if (P == 2) chunk_inverse<E, DK>(sK, LK, st, s_inv, s_inv + C * (C + 4), T, tid);       // (what was kept of it has one part)
    if (w < NB) {                                                  // P's transpose, sixteen of its rows to a wave
        const int s = 16 * w + c;
        for (int tb = w & ~1; tb < NB; ++tb) {
            f32x4 x = zero4();
            if (tb >= w) {
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) x = mma(rows_op(sQ, LK, 16 * tb, 32 * ks, lane), rows_op(sK, LK, 16 * w, 32 * ks, lane), x);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int t = 16 * tb + 4 * q + i;
                    x[i] = s <= t ? a.scale * st.decay(t, s) * x[i] : 0.f;
                }
            }
            Pt.put4(s, 16 * tb + 4 * q, x);
        }
    }
    if (tid < C) s_qu[tid] = a.scale * st.up[tid];
    __syncthreads();
#pragma unroll 1
    for (int p = w; p < (DK + DV) / 16; p += 4) {
        read_afresh();
        f32x4 x[NB];
        Op<E, 2> xo[KC];
        if (p < DV / 16) {
            Op<E, 2> qo[KC];
#pragma unroll
            for (int b = 0; b < NB; ++b) x[b] = zero4();
#pragma unroll
            for (int ks = 0; ks < KC; ++ks) {
                const Op<E, 1> o = cols_op(sO, LV, 32 * ks, 16 * p, lane);
                qo[ks] = scaled<E, 2>(o, s_qu, 32 * ks, lane);
#pragma unroll
                for (int b = 0; b <= 2 * ks + 1; ++b) x[b] = mma(Pt.rows(16 * b, 32 * ks, lane), o, x[b]);
            }
#pragma unroll
            for (int ks = 0; ks < KC; ++ks) xo[ks] = operand<E, 2>(x[2 * ks], x[2 * ks + 1]);
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

__device__ __forceinline__ float dot4(f32x4 a, f32x4 b) { return fmaf(a[0], b[0], fmaf(a[1], b[1], fmaf(a[2], b[2], a[3] * b[3]))); }
template <typename E> __device__ __forceinline__ f32x4 wide4(const E* p) { return __builtin_convertvector(*(const Vec4<E>*)p, f32x4); }
// over the four lanes that have a column of a tile
__device__ __forceinline__ float column_sum(float x)
{
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}
// A workgroup has a chunk and a key head, and goes over that one's value heads: the sums of dQ and dK over them stay in registers.
template <typename E, int DK, int DV>
__global__ __launch_bounds__(256, DK + DV == 128 ? 2 : 1) void delta_grad_kernel(DeltaArgs a)
{
    constexpr int C = DeltaChunk<E>::C, NB = C / 16, KC = C / 32, KS = DK / 32, VS = DV / 32, LK = DK + kPad<E>, LV = DV + kPad<E>;
    constexpr int LT = C + kPad<E>, LS = 64 + kPad<E>;
    __shared__ __align__(16) E sQ[C * LK], sK[C * LK], sV[C * LV], sO[C * LV], sU[C * LV], sT[C * LT], sP[C * LT], sS[DV * LS];
    __shared__ ChunkSteps<C> st;
    __shared__ float s_db[4][C], s_dg[C], s_kc[4], s_ss[4];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, q = lane >> 4, c = lane & 15;
    const int place = blockIdx.x / a.Hk, hk = blockIdx.x - place * a.Hk, share = a.H / a.Hk;
    if (place >= a.places) {
        const int b = blockIdx.x - a.places * a.Hk;
        clear_rows(a.rows, b, (E*)a.dQ, a.Hk * DK);
        clear_rows(a.rows, b, (E*)a.dK, a.Hk * DK);
        clear_rows(a.rows, b, (E*)a.dV, a.H * DV);
        clear_rows(a.rows, b, (E*)a.dg, a.H);
        clear_rows(a.rows, b, (E*)a.dbeta, a.H);
        return;
    }
    const Chunk ch = chunk_at(a.rows, C, place, lane);
    if (ch.n <= 0) return;
    Tile<E, C, DK> ty, tk;
    ty.fetch((const E*)a.Q + hk * DK, a.ldq, ch.row, ch.n, tid);
    tk.fetch((const E*)a.K + hk * DK, a.ldk, ch.row, ch.n, tid);
    const Planes<E, 1> Pm{sP, LT, 0}, Tm{sT, LT, 0}, Um{sU, LV, 0}, Rm{sV, LV, 0};
    f32x4 sumQ[DK / 16], sumK[DK / 16];
#pragma unroll
    for (int d = 0; d < DK / 16; ++d) sumQ[d] = sumK[d] = zero4();
    for (int hh = 0; hh < share; ++hh) {
        const int h = hk * share + hh;
        const size_t at = (size_t)place * a.H + h;
        const E *S0 = (const E*)a.S0 + at * (DK * DV), *dS = (const E*)a.dS + at * (DK * DV);
        Op<E, 1> so[KS], bo[KS];                                       // the states' operands, of the wave's next columns
        auto next = [&](int eg) {
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                so[ks] = load_op<E, 1>(S0 + (eg * KS + ks) * 512, lane);
                bo[ks] = load_op<E, 1>(dS + (eg * KS + ks) * 512, lane);
            }
        };
        {
            Tile<E, C, DV> v, o;
            Tile<E, C, C> m;
            const Steps s = fetch_steps((const E*)a.g, a.ldg, (const E*)a.beta, a.ldb, ch.row, h, ch.n, lane);
            v.fetch((const E*)a.V + h * DV, a.ldv, ch.row, ch.n, tid);
            o.fetch((const E*)a.dO + h * DV, a.lddo, ch.row, ch.n, tid);
            m.fetch((const E*)a.T + at * (C * C), C, 0, C, tid);
            next(w);
            if (hh > 0) __syncthreads();
            put_steps(st, s, ch.n, tid);
            if (hh == 0) {
                ty.put(sQ, LK, ch.n, tid);
                tk.put(sK, LK, ch.n, tid);
            }
            v.put(sV, LV, ch.n, tid);
            o.put(sO, LV, ch.n, tid);
            m.put(sT, LT, C, tid);
        }
        __syncthreads();
        if (w < NB) {                                                  // P's transpose
            const int s = 16 * w + c;
            for (int tb = w & ~1; tb < NB; ++tb) {
                f32x4 x = zero4();
                if (tb >= w) {
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) x = mma(rows_op(sQ, LK, 16 * tb, 32 * ks, lane), rows_op(sK, LK, 16 * w, 32 * ks, lane), x);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int t = 16 * tb + 4 * q + i;
                        x[i] = s <= t ? a.scale * st.decay(t, s) * x[i] : 0.f;
                    }
                }
                Pm.put4(s, 16 * tb + 4 * q, x);
            }
        }
        __syncthreads();
        // U and dR, sixteen value columns at a time
        float db[NB], ss = 0.f;
#pragma unroll
        for (int b = 0; b < NB; ++b) db[b] = 0.f;
#pragma unroll 1
        for (int eg = w; eg < DV / 16; eg += 4) {
            read_afresh();
            Op<E, 2> ro[KC];
            f32x4 x[NB], y[NB];
#pragma unroll
            for (int b = 0; b < NB; ++b) x[b] = y[b] = zero4();
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const Op<E, 1> s = so[ks], d = bo[ks];
                f32x8 sf, df;
                if constexpr (sizeof(E) == 4) { sf = s.v; df = d.v; }
                else { sf = __builtin_convertvector(s.h, f32x8); df = __builtin_convertvector(d.h, f32x8); }
#pragma unroll
                for (int j = 0; j < 8; ++j) ss = fmaf(sf[j], df[j], ss);
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    const Op<E, 1> k = rows_op(sK, LK, 16 * b, 32 * ks, lane);
                    x[b] = mma(k, s, x[b]);
                    y[b] = mma(k, d, y[b]);
                }
            }
#pragma unroll
            for (int b = 0; b < NB; ++b) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int t = 16 * b + 4 * q + i;
                    x[b][i] = st.beta[t] * fmaf(-st.up[t], x[b][i], to_f(sV[t * LV + 16 * eg + c]));
                }
                y[b] *= *(const f32x4*)(st.down + 16 * b + 4 * q);
            }
#pragma unroll
            for (int ks = 0; ks < KC; ++ks) ro[ks] = operand<E, 2>(x[2 * ks], x[2 * ks + 1]);
            if (eg + 4 < DV / 16) next(eg + 4);
            read_afresh();
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                f32x4 u = zero4();
#pragma unroll
                for (int ks = 0; ks <= b / 2; ++ks) u = mma(ro[ks], Tm.rows(16 * b, 32 * ks, lane), u);
                Um.put4(16 * b + c, 16 * eg + 4 * q, u);
            }
            read_afresh();
#pragma unroll
            for (int ks = 0; ks < KC; ++ks) {
                const Op<E, 1> o = cols_op(sO, LV, 32 * ks, 16 * eg, lane);
#pragma unroll
                for (int b = 0; b <= 2 * ks + 1; ++b) y[b] = mma(Pm.rows(16 * b, 32 * ks, lane), o, y[b]);
            }
#pragma unroll
            for (int ks = 0; ks < KC; ++ks) ro[ks] = operand<E, 2>(y[2 * ks], y[2 * ks + 1]);
            read_afresh();
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const int t = 16 * b + c;
                f32x4 r = zero4();
#pragma unroll
                for (int ks = b / 2; ks < KC; ++ks) r = mma(ro[ks], Tm.cols(32 * ks, 16 * b, lane), r);
                db[b] += dot4(r, wide4(sV + t * LV + 16 * eg + 4 * q));
                Rm.put4(t, 16 * eg + 4 * q, r);                       // (dR where the value was: no other lane reads that one)
                if (t < ch.n)
                    *(Vec4<E>*)((E*)a.dV + (size_t)(ch.row + t) * (a.H * DV) + h * DV + 16 * eg + 4 * q) =
                        __builtin_convertvector(r * splat4(st.beta[t]), Vec4<E>);
            }
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const float x = column_sum(db[b]);
            if (q == 0) s_db[w][16 * b + c] = x;
        }
#pragma unroll
        for (int d = 1; d < 64; d *= 2) ss += __shfl_xor(ss, d);
        if (lane == 0) s_ss[w] = ss;
        Op<E, 1> s0[DV / 32], s1[DV / 32];                             // S and dS_next, sixty-four of a row's columns, on their way to LDS
        auto fetch = [&](Op<E, 1>(&to)[DV / 32], const E* from, int half) {
#pragma unroll
            for (int i = 0; i < DV / 32; ++i) to[i] = load_op<E, 1>(from + (((w + 4 * i) >> 1) * KS + 2 * half + (w & 1)) * 512, lane);
        };
        auto put = [&](const Op<E, 1>(&x)[DV / 32]) {
#pragma unroll
            for (int i = 0; i < DV / 32; ++i) {
                E* to = sS + (16 * ((w + 4 * i) >> 1) + c) * LS + 32 * (w & 1) + 4 * q;
                if constexpr (sizeof(E) == 4) {
                    *(f32x4*)to = __builtin_shufflevector(x[i].v, x[i].v, 0, 1, 2, 3);
                    *(f32x4*)(to + 16) = __builtin_shufflevector(x[i].v, x[i].v, 4, 5, 6, 7);
                } else {
                    *(bf16x4*)to = __builtin_shufflevector(x[i].h, x[i].h, 0, 1, 2, 3);
                    *(bf16x4*)(to + 16) = __builtin_shufflevector(x[i].h, x[i].h, 4, 5, 6, 7);
                }
            }
        };
        fetch(s0, S0, 0);
        fetch(s1, dS, 0);
        __syncthreads();
        // X and beta Y, sixteen tokens to a wave
        const int t = 16 * w + c;
        float dbeta = 0.f, dgamma = 0.f, kc = 0.f;
        if (w < NB) {
            for (int sb = 0; sb <= (w | 1); ++sb) {
                f32x4 x = zero4(), y = zero4(), g = zero4();
                if (sb <= w) {
#pragma unroll
                    for (int ks = 0; ks < VS; ++ks) {
                        const Op<E, 1> u = rows_op(sU, LV, 16 * sb, 32 * ks, lane);
                        x = mma(u, rows_op(sO, LV, 16 * w, 32 * ks, lane), x);
                        y = mma(u, rows_op(sV, LV, 16 * w, 32 * ks, lane), y);
                    }
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) g = mma(rows_op(sK, LK, 16 * sb, 32 * ks, lane), rows_op(sK, LK, 16 * w, 32 * ks, lane), g);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int s = 16 * sb + 4 * q + i;
                        const float d = s <= t ? st.decay(t, s) : 0.f;
                        x[i] = s <= t ? a.scale * d * x[i] : 0.f;
                        y[i] = s < t ? d * y[i] : 0.f;
                        dbeta = s < t ? fmaf(-y[i], g[i], dbeta) : dbeta;
                    }
                }
                Pm.put4(t, 16 * sb + 4 * q, x);
                Tm.put4(t, 16 * sb + 4 * q, y * splat4(st.beta[t]));
            }
        }
        // the gradients of queries and keys, sixty-four columns at a time
#pragma unroll
        for (int half = 0; half < DK / 64; ++half) {
            f32x4 dq[4], rd[4];
            if (half > 0) __syncthreads();
            put(s0);
            __syncthreads();
            if (w < NB) {
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    read_afresh();
                    const int col = 64 * half + 16 * d;
                    f32x4 x = zero4(), y = zero4();
#pragma unroll
                    for (int ks = 0; ks < VS; ++ks) {
                        const Op<E, 1> s = cols_op(sS, LS, 32 * ks, 16 * d, lane);
                        x = mma(s, rows_op(sO, LV, 16 * w, 32 * ks, lane), x);
                        y = mma(s, rows_op(sV, LV, 16 * w, 32 * ks, lane), y);
                    }
                    x *= splat4(a.scale * st.up[t]);
                    y *= splat4(st.up[t]);
                    dbeta -= dot4(y, wide4(sK + t * LK + col + 4 * q));
                    y *= splat4(st.beta[t]);
                    for (int ks = 0; ks <= w / 2; ++ks) {
                        const Op<E, 1> k = cols_op(sK, LK, 32 * ks, col, lane);
                        x = mma(k, Pm.rows(16 * w, 32 * ks, lane), x);
                        y = mma(k, Tm.rows(16 * w, 32 * ks, lane), y);
                    }
                    dgamma += dot4(x, wide4(sQ + t * LK + col + 4 * q)) - dot4(y, wide4(sK + t * LK + col + 4 * q));
                    dq[d] = x;
                    rd[d] = y;
                }
            }
            __syncthreads();
            put(s1);
            if (half + 1 < DK / 64) {
                fetch(s0, S0, half + 1);
                fetch(s1, dS, half + 1);
            }
            __syncthreads();
            if (w < NB) {
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    read_afresh();
                    const int col = 64 * half + 16 * d;
                    f32x4 x = zero4(), y = zero4();
#pragma unroll
                    for (int ks = 0; ks < VS; ++ks) x = mma(cols_op(sS, LS, 32 * ks, 16 * d, lane), rows_op(sU, LV, 16 * w, 32 * ks, lane), x);
                    x *= splat4(st.down[t]);
                    const f32x4 k = wide4(sK + t * LK + col + 4 * q);
                    kc += dot4(x, k);
                    for (int ks = w / 2; ks < KC; ++ks) {
                        x = mma(cols_op(sQ, LK, 32 * ks, col, lane), Pm.cols(32 * ks, 16 * w, lane), x);
                        y = mma(cols_op(sK, LK, 32 * ks, col, lane), Tm.cols(32 * ks, 16 * w, lane), y);
                    }
                    x -= y;
                    dgamma -= dot4(x, k);
                    sumQ[4 * half + d] += dq[d];
                    sumK[4 * half + d] += x - rd[d];
                }
            }
        }
        if (w < NB) {
            dbeta = column_sum(dbeta);
            dgamma = column_sum(dgamma);
            if (q == 0) {
                if (t < ch.n)
                    ((E*)a.dbeta)[(size_t)(ch.row + t) * a.H + h] = from_f<E>(dbeta + ((s_db[0][t] + s_db[1][t]) + (s_db[2][t] + s_db[3][t])));
                s_dg[t] = dgamma;
            }
        }
#pragma unroll
        for (int d = 1; d < 64; d *= 2) kc += __shfl_xor(kc, d);
        if (lane == 0) s_kc[w] = kc;
        __syncthreads();
        if (a.g != nullptr && tid < 64) {
            float x = tid < C ? s_dg[tid] : 0.f;
            if (tid == C - 1) x += st.whole * ((s_ss[0] + s_ss[1]) + (s_ss[2] + s_ss[3])) + ((s_kc[0] + s_kc[1]) + (s_kc[2] + s_kc[3]));
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const float y = __shfl_down(x, d);
                if (tid + d < 64) x += y;
            }
            if (tid < ch.n) ((E*)a.dg)[(size_t)(ch.row + tid) * a.H + h] = from_f<E>(x);
        }
    }
    if (w < NB) {
        const int t = 16 * w + c;
        if (t < ch.n) {
            E* dq = (E*)a.dQ + (size_t)(ch.row + t) * (a.Hk * DK) + hk * DK + 4 * q;
            E* dk = (E*)a.dK + (size_t)(ch.row + t) * (a.Hk * DK) + hk * DK + 4 * q;
#pragma unroll
            for (int d = 0; d < DK / 16; ++d) {
                *(Vec4<E>*)(dq + 16 * d) = __builtin_convertvector(sumQ[d], Vec4<E>);
                *(Vec4<E>*)(dk + 16 * d) = __builtin_convertvector(sumK[d], Vec4<E>);
            }
        }
    }
}

// -------------------------------------------------------------------------------------------------------------------- host
hipError_t launch_delta_bwd(DeltaArgs a, const DeltaPlan& p, char* ws, char* saved, bool has_saved, int dk, int dv, int dtype, hipStream_t st)
{
    ProfScope prof(KID_DELTA_BWD, st);
    hipError_t e = hipSuccess;
    if (!has_saved) {
        if ((e = launch_delta_states(a, p, ws, nullptr, dk, dv, dtype, st)) != hipSuccess) return e;
    } else {
        a.places = p.places;
        a.N = ws + p.N;
        a.Z = (float*)(ws + p.Z);
        a.T = saved + p.T;
        a.S0 = saved + p.S0;
        a.whole = (float*)(saved + p.whole);
    }
    a.dS = ws + p.dS;
    if (p.places > 0) {
        const dim3 grid((unsigned)((size_t)p.places * a.H));
#define CHELA_RUN(E, DK, DV)                                                                                          \
    do {                                                                                                              \
        if (sizeof(E) == 2 && p.parts == 2) hipLaunchKernelGGL((delta_bwd_prep_kernel<E, DK, DV, 3 - sizeof(E) / 2>), grid, dim3(256), 0, st, a); \
        else hipLaunchKernelGGL((delta_bwd_prep_kernel<E, DK, DV, 1>), grid, dim3(256), 0, st, a);                    \
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
#define CHELA_RUN(E, DK, DV) hipLaunchKernelGGL((delta_grad_kernel<E, DK, DV>), grid, dim3(256), 0, st, a)
    CHELA_DELTA(CHELA_RUN)
#undef CHELA_RUN
    return hipGetLastError();
}

}  // namespace chela
