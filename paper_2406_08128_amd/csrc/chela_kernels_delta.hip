// Gated delta rule, forward and single tokens, gfx950.
//
// Per head, with a state S of dk x dv, alpha = e^g:
//     S' = alpha_t S_{t-1},   u_t = beta_t (v_t - S'^T k_t),   S_t = S' + k_t u_t^T,   o_t = scale S_t^T q_t.
// A chunk of C tokens at once, gamma the running sum of g in it, S the state in front of it, D_ts = e^(gamma_t - gamma_s):
//     (1 + A) U = beta (V - e^gamma K S),  A_ts = beta_t D_ts k_t . k_s for s < t, 0 otherwise;   T = (1 + A)^-1,
//     O = scale e^gamma Q S + P U,  P_ts = scale D_ts q_t . k_s for s <= t,
//     S_next = e^(gamma_C) S + K~^T U = w S - N S + Z,   K~_s = e^(gamma_C - gamma_s) k_s,
//     N = K~^T T (beta e^gamma K) + w - e^(gamma_C),   Z = K~^T T (beta V),   w = min(1, e^(gamma_C)).
// Three launches: one works N, Z and T out for all chunks at once, one walks the chunks with the states, a product each, one makes all
// outputs from the states in front of the chunks.  In long sequences the first and the last take runs of chunks (chunks_to_a_run), T comes in a
// launch of its own, and the walk has a step to a run.
// Times below: us, 65536 tokens in 4 sequences, 12 heads of 64, bf16 without states (a), or 1 sequence, 16 heads of 128, with states (b).
#include "chela_delta.h"

namespace chela {

// ---- a chunk's T, N and Z.  All of it on what is in LDS, thirty-two columns of N or Z to a wave.  6007 tokens in 11 sequences, 12 heads of 64, with
// states: 22, a round and a half of workgroups, each of which waits for its tiles, then for the inverse, a row after the other.
template <typename E, int DK, int DV, int P>
__global__ __launch_bounds__(256, DK + DV == 128 ? 4 : 2) void delta_prep_kernel(DeltaArgs a)
{
    constexpr int C = DeltaChunk<E>::C, NB = C / 16, KC = C / 32, LK = DK + kPad<E>, LV = DV + kPad<E>, LT = C + kPadT<E>;
    __shared__ __align__(16) E sK[C * LK], sV[C * LV], sT[inverse_room<E>()];
    __shared__ ChunkSteps<C> st;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), q = lane >> 4, c = lane & 15;
    const int place = blockIdx.x / a.H, h = blockIdx.x - place * a.H, hk = h / (a.H / a.Hk);
    const Chunk ch = chunk_at(a.rows, C, place, lane);
    if (ch.n <= 0) return;
    {
        Tile<E, C, DK> k;
        Tile<E, C, DV> v;
        const Steps s = fetch_steps((const E*)a.g, a.ldg, (const E*)a.beta, a.ldb, ch.row, h, ch.n, lane);
        k.fetch((const E*)a.K + hk * DK, a.ldk, ch.row, ch.n, tid);
        v.fetch((const E*)a.V + h * DV, a.ldv, ch.row, ch.n, tid);
        put_steps(st, s, ch.n, tid);
        k.put(sK, LK, ch.n, tid);
        v.put(sV, LV, ch.n, tid);
    }
    __syncthreads();
    const Planes<E, 2> T{sT, LT, C * LT};
    chunk_inverse<E, DK>(sK, LK, st, (float*)sT, T, tid);
    const size_t at = (size_t)place * a.H + h;
    PackedT<E, C, 256>::store(WordsOfPlanes<E>{T}, (E*)a.T + at * (C * C), tid);             // for the kernels behind
    if (tid == 0) a.whole[at] = no_growth(st.whole);
    const float grown = st.whole - no_growth(st.whole);
    // T (beta e^gamma K), T (beta V), thirty-two columns at a time, and what K~ makes of them
#pragma unroll 1
    for (int p = w; p < (DK + DV) / 32; p += 4) {
        read_afresh();
        const bool of_k = p < DK / 32;
        const int col = 32 * (of_k ? p : p - DK / 32);
        const E* X = of_k ? sK : sV;
        const int ldx = of_k ? LK : LV;
        const float* f = of_k ? st.bu : st.beta;          // (N is kept with its sign changed)
        f32x4 y[NB][2];
#pragma unroll
        for (int b = 0; b < NB; ++b) y[b][0] = y[b][1] = zero4();
#pragma unroll
        for (int ks = 0; ks < KC; ++ks) {
            const Op<E, 2> x0 = scaled<E, 2>(cols_op(X, ldx, 32 * ks, col, lane), f, 32 * ks, lane);
            const Op<E, 2> x1 = scaled<E, 2>(cols_op(X, ldx, 32 * ks, col + 16, lane), f, 32 * ks, lane);
#pragma unroll
            for (int b = 2 * ks; b < NB; ++b) {
                const Op<E, 2> m = T.rows(16 * b, 32 * ks, lane);
                y[b][0] = mma(m, x0, y[b][0]);
                y[b][1] = mma(m, x1, y[b][1]);
            }
        }
        Op<E, 2> yo[KC][2];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const f32x4 d = *(const f32x4*)(st.down + 16 * b + 4 * q);
            y[b][0] *= d;
            y[b][1] *= d;
        }
#pragma unroll
        for (int ks = 0; ks < KC; ++ks) {
            yo[ks][0] = operand<E, 2>(y[2 * ks][0], y[2 * ks + 1][0]);
            yo[ks][1] = operand<E, 2>(y[2 * ks][1], y[2 * ks + 1][1]);
        }
#pragma unroll
        for (int n = 0; n < DK / 16; ++n) {
            f32x4 r0 = zero4(), r1 = zero4();
            if (of_k && n / 2 == p) {
                if (n % 2 == 0) r0 = plus_diagonal(r0, grown, lane);
                else r1 = plus_diagonal(r1, grown, lane);
            }
#pragma unroll
            for (int ks = 0; ks < KC; ++ks) {
                const Op<E, 1> k = cols_op(sK, LK, 32 * ks, 16 * n, lane);
                if (of_k) { r0 = mma(yo[ks][0], k, r0); r1 = mma(yo[ks][1], k, r1); }
                else { r0 = mma(k, yo[ks][0], r0); r1 = mma(k, yo[ks][1], r1); }
            }
            if (of_k) {
                store_op<E, P>((E*)a.N + (at * (DK / 16 * (DK / 32)) + n * (DK / 32) + p) * kOpElems<E, P>, operand<E, P>(r0, r1), lane);
            } else {
                float* z = a.Z + at * (DK * DV) + (size_t)(col / 16 * (DK / 16) + n) * 256 + 4 * lane;
                *(f32x4*)z = r0;
                *(f32x4*)(z + DK / 16 * 256) = r1;
            }
        }
    }
}

// ---- T alone, of all chunks, for runs of them (within a run's workgroup it would be one chunk's after the other: (b) 890 for both kernels in one, 820 in
// two).  (a) 71, 200 MB, where the copy's rate would give 39: the inverse's steps wait for each other; five workgroups to a compute unit.  (T goes through LDS as
// words of both parts: as two planes, which only products need, 75.)
template <typename E, int DK>
__global__ __launch_bounds__(256, 4) void delta_inverse_kernel(DeltaArgs a)
{
    constexpr int C = DeltaChunk<E>::C, LK = DK + kPad<E>;
    __shared__ __align__(16) E sK[C * LK];
    __shared__ __align__(16) float sT[C * (C + 4)];
    __shared__ ChunkSteps<C> st;
    const int tid = threadIdx.x, lane = tid & 63;
    const int i = blockIdx.x / a.H, h = blockIdx.x - i * a.H, hk = h / (a.H / a.Hk);
    const Chunk ch = chunk_at(a.rows, C, i, lane);
    if (ch.n <= 0) return;
    Tile<E, C, DK> k;
    const Steps s = fetch_steps((const E*)a.g, a.ldg, (const E*)a.beta, a.ldb, ch.row, h, ch.n, lane);
    k.fetch((const E*)a.K + hk * DK, a.ldk, ch.row, ch.n, tid);
    put_steps(st, s, ch.n, tid);
    k.put(sK, LK, ch.n, tid);
    __syncthreads();
    const Words<E> T{(unsigned*)sT, C + 4};
    chunk_inverse<E, DK>(sK, LK, st, sT, T, tid);
    PackedT<E, C, 256>::store(T, (E*)a.T + ((size_t)i * a.H + h) * (C * C), tid);
}

// ---- the same for a run of chunks: one N and one Z for all of them, so that the walk has fewer steps and less to read.  The state behind the
// run's first chunks is taken through the next as the walk does it, Z beside what is left of the identity (X = M - w, M the transition so far,
// w = e^(sum of all log decays so far), held to 1), thirty-two columns to a wave:
//     U = T (beta V - beta e^gamma K Z),   or of X's columns  -T beta e^gamma K (X + w);   X <- e^gamma X + K~^T U + e^gamma w - w_next.
// (K is what the caller gave and has one part, T K of the chunk alone would have two: 119 and 574 so.)  (a) 107, 400 MB at 3.7 TB/s; (b) 426,
// instruction issue: vector instructions 56 % of the time (values split into two parts, scaled), matrix instructions 34 (340 GFLOP with all
// parts, 0.8 PFLOP/s); 187 registers, two waves to a SIMD.  For heads of 64 and 64 three waves are asked for (vector 77 %, matrix 31): the compiler finds three without
// that too, and 5 % more time; where there are 128 value columns it spills for them.
template <typename E, int DK, int DV, int P>
__global__ __launch_bounds__((DK + DV) * 2, DK + DV == 128 ? 3 : 1) void delta_prep_run_kernel(DeltaArgs a)
{
    constexpr int C = DeltaChunk<E>::C, NB = C / 16, KC = C / 32, KS = DK / 32, LK = DK + kPad<E>, LV = DV + kPad<E>, LT = C + kPad<E>;
    constexpr int NT = (DK + DV) * 2;
    __shared__ __align__(16) E sK[C * LK], sV[C * LV], sT[kScores<E>];
    __shared__ ChunkSteps<C> st;
    const int tid0 = threadIdx.x, lane0 = tid0 & 63, w = __builtin_amdgcn_readfirstlane(tid0 >> 6);
    const int place = blockIdx.x / a.H, h = blockIdx.x - place * a.H, hk = h / (a.H / a.Hk);
    const Chunk ch = chunk_at(a.rows, C * a.run, place, lane0);
    if (ch.n <= 0) return;
    const size_t at = (size_t)place * a.H + h;
    const int chunk0 = chunk_place(a.rows, C, ch, a.run, 0);
    const bool of_k = w < DK / 32;
    const int col = 32 * (of_k ? w : w - DK / 32);
    Tile<E, C, DK, NT> tk;
    Tile<E, C, DV, NT> tv;
    PackedT<E, C, NT> tt;
    Steps ts;
    auto fetch = [&](int r, int tid, int lane) {
        const int row = ch.row + r * C, n = min(C, ch.n - r * C);
        ts = fetch_steps((const E*)a.g, a.ldg, (const E*)a.beta, a.ldb, row, h, n, lane);
        tk.fetch((const E*)a.K + hk * DK, a.ldk, row, n, tid);
        tv.fetch((const E*)a.V + h * DV, a.ldv, row, n, tid);
        tt.fetch((const E*)a.T + ((size_t)(chunk0 + r) * a.H + h) * (C * C), tid);
    };
    fetch(0, tid0, lane0);
    const Planes<E, 2> T{sT, LT, C * LT};
    f32x4 X[DK / 16][2];
#pragma unroll
    for (int d = 0; d < DK / 16; ++d) X[d][0] = X[d][1] = zero4();
    float before = 1.f;
    for (int r = 0; r * C < ch.n; ++r) {
        const int n = min(C, ch.n - r * C);
        const bool last = (r + 1) * C >= ch.n;
        int lane = lane0;
        asm volatile("" : "+v"(lane));             // (addresses are worked out where they are used: kept over the chunks, they fill the registers)
        const int tid = 64 * w + lane, q = lane >> 4, c = lane & 15;
        if (r > 0) __syncthreads();
        put_steps(st, ts, n, tid);
        tk.put(sK, LK, n, tid);
        tv.put(sV, LV, n, tid);
        tt.put(T, tid);
        if (!last) fetch(r + 1, tid, lane);
        __syncthreads();
        // beta V - beta e^gamma K Z, or of the transition the same without V
        f32x4 y[NB][2];
#pragma unroll
        for (int b = 0; b < NB; ++b) y[b][0] = y[b][1] = zero4();
        if (of_k)
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                y[b][0] = splat4(before) * tile_of(sK, LK, 16 * b, col, lane);
                y[b][1] = splat4(before) * tile_of(sK, LK, 16 * b, col + 16, lane);
            }
        if (r > 0)
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
            const f32x4 f = *(const f32x4*)(st.bu + 16 * b + 4 * q);
            y[b][0] *= f;
            y[b][1] *= f;
            if (!of_k) {
                const f32x4 be = *(const f32x4*)(st.beta + 16 * b + 4 * q);
                y[b][0] += be * tile_of(sV, LV, 16 * b, col, lane);
                y[b][1] += be * tile_of(sV, LV, 16 * b, col + 16, lane);
            }
        }
        Op<E, 2> yo[KC][2];
#pragma unroll
        for (int ks = 0; ks < KC; ++ks)
#pragma unroll
            for (int g = 0; g < 2; ++g) yo[ks][g] = operand<E, 2>(y[2 * ks][g], y[2 * ks + 1][g]);
        // what the tokens write, T of it
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            y[b][0] = y[b][1] = zero4();
#pragma unroll
            for (int ks = 0; ks <= b / 2; ++ks) {
                const Op<E, 2> m = T.rows(16 * b, 32 * ks, lane);
                y[b][0] = mma(m, yo[ks][0], y[b][0]);
                y[b][1] = mma(m, yo[ks][1], y[b][1]);
            }
            const f32x4 d = *(const f32x4*)(st.down + 16 * b + 4 * q);
            y[b][0] *= d;
            y[b][1] *= d;
        }
#pragma unroll
        for (int ks = 0; ks < KC; ++ks)
#pragma unroll
            for (int g = 0; g < 2; ++g) yo[ks][g] = operand<E, 2>(y[2 * ks][g], y[2 * ks + 1][g]);
        const float whole = st.whole, after = no_growth(before * whole), grown = before * whole - after;
#pragma unroll
        for (int n0 = 0; n0 < DK / 16; n0 += 2) {
            read_afresh();
            f32x4 z[2][2];                                 // [row of tiles][columns]
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int g = 0; g < 2; ++g) z[i][g] = X[n0 + i][g] * splat4(whole);
            if (n0 / 2 == w) {                             // (only of X, whose waves come first)
                z[0][0] = plus_diagonal(z[0][0], grown, lane);
                z[1][1] = plus_diagonal(z[1][1], grown, lane);
            }
            if (last && of_k) {
                // as N is read, the columns of X down the rows of a tile: its old part by products with the identity
                const Op<E, 2> x0 = operand<E, 2>(z[0][0], z[1][0]), x1 = operand<E, 2>(z[0][1], z[1][1]);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    f32x4 lo = zero4(), hi = zero4();
#pragma unroll
                    for (int j = 0; j < 4; ++j) lo[j] = 4 * q + j == c ? 1.f : 0.f;
                    const Op<E, 1> one = i == 0 ? operand<E, 1>(lo, hi) : operand<E, 1>(hi, lo);
                    f32x4 r0 = mma(x0, one, zero4()), r1 = mma(x1, one, zero4());
#pragma unroll
                    for (int ks = 0; ks < KC; ++ks) {
                        const Op<E, 1> k = cols_op(sK, LK, 32 * ks, 16 * (n0 + i), lane);
                        r0 = mma(yo[ks][0], k, r0);
                        r1 = mma(yo[ks][1], k, r1);
                    }
                    store_op<E, P>((E*)a.N + (at * (DK / 16 * KS) + (n0 + i) * KS + w) * kOpElems<E, P>, operand<E, P>(r0, r1), lane);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int ks = 0; ks < KC; ++ks) {
                        const Op<E, 1> k = cols_op(sK, LK, 32 * ks, 16 * (n0 + i), lane);
                        z[i][0] = mma(k, yo[ks][0], z[i][0]);
                        z[i][1] = mma(k, yo[ks][1], z[i][1]);
                    }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        X[n0 + i][g] = z[i][g];
                        if (last) *(f32x4*)(a.Z + at * (DK * DV) + (size_t)((col / 16 + g) * (DK / 16) + n0 + i) * 256 + 4 * lane) = z[i][g];
                    }
            }
        }
        before = after;
    }
    if (tid0 == 0) a.whole[at] = before;
}

// ---- the walk: S <- w S + Z - N S from chunk to chunk (N comes negated), sixteen of S's columns to a workgroup, sixteen of its rows to a wave.
// Each wave keeps its rows in fp32 and hands them to the others as operands, through LDS; what the next chunks need is on its way
// meanwhile.  REV: from the last chunk to the first, with the states' gradients.  (a) 32 for 64 runs: a step is one wave's turn to LDS, a barrier and
// a product.  Chunk by chunk 110; 32768 tokens in 8 sequences, 12 heads of 64 and 128, so 89: 690 MB through the L2s, each head's N to all groups of
// columns.  (Thirty-two columns to a workgroup, which halves that, leaves too few of them: slower.)
template <typename E, int DK, int P, bool REV>
__global__ __launch_bounds__(DK * 4) void delta_walk_kernel(DeltaArgs a, int DV)
{
    constexpr int C = DeltaChunk<E>::C, KS = DK / 32, NE = kOpElems<E, P>, OE = kOpElems<E, 2>, AHEAD = DK == 64 && P == 1 ? 8 : 4;
    __shared__ __align__(16) E sS[2][KS * OE];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), q = lane >> 4, c = lane & 15;
    // (workgroups go to the eight L2s in turn: those of one head, which read the same N, to one of them)
    const int groups = DV / 16, all = a.rows.n_seq * a.H * groups, id = (int)(blockIdx.x & 7) * ((all + 7) / 8) + (int)(blockIdx.x >> 3);
    if (id >= all) return;
    const int eg = id % groups, h = id / groups % a.H, seq = id / groups / a.H;
    const int first = chunk_key(a.rows, C * a.run, seq), n = min(chunks_in(a.rows, C * a.run, seq), a.places - first);
    const int slot = slot_of(a.rows, seq);
    const float* from = REV ? a.dS_out : a.S_in;
    float* to = REV ? a.dS_in : a.S_out;
    E* keep = (E*)(REV ? a.dS : a.S0) + (size_t)eg * (DK * 16) + (w >> 1) * 512 + 8 * lane + 4 * (w & 1);
    const float* z = a.Z + (size_t)(eg * (DK / 16) + w) * 256 + 4 * lane;
    const E* nn = (const E*)a.N + (size_t)w * KS * NE;
    f32x4 S = zero4();
    const size_t mine = (((size_t)max(slot, 0) * a.H + h) * DK + 16 * w + 4 * q) * DV + 16 * eg + c;
    if (from != nullptr && slot >= 0)
#pragma unroll
        for (int j = 0; j < 4; ++j) S[j] = from[mine + (size_t)j * DV];
    Op<E, P> N[AHEAD][KS];
    f32x4 Z[AHEAD];
    float whole[AHEAD];
    auto load = [&](int u, int k) {
        k = min(k, n - 1);
        const size_t at = (size_t)(first + (REV ? n - 1 - k : k)) * a.H + h;
        whole[u] = a.whole[at];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) N[u][ks] = load_op<E, P>(nn + at * (DK / 16 * KS * NE) + ks * NE, lane);
        Z[u] = *(const f32x4*)(z + at * ((size_t)DK * DV));
    };
    if (n > 0) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) load(u, u);
    }
    for (int k0 = 0; k0 < n; k0 += AHEAD) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int k = k0 + u;
            if (k >= n) break;
            E* out = keep + ((size_t)(first + (REV ? n - 1 - k : k)) * a.H + h) * ((size_t)DK * DV);
            // (the wave's rows are one half of an operand's terms)
            E* half = sS[u & 1] + (w >> 1) * OE + 8 * lane + 4 * (w & 1);
            if constexpr (sizeof(E) == 4) {
                *(f32x4*)half = S;
                *(f32x4*)out = S;
            } else {
                const bf16x4 hi = __builtin_convertvector(S, bf16x4);
                *(bf16x4*)half = hi;
                *(bf16x4*)(half + 512) = __builtin_convertvector(S - widen(hi), bf16x4);
                *(bf16x4*)out = hi;
            }
            __syncthreads();
            S = S * whole[u] + Z[u];
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) S = mma(N[u][ks], load_op<E, 2>(sS[u & 1] + ks * OE, lane), S);
            load(u, k + AHEAD);
        }
    }
    if (to != nullptr && slot >= 0)
#pragma unroll
        for (int j = 0; j < 4; ++j) to[mine + (size_t)j * DV] = S[j];
}

// ---- the outputs
// Sixteen value columns to a wave; a run's chunks one after the other, the state from chunk to chunk in the wave's registers.  (a) 136, 600 MB at
// 4.4 TB/s, the states for the gradient among them; (b) 316, 1.2 GB at 3.9: vector instructions 57 % of the time, matrix instructions 32, LDS 50.  The scores
// are worked out behind the inner values, where T was: with room of their own for both parts two workgroups would fit in a compute unit, not three.
template <typename E, int DK, int DV>
__global__ __launch_bounds__(DV * 4, sizeof(E) == 2 ? (DV == 128 ? 4 : DK == 64 ? 3 : 2) : 2) void delta_out_kernel(DeltaArgs a)
{
    constexpr int C = DeltaChunk<E>::C, NB = C / 16, KC = C / 32, KS = DK / 32, LK = DK + kPad<E>, LV = DV + kPad<E>, LT = C + kPad<E>, NT = DV * 4;
    __shared__ __align__(16) E sK[C * LK], sQ[C * LK], sV[C * LV], sT[kScores<E>];          // (T, then P)
    __shared__ ChunkSteps<C> st;
    const int tid0 = threadIdx.x, lane0 = tid0 & 63, w = __builtin_amdgcn_readfirstlane(tid0 >> 6);
    const int place = blockIdx.x / a.H, h = blockIdx.x - place * a.H, hk = h / (a.H / a.Hk);
    if (place >= a.places) {
        clear_rows(a.rows, blockIdx.x - a.places * a.H, (E*)a.O, a.H * DV);
        return;
    }
    const Chunk ch = chunk_at(a.rows, C * a.run, place, lane0);
    if (ch.n <= 0) return;
    const E* S0 = (const E*)a.S0 + ((size_t)place * a.H + h) * (DK * DV) + (size_t)w * (KS * 512);
    const int chunk0 = chunk_place(a.rows, C, ch, a.run, 0);
    Tile<E, C, DK, NT> tk, tq;
    Tile<E, C, DV, NT> tv;
    PackedT<E, C, NT> tt;
    Steps ts;
    auto fetch = [&](int r, int tid, int lane) {
        const int row = ch.row + r * C, n = min(C, ch.n - r * C);
        ts = fetch_steps((const E*)a.g, a.ldg, (const E*)a.beta, a.ldb, row, h, n, lane);
        tk.fetch((const E*)a.K + hk * DK, a.ldk, row, n, tid);
        tq.fetch((const E*)a.Q + hk * DK, a.ldq, row, n, tid);
        tv.fetch((const E*)a.V + h * DV, a.ldv, row, n, tid);
        tt.fetch((const E*)a.T + ((size_t)(chunk0 + r) * a.H + h) * (C * C), tid);
    };
    const Planes<E, 2> T{sT, LT, C * LT};
    Op<E, 1> so[KS];
    f32x4 S[DK / 16];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) so[ks] = load_op<E, 1>(S0 + ks * 512, lane0);
    constexpr bool AHEAD = DV == 64;                       // (with eight waves to a workgroup there are no registers for it)
    if (AHEAD) fetch(0, tid0, lane0);
    for (int r = 0; r * C < ch.n; ++r) {
        const int n = min(C, ch.n - r * C);
        const bool last = (r + 1) * C >= ch.n;
        int lane = lane0;
        asm volatile("" : "+v"(lane));             // (addresses are worked out where they are used: kept over the chunks, they fill the registers)
        const int tid = 64 * w + lane, q = lane >> 4, c = lane & 15;
        if (!AHEAD) fetch(r, tid, lane);
        if (r > 0) __syncthreads();
        put_steps(st, ts, n, tid);
        tk.put(sK, LK, n, tid);
        tq.put(sQ, LK, n, tid);
        tv.put(sV, LV, n, tid);
        tt.put(T, tid);
        if (AHEAD && !last) fetch(r + 1, tid, lane);
        __syncthreads();
        if (a.S0c != nullptr)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
                store_op<E, 1>((E*)a.S0c + ((size_t)(chunk0 + r) * a.H + h) * (DK * DV) + (w * KS + ks) * 512, so[ks], lane);
        Op<E, 2> ro[KC], uo[KC];
        f32x4 x[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            if (b % 2 == 0) read_afresh();
            x[b] = zero4();
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) x[b] = mma(rows_op(sK, LK, 16 * b, 32 * ks, lane), so[ks], x[b]);
            x[b] = x[b] * *(const f32x4*)(st.bu + 16 * b + 4 * q) + *(const f32x4*)(st.beta + 16 * b + 4 * q) * tile_of(sV, LV, 16 * b, 16 * w, lane);
        }
#pragma unroll
        for (int ks = 0; ks < KC; ++ks) ro[ks] = operand<E, 2>(x[2 * ks], x[2 * ks + 1]);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            x[b] = zero4();
#pragma unroll
            for (int ks = 0; ks <= b / 2; ++ks) x[b] = mma(T.rows(16 * b, 32 * ks, lane), ro[ks], x[b]);
        }
#pragma unroll
        for (int ks = 0; ks < KC; ++ks) uo[ks] = operand<E, 2>(x[2 * ks], x[2 * ks + 1]);
        __syncthreads();
        // the scores, where T was
        if (w < NB) {
            const int t = 16 * w + c;
            for (int sb = 0; sb <= (w | 1); ++sb) {
                f32x4 p = zero4();
                if (sb <= w) {
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) p = mma(rows_op(sK, LK, 16 * sb, 32 * ks, lane), rows_op(sQ, LK, 16 * w, 32 * ks, lane), p);
                    p *= splat4(a.scale) * st.decays_from(t, 16 * sb + 4 * q);
                    if (sb == w)
#pragma unroll
                        for (int i = 0; i < 4; ++i) p[i] = 4 * q + i <= c ? p[i] : 0.f;
                }
                T.put4(t, 16 * sb, q, p);
            }
        }
        __syncthreads();
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            if (b % 2 == 0) read_afresh();
            const int t = 16 * b + c;
            f32x4 o = zero4();
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) o = mma(so[ks], rows_op(sQ, LK, 16 * b, 32 * ks, lane), o);
            o *= splat4(a.scale * st.up[t]);
#pragma unroll
            for (int ks = 0; ks <= b / 2; ++ks) o = mma(uo[ks], T.rows(16 * b, 32 * ks, lane), o);
            if (t < n)
                *(Vec4<E>*)((E*)a.O + (size_t)(ch.row + r * C + t) * (a.H * DV) + h * DV + 16 * w + 4 * q) = __builtin_convertvector(o, Vec4<E>);
        }
        if (last) break;
        // the state in front of the next chunk
        const float whole = st.whole;
        if (r == 0) {
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                f32x8 v;
                if constexpr (sizeof(E) == 4) v = so[ks].v;
                else v = __builtin_convertvector(so[ks].h, f32x8);
                S[2 * ks] = __builtin_shufflevector(v, v, 0, 1, 2, 3);
                S[2 * ks + 1] = __builtin_shufflevector(v, v, 4, 5, 6, 7);
            }
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) x[b] *= *(const f32x4*)(st.down + 16 * b + 4 * q);
#pragma unroll
        for (int ks = 0; ks < KC; ++ks) uo[ks] = operand<E, 2>(x[2 * ks], x[2 * ks + 1]);
#pragma unroll
        for (int d = 0; d < DK / 16; ++d) {
            if (d % 4 == 0) read_afresh();
            S[d] *= splat4(whole);
#pragma unroll
            for (int ks = 0; ks < KC; ++ks) S[d] = mma(cols_op(sK, LK, 32 * ks, 16 * d, lane), uo[ks], S[d]);
        }
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) so[ks] = operand<E, 1>(S[2 * ks], S[2 * ks + 1]);
    }
}

// ---- a single token of each request: the state is read and written once, four columns and DK / R rows to a thread.  256 requests, 12 heads of
// 64: 18, 102 MB at 5.7 TB/s; one request 4, a launch.
template <typename E, int DK, int DV>
__global__ __launch_bounds__(256) void delta_step_kernel(DeltaArgs a)
{
    constexpr int L = DV / 4, R = 256 / L, M = DK / R;                // threads to a row, rows at a time, rows to a thread
    __shared__ float sk[DK], sq[DK];
    __shared__ __align__(16) f32x4 s_r[R][L], s_p[R][L];
    __shared__ float s_qk[4];
    const int tid = threadIdx.x, r = blockIdx.x / a.H, h = blockIdx.x - r * a.H, hk = h / (a.H / a.Hk);
    const int l = tid % L, j = tid / L;
    const int slot = slot_of(a.rows, r);
    E* o = (E*)a.O + ((size_t)r * a.H + h) * DV;
    if (slot < 0) {
        if (a.rows.clear) for (int i = tid; i < DV; i += 256) o[i] = (E)0.f;
        return;
    }
    float* S = a.S_out + ((size_t)slot * a.H + h) * (DK * DV) + 4 * l;
    f32x4 x[M];
#pragma unroll
    for (int m = 0; m < M; ++m) x[m] = *(const f32x4*)(S + (size_t)(m * R + j) * DV);
    float alpha = 1.f;
    if (a.g != nullptr) alpha = exp2_(kLog2e * to_f(((const E*)a.g)[(size_t)r * a.ldg + h]));
    const float beta = to_f(((const E*)a.beta)[(size_t)r * a.ldb + h]);
    const E* v = (const E*)a.V + (size_t)r * a.ldv + h * DV + 4 * l;
    f32x4 vv;
#pragma unroll
    for (int i = 0; i < 4; ++i) vv[i] = to_f(v[i]);
    float qk = 0.f;
    for (int i = tid; i < DK; i += 256) {
        const float k = to_f(((const E*)a.K)[(size_t)r * a.ldk + hk * DK + i]), y = to_f(((const E*)a.Q)[(size_t)r * a.ldq + hk * DK + i]);
        sk[i] = k;
        sq[i] = y;
        qk = k * y;
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) qk += __shfl_xor(qk, d);
    if ((tid & 63) == 0) s_qk[tid >> 6] = qk;
    __syncthreads();
    f32x4 rd = zero4(), p = zero4();
#pragma unroll
    for (int m = 0; m < M; ++m) {
        x[m] *= splat4(alpha);
        rd += x[m] * splat4(sk[m * R + j]);
        p += x[m] * splat4(sq[m * R + j]);
    }
    s_r[j][l] = rd;
    s_p[j][l] = p;
    __syncthreads();
    rd = p = zero4();
#pragma unroll
    for (int i = 0; i < R; ++i) { rd += s_r[i][l]; p += s_p[i][l]; }
    const f32x4 u = splat4(beta) * (vv - rd);
#pragma unroll
    for (int m = 0; m < M; ++m) *(f32x4*)(S + (size_t)(m * R + j) * DV) = x[m] + splat4(sk[m * R + j]) * u;
    if (j == 0) {
        const f32x4 y = splat4(a.scale) * (p + splat4(s_qk[0] + s_qk[1]) * u);
        *(Vec4<E>*)(o + 4 * l) = __builtin_convertvector(y, Vec4<E>);
    }
}

// -------------------------------------------------------------------------------------------------------------------- host
bool delta_dims_ok(int dk, int dv) { return (dk == 64 || dk == 128) && (dv == 64 || dv == 128); }

// Chunks to a run, a power of two.  A run's chunks are one after the other in a workgroup, the runs of a sequence in the walk: R c + n w / R for n
// chunks, c and w the times that a chunk takes of either, is least where R^2 = n w / c.  w / c is about 1/16 with heads of 64, 1/8 where there are
// heads of 128 (0.5 us of 8, 1.3 of 12), 1/32 with fp32's shorter chunks.  Measured (us; R = 1, 2, 4, 8, 16), bf16, nothing kept, 12 heads of 64, one
// sequence of 2048 tokens 41 44 57 89 157, of 8192 102 92 90 108 173, of 32768 328 275 235 220 255; 8 of 1024 60 69 76 99 163; 16 heads of
// 128, 2048 tokens 78 74 93 149 269, 8192 355 254 205 207 312, 65536 2475 2057 1621 1401 1299.  With what a gradient needs kept, and the gradient
// (R = 1, 2, 4, 8): 12 heads of 64, one sequence of 4096 48 51 56 85, 69 68 89 158, of 16384 147 136 117 134, 216 185 184 206, 4 of 8192 220 204
// 193 188, 344 322 311 337; 16 heads of 128, 8 of 4096 730 697 616 582, 1270 1393 1268 1220; fp32, 12 heads of 64, 8 of 1024 107 119 114 136, 250
// 250 239 302, one of 4096 104 91 88 93, 170 150 169 169.
static int chunks_to_a_run(long n, int dk, int dv, int dtype)
{
    const int w = dk + dv > 128 ? 8 : dtype != 0 ? 32 : 16;
    int r = 1;
    while (r < 16 && (long)r * r * w < n) r *= 2;
    return r;
}

DeltaPlan make_delta_plan(int T, int n_seq, bool packed, int H, int Hk, int dk, int dv, int dtype, bool is_bwd, bool has_saved, bool fine)
{
    DeltaPlan p{};
    const size_t es = dtype != 0 ? 4 : 2;
    p.parts = dtype == 0 && fine ? 2 : 1;
    p.chunk = dtype != 0 ? kDeltaChunkF32 : kDeltaChunkBf16;
    const int len = n_seq > 0 ? T / n_seq : 0;
    auto places = [&](int tokens) { return T <= 0 || n_seq <= 0 ? 0 : packed ? T / tokens + n_seq : n_seq * ((len + tokens - 1) / tokens); };
    p.run = chunks_to_a_run(((long)len + p.chunk - 1) / p.chunk, dk, dv, dtype);
    if (is_bwd && H != Hk) p.run = 1;                          // (a gradient walks the runs with a state for one value head)
    p.chunks = places(p.chunk);
    p.places = places(p.chunk * p.run);
    const size_t all = (size_t)p.chunks * H, n = is_bwd && !has_saved ? all : (size_t)p.places * H;      // (the states are then walked chunk by chunk)
    auto room = [](size_t& at, size_t bytes) { const size_t was = at; at += (bytes + 255) & ~(size_t)255; return was; };
    p.own_states = !is_bwd && p.run > 1;
    p.T = room(p.saved_bytes, all * p.chunk * p.chunk * es);
    p.S0c = p.saved_bytes;
    if (is_bwd || has_saved || !p.own_states) room(p.saved_bytes, all * dk * dv * es);
    p.N = room(p.bytes, n * p.parts * dk * dk * es);
    p.Z = room(p.bytes, n * dk * dv * sizeof(float));
    p.whole = room(p.bytes, n * sizeof(float));
    if (p.own_states) p.S0 = room(p.bytes, n * dk * dv * es);
    if (is_bwd) p.dS = room(p.bytes, (size_t)p.places * H * dk * dv * es);
    p.saved_at = p.bytes;
    if (!has_saved) p.bytes += p.saved_bytes;
    return p;
}

hipError_t launch_delta_walk(const DeltaArgs& a, bool reverse, int parts, int dk, int dv, int dtype, hipStream_t st)
{
    if (a.rows.n_seq == 0) return hipSuccess;
    const dim3 grid((unsigned)(((size_t)a.rows.n_seq * a.H * (dv / 16) + 7) / 8 * 8));
#define CHELA_W(E, DK, P)                                                                                             \
    if (reverse) hipLaunchKernelGGL((delta_walk_kernel<E, DK, P, true>), grid, dim3(DK * 4), 0, st, a, dv);        \
    else hipLaunchKernelGGL((delta_walk_kernel<E, DK, P, false>), grid, dim3(DK * 4), 0, st, a, dv)
    if (dtype != 0) { if (dk == 64) { CHELA_W(float, 64, 1); } else { CHELA_W(float, 128, 1); } }
    else if (parts == 2) { if (dk == 64) { CHELA_W(bf16, 64, 2); } else { CHELA_W(bf16, 128, 2); } }
    else { if (dk == 64) { CHELA_W(bf16, 64, 1); } else { CHELA_W(bf16, 128, 1); } }
#undef CHELA_W
    return hipGetLastError();
}

// T of all chunks, the states in front of all runs.
hipError_t launch_delta_states(DeltaArgs& a, const DeltaPlan& p, int dk, int dv, int dtype, hipStream_t st)
{
    if (p.places > 0) {
        const dim3 grid((unsigned)((size_t)a.places * a.H)), chunks((unsigned)((size_t)p.chunks * a.H));
#define CHELA_RUN(E, DK, DV)                                                                                          \
    do {                                                                                                              \
        constexpr int P2 = sizeof(E) == 2 ? 2 : 1;                                                                    \
        if (a.run > 1) {                                                                                              \
            hipLaunchKernelGGL((delta_inverse_kernel<E, DK>), chunks, dim3(256), 0, st, a);                           \
            if (p.parts == 2) hipLaunchKernelGGL((delta_prep_run_kernel<E, DK, DV, P2>), grid, dim3((DK + DV) * 2), 0, st, a); \
            else hipLaunchKernelGGL((delta_prep_run_kernel<E, DK, DV, 1>), grid, dim3((DK + DV) * 2), 0, st, a);       \
        } else {                                                                                                      \
            if (p.parts == 2) hipLaunchKernelGGL((delta_prep_kernel<E, DK, DV, P2>), grid, dim3(256), 0, st, a);      \
            else hipLaunchKernelGGL((delta_prep_kernel<E, DK, DV, 1>), grid, dim3(256), 0, st, a);                    \
        }                                                                                                             \
    } while (0)
        CHELA_DELTA(CHELA_RUN)
#undef CHELA_RUN
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return launch_delta_walk(a, false, p.parts, dk, dv, dtype, st);
}

hipError_t launch_delta_fwd(DeltaArgs a, const DeltaPlan& p, char* ws, char* saved, int dk, int dv, int dtype, hipStream_t st)
{
    ProfScope prof(KID_DELTA, st);
    const bool kept = saved != nullptr;
    if (!kept) saved = ws + p.saved_at;
    a.places = p.places;
    a.run = p.run;
    a.N = ws + p.N;
    a.Z = (float*)(ws + p.Z);
    a.whole = (float*)(ws + p.whole);
    a.T = saved + p.T;
    a.S0 = p.own_states ? ws + p.S0 : saved + p.S0c;
    a.S0c = p.own_states && kept ? saved + p.S0c : nullptr;
    const hipError_t e = launch_delta_states(a, p, dk, dv, dtype, st);
    if (e != hipSuccess) return e;
    const bool clear = a.rows.clear && a.rows.cu != nullptr;
    const size_t blocks = (size_t)p.places * a.H + (clear ? (a.rows.T + 63) / 64 : 0);
    if (blocks == 0) return hipSuccess;
    const dim3 grid((unsigned)blocks);
#define CHELA_RUN(E, DK, DV) hipLaunchKernelGGL((delta_out_kernel<E, DK, DV>), grid, dim3(DV * 4), 0, st, a)
    CHELA_DELTA(CHELA_RUN)
#undef CHELA_RUN
    return hipGetLastError();
}

hipError_t launch_delta_step(const DeltaArgs& a, int dk, int dv, int dtype, hipStream_t st)
{
    ProfScope prof(KID_DELTA_STEP, st);
    const dim3 grid((unsigned)((size_t)a.rows.n_seq * a.H));
#define CHELA_RUN(E, DK, DV) hipLaunchKernelGGL((delta_step_kernel<E, DK, DV>), grid, dim3(256), 0, st, a)
    CHELA_DELTA(CHELA_RUN)
#undef CHELA_RUN
    return hipGetLastError();
}

}  // namespace chela
