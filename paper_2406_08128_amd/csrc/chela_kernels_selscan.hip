// Selective state space scan for gfx950: prompts, gradient, single tokens.
//
// Per channel c (of group g) and state n, with dl_t = softplus(delta_t + bias) or delta_t + bias:
//     h_t[n] = exp(dl_t A[n]) h_{t-1}[n] + dl_t u_t B_t[n],   y_t = sum_n C_t[n] h_t[n] + D u_t,   out_t = y_t silu(z_t).
// Gradient, with dy_t = dout_t silu(z_t), a_t[n] = exp(dl_t A[n]), q_t[n] = a_t[n] g_t[n] and p_t[n] = a_t[n] h_{t-1}[n], as the forward walk has them again:
//     g_t[n] = C_t[n] dy_t + q_{t+1}[n]                             (the gradient of h_t)
//     dC_t[n] = sum_c dy_t h_t[n],   dB_t[n] = sum_c g_t[n] dl_t u_t,   dA[n] = sum_t dl_t g_t[n] p_t[n],   dD = sum_t dy_t u_t
//     du_t = dl_t sum_n g_t[n] B_t[n] + D dy_t,   d(dl_t) = u_t sum_n g_t[n] B_t[n] + sum_n A[n] g_t[n] p_t[n]
//     dz_t = dout_t y_t silu'(z_t);  d(delta_t) = d(dl_t) sigmoid(delta_t + bias) under the softplus.
//
// All of it is fp32 on the vector ALU: the decay differs from channel to channel and from state to state, so there is no matrix
// product in it.
//
// Split.  A lane owns a channel, a wave 64 of one group.  The rows are cut into chunks wherever the sequences begin and end: a
// first pass leaves, per chunk, what its rows add to the state behind them (the state itself, if a sequence begins in it) and the sum
// of its step sizes, of which the chunk's decay is exp(A sum); a second one makes the state in front of each chunk of these, and a third
// walks the chunks.
//
// What bounds it is the vector ALU's issue.  A row of 16 states takes 48 operations and 16 exponentials in the first pass, 64 and 16 in the
// third; alone, from registers, the latter keep a SIMD busy for 409 cycles (an operation 3, an exponential 12).  65536 rows in four sequences, 1536
// channels, 16 states, bf16, us: first pass 304 (the issue's floor 224), third with its saved states 417 (262; 1.6 GB at 3.9 TB/s), gradient:
// first pass 346, walk 1230, carries 25 and 16, sums of dB and dC over the channels' waves 59.  By the counters the vector ALUs are at work
// for all of the two passes' time and for 94 % of the gradient's walk: a row there takes 97 vector instructions per four states, 48 that the
// formulas have, 24 for the sums over channels, 25 for what a row has once (softplus, gate, conversions, its results' sums over states).
//
// The states that a forward call saves for its gradient take 0.8 GB at that size.  Without them the gradient walks the rows forward itself:
// 2080 us in all instead of 1500, and the forward call 676 instead of 693.
#include "chela_rows.h"
#include <type_traits>

namespace chela {

struct ScanShape {
    Rows rows;
    int D, N, G, Dg, nb;              // channels per group, waves per group
    int chunk, n_chunk, softplus, same_buffer;
};

struct ScanFwd {
    ScanShape s;
    const void *U, *delta, *Z, *Bm, *Cm;
    long ldu, ldd, ldz, ldb, ldc;
    const float *A, *Dskip, *dbias, *S_in;
    float *S_out, *saved, *totals, *sums, *fin;
    void* Y;
};

// Sequences without rows hand their states (or, in the backward call, the states' gradients) on: workgroup `first` of `groups`.
__device__ __forceinline__ void pass_states_on(const Rows& rows, const float* from, float* to, long n, int first, int groups)
{
    for (int s = first; s < rows.n_seq; s += groups) {
        if (seq_begin(rows, s) < seq_end(rows, s)) continue;
        const int slot = slot_of(rows, s);
        if (slot < 0) continue;
        for (long i = threadIdx.x; i < n; i += blockDim.x) to[slot * n + i] = from ? from[slot * n + i] : 0.f;
    }
}
__global__ __launch_bounds__(256) void selscan_empty_kernel(Rows rows, const float* from, float* to, long n)
{
    pass_states_on(rows, from, to, n, blockIdx.x, gridDim.x);
}

// Behind a call that writes its states over those it reads: the sequences that end in another chunk than they begin in.
__global__ __launch_bounds__(256) void selscan_finish_kernel(ScanShape s, const float* __restrict__ fin, float* __restrict__ S_out)
{
    const int c = blockIdx.y, t0 = c * s.chunk;
    const int q = seq_of(s.rows, t0);
    if (q < 0 || q >= s.rows.n_seq || seq_begin(s.rows, q) == t0 || seq_end(s.rows, q) > min(t0 + s.chunk, s.rows.T)) return;
    const int slot = slot_of(s.rows, q);
    if (slot < 0) return;
    const long n = (long)s.N * s.D;
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long)gridDim.x * 256) S_out[(size_t)slot * n + i] = fin[(size_t)c * n + i];
}

// The chunks' totals turned into what each chunk begins with, in place, in order (forward: from the first chunk on, state and decay; backward:
// from the last chunk on).  A chunk whose sum of step sizes is the mark has a sequence's beginning (end) in it: what comes to it ends there.
// (A sum that is not a number by itself comes with totals that are none.)  Workgroups from `groups` on: pass_states_on().
// Latency-bound: four waves share the chunks of 64 elements, each makes one step of its 32, takes in what is in front of them from the
// others, and goes over them again, all from registers.
__device__ __forceinline__ float reset_mark() { return __uint_as_float(0x7fc00000u); }
// exp(A sum) h + H, half of the exponent at a time: over many rows the decay itself may be nothing that a float holds (2^-140, 2^160) where the
// state is, before and behind.  half_A2: A / 2 in units of ln 2.  (A state of zero stays so however much growth has come together.)
__device__ __forceinline__ float carried(float h, float sum, float half_A2, float H)
{
    const float e = exp2_(sum * half_A2);
    return sum != sum || h == 0.f ? H : fmaf(e, e * h, H);
}
template <bool BWD>
__global__ __launch_bounds__(256) void selscan_carry_kernel(const float* __restrict__ A, float* __restrict__ totals,
                                                           const float* __restrict__ sums, int n_chunk, int D, long ND, int groups, Rows rows,
                                                           const float* from, float* to)
{
    if ((int)blockIdx.x >= groups) {
        pass_states_on(rows, from, to, ND, blockIdx.x - groups, gridDim.x - groups);
        return;
    }
    __shared__ float s_h[4][64], s_sum[4][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const bool live = (long)blockIdx.x * 64 + lane < ND;
    const long i = live ? (long)blockIdx.x * 64 + lane : ND - 1;
    const int ch = (int)(i % D);
    const float half_A2 = A[i] * (0.5f * kLog2e);
    float base = 0.f;                                // what comes to the 4 * AT chunks
    constexpr int AT = 32;                           // chunks whose totals are read together
    // (the chunk that nothing comes behind has no totals: its place holds anything, and what is made of it goes nowhere)
    for (int k = 0; k < n_chunk; k += 4 * AT) {
        float H[AT], sd[AT], h = 0.f, sum = 0.f;
#pragma unroll
        for (int j = 0; j < AT; ++j) {
            const int o = min(k + w * AT + j, n_chunk - 1), c = BWD ? n_chunk - 1 - o : o;
            H[j] = totals[(size_t)c * ND + i];
            sd[j] = sums[(size_t)c * D + ch];
        }
        // (what is worked out for places behind the last chunk goes nowhere; were it left out, the loads would wait in turn)
#pragma unroll
        for (int j = 0; j < AT; ++j) {
            h = carried(h, sd[j], half_A2, H[j]);
            sum += sd[j];                            // (the mark stays)
        }
        s_h[w][lane] = h;
        s_sum[w][lane] = sum;
        __syncthreads();
        h = base;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            if (v < w) h = carried(h, s_sum[v][lane], half_A2, s_h[v][lane]);
            base = carried(base, s_sum[v][lane], half_A2, s_h[v][lane]);
        }
#pragma unroll
        for (int j = 0; j < AT; ++j) {
            const int o = k + w * AT + j, c = BWD ? n_chunk - 1 - o : o;
            if (o < n_chunk && live) totals[(size_t)c * ND + i] = h;
            h = carried(h, sd[j], half_A2, H[j]);
        }
        __syncthreads();                             // (the sums have been read)
    }
}

enum { SCAN_TOTALS = 0, SCAN_OUT = 1, SCAN_SAVE = 2 };        // what a walk leaves: the chunks' totals, the output, only the saved states
constexpr int GT = 4;                                        // rows of a group: loaded together, one group ahead

// A group's input and output maps: each lane loads its share of the GT * 2N values, wherever they lie, and puts them into LDS as fp32, from
// where every lane reads those of a row at one address.  (Through the scalar cache each row waited for them, and a scalar operand halves an
// instruction's rate.)
template <typename IO, int N>
struct Maps {
    static constexpr int PER = GT * 2 * N / 64, LPR = 64 / GT;      // values of a lane, lanes of a row: the first half of them has B's
    static_assert(PER >= 1 && N % PER == 0, "");
    IO v[PER];
    static __device__ __forceinline__ bool has_c(int lane) { return lane & (LPR / 2); }
    __device__ __forceinline__ void load(const IO* Bm, const IO* Cm, long ldb, long ldc, int t, int last, int lane)
    {
        const long r = min(t + lane / LPR, last);
        const int k = lane % (LPR / 2) * PER;
        const IO* p = has_c(lane) ? Cm + r * ldc + k : Bm + r * ldb + k;
#pragma unroll
        for (int i = 0; i < PER; ++i) v[i] = p[i];
    }
    __device__ __forceinline__ void put(float (*to)[2 * N], int lane) const
    {
        float* p = &to[lane / LPR][lane % LPR * PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) p[i] = to_f(v[i]);
    }
};
__device__ __forceinline__ void wave_fence() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

template <typename IO, int N, int MODE>
__global__ __launch_bounds__(64) void selscan_fwd_kernel(ScanFwd a)
{
    __shared__ __align__(16) float s_bc[2][GT][2 * N];
    const ScanShape& s = a.s;
    const Rows& R = s.rows;
    const int lane = threadIdx.x;
    const int g = blockIdx.x / s.nb;
    const unsigned ch = g * s.Dg + min((int)(blockIdx.x % s.nb) * 64 + lane, s.Dg - 1);
    // (lanes behind the group's last channel do what that one's lane does, and leave the same values in the same places)
    const int c = blockIdx.y, t0 = c * s.chunk, t1 = min(t0 + s.chunk, R.T);
    const size_t ND = (size_t)N * s.D;

    float A2[N], h[N];
#pragma unroll
    for (int n = 0; n < N; ++n) { A2[n] = a.A[(size_t)n * s.D + ch] * kLog2e; h[n] = 0.f; }
    const float bias = a.dbias ? a.dbias[ch] : 0.f, skip = a.Dskip ? a.Dskip[ch] : 0.f;

    const bool gated = MODE == SCAN_OUT && a.Z != nullptr;
    const IO *Bm = (const IO*)a.Bm + (size_t)g * N, *Cm = (const IO*)a.Cm + (size_t)g * N;
    const unsigned och = ch * sizeof(IO);
    IO* Y = (IO*)a.Y + (size_t)t0 * s.D;                     // (of the row that comes next)
    RowWalk<IO> pu, pd, pz;
    pu.start(a.U, a.ldu, t0);
    pd.start(a.delta, a.ldd, t0);
    if (gated) pz.start(a.Z, a.ldz, t0);
    IO nu[GT], nd[GT], nz[GT];
    Maps<IO, N> maps;
    auto load = [&](int t) {
#pragma unroll
        for (int i = 0; i < GT; ++i) {
            const bool more = t + i < R.T - 1;
            nu[i] = pu.get(och);
            pu.next(more);
            nd[i] = pd.get(och);
            pd.next(more);
            if (gated) { nz[i] = pz.get(och); pz.next(more); }
        }
        if (MODE == SCAN_OUT || !maps.has_c(lane)) maps.load(Bm, Cm, a.ldb, a.ldc, t, R.T - 1, lane);
    };
    load(t0);                                                // (on their way while the sequence is looked for)
    int q = seq_of_wave(R, t0, lane);                        // the sequence the walk is in, and its rows
    if (q < 0) q = 0;
    int beg = q < R.n_seq ? seq_begin(R, q) : R.T, end = q < R.n_seq ? seq_end(R, q) : R.T;
    if (MODE != SCAN_TOTALS && c > 0 && beg < t0 && q < R.n_seq) {
        const float* H = a.totals + (size_t)c * ND + ch;
#pragma unroll
        for (int n = 0; n < N; ++n) h[n] = H[(size_t)n * s.D];
    }

    if (MODE == SCAN_OUT && R.clear) {                       // rows of no sequence
        const int first = R.n_seq > 0 ? seq_begin(R, 0) : 0, stop = R.n_seq > 0 ? seq_end(R, R.n_seq - 1) : 0;
        if (t0 < first || t1 > stop)
#pragma unroll 1
            for (int r = t0; r < t1; ++r)
                if (r < first || r >= stop) row_store((IO*)a.Y + (size_t)r * s.D, och, (IO)0.f);
    }

    // (a row's address is the same in all lanes: scalar base, 32-bit lane offset)
    float sum = 0.f;
    bool began = false;
    auto row = [&](const float* bc, float dl, float u, float gate) {
        const float du = dl * u;
        float y[2] = {skip * u, 0.f};
#pragma unroll
        for (int n = 0; n < N; ++n) {
            h[n] = fmaf(exp2_(dl * A2[n]), h[n], du * bc[n]);
            if (MODE == SCAN_OUT) y[n & 1] = fmaf(bc[N + n], h[n], y[n & 1]);
        }
        if (MODE == SCAN_TOTALS) sum += dl;
        if (MODE == SCAN_OUT) row_store(Y, och, from_f<IO>((y[0] + y[1]) * gate));
    };

    for (int t = t0; t < t1; t += GT) {
        float u[GT], dl[GT], gate[GT];
        float(*bc)[2 * N] = s_bc[(t / GT) & 1];
#pragma unroll
        for (int i = 0; i < GT; ++i) { u[i] = to_f(nu[i]); dl[i] = to_f(nd[i]) + bias; gate[i] = gated ? to_f(nz[i]) : 1.f; }
        if (MODE == SCAN_OUT || !maps.has_c(lane)) maps.put(bc, lane);
        wave_fence();
        if (t + GT < t1) load(t + GT);
        if (s.softplus)
#pragma unroll
            for (int i = 0; i < GT; ++i) dl[i] = softplus_(dl[i]);
        if (gated)
#pragma unroll
            for (int i = 0; i < GT; ++i) gate[i] *= sigmoid_(gate[i]);
        if (MODE != SCAN_TOTALS && a.saved && (t & (kSelscanTile - 1)) == 0) {
            float* to = a.saved + (size_t)(t / kSelscanTile) * ND;
#pragma unroll
            for (int n = 0; n < N; ++n) row_store(to + (size_t)n * s.D, ch * 4, h[n]);
        }
        if (beg < t && t + GT < end && t + GT <= t1) {       // no sequence begins or ends here
#pragma unroll
            for (int i = 0; i < GT; ++i) {
                row(bc[i], dl[i], u[i], gate[i]);
                Y += s.D;
                __builtin_amdgcn_sched_barrier(0);           // (or all rows' maps are read into registers first)
            }
            continue;
        }
#pragma unroll 1
        for (int i = 0; i < GT; ++i) {
            const int r = t + i;
            if (i > 0) Y += s.D;
            while (q < R.n_seq && end <= r) {
                ++q;
                if (q < R.n_seq) { beg = seq_begin(R, q); end = seq_end(R, q); }
            }
            if (r >= t1 || q >= R.n_seq || r < beg) continue;
            const int slot = a.S_in || a.S_out ? slot_of(R, q) : -1;
            if (r == beg) {
                began = true;
#pragma unroll
                for (int n = 0; n < N; ++n) h[n] = a.S_in && slot >= 0 ? a.S_in[(size_t)slot * ND + (size_t)n * s.D + ch] : 0.f;
            }
            float ui = u[0], di = dl[0], gi = gate[0];
#pragma unroll
            for (int j = 1; j < GT; ++j) if (i == j) { ui = u[j]; di = dl[j]; gi = gate[j]; }
            row(bc[i], di, ui, gi);
            if (MODE == SCAN_OUT && r == end - 1 && a.S_out && slot >= 0) {
                // (over the states that other workgroups of the sequence may still read: later, by selscan_finish_kernel)
                float* to = s.same_buffer && beg < t0 ? a.fin + (size_t)c * ND + ch : a.S_out + (size_t)slot * ND + ch;
#pragma unroll
                for (int n = 0; n < N; ++n) to[(size_t)n * s.D] = h[n];
            }
        }
        Y += s.D;
    }
    if (MODE == SCAN_TOTALS) {
        float* H = a.totals + (size_t)c * ND + ch;
#pragma unroll
        for (int n = 0; n < N; ++n) H[(size_t)n * s.D] = h[n];
        a.sums[(size_t)c * s.D + ch] = began ? reset_mark() : sum;
    }
}

// ---------------------------------------------------------------------------------------------------------------- gradient
struct ScanBwd {
    ScanShape s;
    const void *U, *delta, *Z, *dY, *Bm, *Cm;
    long ldu, ldd, ldz, lddy, ldb, ldc;
    const float *A, *Dskip, *dbias, *S_in, *dS_out, *saved;
    float *dS_in, *totals, *sums, *part_bc, *part_A, *part_D;
    void *dU, *ddelta, *dZ;
};

// What the rows of a chunk add to q in front of it (q itself, if a sequence ends in it), the walk going from the last row to the first.
template <typename IO, int N>
__global__ __launch_bounds__(64) void selscan_bwd_totals_kernel(ScanBwd a)
{
    __shared__ __align__(16) float s_bc[2][GT][2 * N];
    const ScanShape& s = a.s;
    const Rows& R = s.rows;
    const int lane = threadIdx.x;
    const int g = blockIdx.x / s.nb;
    const unsigned ch = g * s.Dg + min((int)(blockIdx.x % s.nb) * 64 + lane, s.Dg - 1);
    const int c = blockIdx.y + 1, t0 = c * s.chunk, t1 = min(t0 + s.chunk, R.T);       // (nothing is in front of the first chunk)
    const size_t ND = (size_t)N * s.D;

    float A2[N], q[N];
#pragma unroll
    for (int n = 0; n < N; ++n) { A2[n] = a.A[(size_t)n * s.D + ch] * kLog2e; q[n] = 0.f; }
    const float bias = a.dbias ? a.dbias[ch] : 0.f;
    const bool gated = a.Z != nullptr;
    const IO *Bm = (const IO*)a.Bm + (size_t)g * N, *Cm = (const IO*)a.Cm + (size_t)g * N;
    float sum = 0.f;
    bool ended = false;
    IO nd[GT], nz[GT], ny[GT];
    Maps<IO, N> maps;
    const unsigned och = ch * sizeof(IO);
    const int last = t0 + (t1 - 1 - t0) / GT * GT;
    RowWalk<IO> pd, py, pz;
    pd.start(a.delta, a.ldd, min(last + GT - 1, R.T - 1));
    py.start(a.dY, a.lddy, min(last + GT - 1, R.T - 1));
    if (gated) pz.start(a.Z, a.ldz, min(last + GT - 1, R.T - 1));
    auto load = [&](int t) {
#pragma unroll
        for (int i = GT - 1; i >= 0; --i) {
            const bool more = t + i < R.T && t + i > 0;
            nd[i] = pd.get(och);
            pd.back(more);
            ny[i] = py.get(och);
            py.back(more);
            if (gated) { nz[i] = pz.get(och); pz.back(more); }
        }
        if (maps.has_c(lane)) maps.load(Bm, Cm, a.ldb, a.ldc, t, R.T - 1, lane);
    };
    load(last);
    int sq = seq_of_wave(R, t1 - 1, lane), beg = 0, end = 0;
    if (sq >= R.n_seq) sq = R.n_seq - 1;
    if (sq >= 0) { beg = seq_begin(R, sq); end = seq_end(R, sq); }
    auto row = [&](const float* bc, float dl, float dy) {
#pragma unroll
        for (int n = 0; n < N; ++n) q[n] = exp2_(dl * A2[n]) * fmaf(bc[N + n], dy, q[n]);
        sum += dl;
    };
    for (int t = last; t >= t0; t -= GT) {
        float dl[GT], dy[GT];
        float(*bc)[2 * N] = s_bc[(t / GT) & 1];
#pragma unroll
        for (int i = 0; i < GT; ++i) { dl[i] = to_f(nd[i]) + bias; dy[i] = to_f(ny[i]); }
        if (gated)
#pragma unroll
            for (int i = 0; i < GT; ++i) dy[i] *= to_f(nz[i]) * sigmoid_(to_f(nz[i]));
        if (maps.has_c(lane)) maps.put(bc, lane);
        wave_fence();
        if (t > t0) load(t - GT);
        if (s.softplus)
#pragma unroll
            for (int i = 0; i < GT; ++i) dl[i] = softplus_(dl[i]);
        if (sq >= 0 && beg <= t && t + GT < end && t + GT <= t1) {
#pragma unroll
            for (int i = GT - 1; i >= 0; --i) {
                row(bc[i], dl[i], dy[i]);
                __builtin_amdgcn_sched_barrier(0);
            }
            continue;
        }
#pragma unroll 1
        for (int i = GT - 1; i >= 0; --i) {
            const int r = t + i;
            while (sq >= 0 && beg > r) {
                --sq;
                if (sq >= 0) { beg = seq_begin(R, sq); end = seq_end(R, sq); }
            }
            if (r >= t1 || sq < 0 || r >= end) continue;
            if (r == end - 1) {
                ended = true;
                const int slot = slot_of(R, sq);
#pragma unroll
                for (int n = 0; n < N; ++n) q[n] = a.dS_out && slot >= 0 ? a.dS_out[(size_t)slot * ND + (size_t)n * s.D + ch] : 0.f;
            }
            float di = dl[0], yi = dy[0];
#pragma unroll
            for (int j = 1; j < GT; ++j) if (i == j) { di = dl[j]; yi = dy[j]; }
            row(bc[i], di, yi);
        }
    }
    float* Q = a.totals + (size_t)c * ND + ch;
#pragma unroll
    for (int n = 0; n < N; ++n) Q[(size_t)n * s.D] = q[n];
    a.sums[(size_t)c * s.D + ch] = ended ? reset_mark() : sum;
}

// Sums over the wave's lanes of many values at once: a step adds two lanes' worth and deals two values out to the two, so the values
// get fewer as they get more complete.  Within rows of 16 lanes by DPP, across them by swaps (which take three times as long and come last).
template <int CTRL>
__device__ __forceinline__ float dpp(float x)
{
    return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, 0xf, 0xf, true));
}
template <int CTRL>
__device__ __forceinline__ float deal(float x, float y, bool second)       // x's partial sums to the lanes that are not `second`, y's to those that are
{
    const float keep = second ? y : x, send = second ? x : y;
    return keep + dpp<CTRL>(send);
}
constexpr int ROR8 = 0x128, HALF_MIRROR = 0x141, XOR2 = 0x4E, XOR1 = 0xB1;
__device__ __forceinline__ float deal32(float x, float y)      // x's to the lower half of the lanes, y's to the upper
{
    u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(y), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float deal16(float x, float y)      // x's to the even rows of 16 lanes, y's to the odd ones
{
    u32x2 r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(y), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// Eight values' sums over rows of 16 lanes but for lanes that differ in bit 0: lane l has that of value 4 (bit 3) + 2 (bit 2) + (bit 1).
__device__ __forceinline__ float sum8(const float (&v)[8], int lane)
{
    float r[4], w[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = deal<ROR8>(v[i], v[i + 4], lane & 8);
#pragma unroll
    for (int i = 0; i < 2; ++i) w[i] = deal<HALF_MIRROR>(r[i], r[i + 2], lane & 4);
    return deal<XOR2>(w[0], w[1], lane & 2);
}

constexpr int NPW = 4, TB = kSelscanTile;         // states of a wave, rows of a tile

// A workgroup walks its chunk from the last tile to the first.  Wave w has states 4w .. 4w+3 of the same 64 channels: a tile's
// decays and states then fit its registers.  The step sizes and the like of a tile are worked out once, by all waves, and shared.
// Tiles of 8 rows leave room for three waves per SIMD, tiles of 16 for two: 1310 us against 1440 (65536 rows, 1536 channels, 16 states).
// (With 32 states a workgroup is eight waves of 167 registers, of which a CU holds one: two waves per SIMD.  With 8 and 16 states three waves
// are had at the price of 23 to 26 and 2 to 4 spilled registers.)
template <typename IO, int N>
__global__ __launch_bounds__(N / NPW * 64, 3) void selscan_bwd_kernel(ScanBwd a)
{
    constexpr int W = N / NPW, PER = TB / W;                       // waves; rows of a tile that a thread looks after
    static_assert(TB % W == 0, "");
    __shared__ float s_dl[TB][64], s_x[TB][64], s_dy[TB][64], s_part[W][3][TB][64];
    __shared__ __align__(16) float s_bc[TB][2 * N];
    const ScanShape& s = a.s;
    const Rows& R = s.rows;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = blockIdx.x / s.nb, b = blockIdx.x % s.nb, in_group = b * 64 + lane;
    const bool live = in_group < s.Dg;
    const unsigned ch = g * s.Dg + min(in_group, s.Dg - 1);
    const int c = blockIdx.y, t0 = c * s.chunk, t1 = min(t0 + s.chunk, R.T);
    const size_t ND = (size_t)N * s.D, first = (size_t)(w * NPW) * s.D, mine = first + ch;      // of a state's N * D floats, this wave's first and this lane's

    float A[NPW], A2[NPW], q[NPW], dA[NPW];
#pragma unroll
    for (int n = 0; n < NPW; ++n) {
        A[n] = a.A[mine + (size_t)n * s.D];
        A2[n] = A[n] * kLog2e;
        q[n] = dA[n] = 0.f;
    }
    const float bias = a.dbias ? a.dbias[ch] : 0.f, skip = a.Dskip ? a.Dskip[ch] : 0.f;
    const IO *U = (const IO*)a.U, *De = (const IO*)a.delta, *dY = (const IO*)a.dY, *Z = (const IO*)a.Z;
    IO *dU = (IO*)a.dU, *dDe = (IO*)a.ddelta, *dZ = (IO*)a.dZ;

    // a thread's share of the tile's TB * 2N map values
    constexpr int MV = TB * 2 * N / (W * 64);
    const int mt = threadIdx.x * MV / (2 * N), mk = threadIdx.x * MV % (2 * N);
    const IO* M = mk < N ? (const IO*)a.Bm + (size_t)g * N + mk : (const IO*)a.Cm + (size_t)g * N + mk - N;
    const long ldm = mk < N ? a.ldb : a.ldc;
    IO nu[PER], nd[PER], nz[PER], ny[PER], nm[MV];
    float nh[NPW];
    const unsigned och = ch * sizeof(IO);
    auto load = [&](int t) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const long r = min(t + w + i * W, R.T - 1);
            nu[i] = row_load(U + r * a.ldu, och);
            nd[i] = row_load(De + r * a.ldd, och);
            ny[i] = row_load(dY + r * a.lddy, och);
            if (Z) nz[i] = row_load(Z + r * a.ldz, och);
        }
        const IO* m = M + min(t + mt, R.T - 1) * ldm;
#pragma unroll
        for (int k = 0; k < MV; ++k) nm[k] = m[k];
        const float* from = a.saved + (size_t)(t / TB) * ND + first;
#pragma unroll
        for (int n = 0; n < NPW; ++n) nh[n] = row_load(from + (size_t)n * s.D, ch * 4);
    };
    float dD = 0.f, dbias = 0.f;
    // where sum8()'s value of this lane goes, of a row's 2N
    float* part = a.part_bc + ((size_t)b * R.T * s.G + g) * (2 * N);
    const int at = ((lane >> 3) & 1) * N + w * NPW + ((lane >> 2) & 1) * 2 + ((lane >> 1) & 1);
    const int last = t0 + (t1 - 1 - t0) / TB * TB;
    load(last);
    int sq = seq_of_wave(R, t1 - 1, lane), beg = 0, end = 0;
    const bool inside = sq >= 0 && sq < R.n_seq;
    if (sq >= R.n_seq) sq = R.n_seq - 1;
    if (sq >= 0) { beg = seq_begin(R, sq); end = seq_end(R, sq); }
    if (inside && end > t1) {                     // the sequence goes on in the chunks behind
        const float* Q = a.totals + (size_t)c * ND + mine;
#pragma unroll
        for (int n = 0; n < NPW; ++n) q[n] = Q[(size_t)n * s.D];
    }

    for (int t = last; t >= t0; t -= TB) {
        // of a row that the thread looks after: u, the step size's slope, dout silu(z), dout silu'(z)
        float u[PER], slope[PER], dy[PER], dz[PER], h0[NPW], tA[NPW];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            // (lanes behind the group's last channel: nothing that reaches the sums over channels)
            u[i] = live ? to_f(nu[i]) : 0.f;
            dy[i] = live ? to_f(ny[i]) : 0.f;
            float dl = to_f(nd[i]) + bias;
            slope[i] = 1.f;
            if (s.softplus) dl = softplus_(dl, &slope[i]);
            if (Z) {
                const float z = to_f(nz[i]), sg = sigmoid_(z), si = z * sg;
                dz[i] = dy[i] * fmaf(si, 1.f - sg, sg);
                dy[i] *= si;
            }
            const int k = w + i * W;
            s_dl[k][lane] = dl;
            s_x[k][lane] = dl * u[i];
            s_dy[k][lane] = dy[i];
        }
#pragma unroll
        for (int k = 0; k < MV; ++k) s_bc[mt][mk + k] = to_f(nm[k]);
#pragma unroll
        for (int n = 0; n < NPW; ++n) { h0[n] = nh[n]; tA[n] = 0.f; }
        if (t > t0) load(t - TB);
        __syncthreads();
        const bool whole = sq >= 0 && beg < t && t + TB < end && t + TB <= t1;
        auto state_in_front = [&](int sequence, float (&to)[NPW]) {
            const int slot = a.S_in ? slot_of(R, sequence) : -1;
#pragma unroll
            for (int n = 0; n < NPW; ++n) to[n] = slot >= 0 ? a.S_in[(size_t)slot * ND + mine + (size_t)n * s.D] : 0.f;
        };
        auto tile = [&](auto is_whole) {
            constexpr bool WHOLE = decltype(is_whole)::value;
            // forward: the tile's states and decays
            float h[TB][NPW], dec[TB][NPW];
            int fq = 0, fb = 0;                    // (the sequence that the tile's first rows are in)
            if (!WHOLE) {
                fq = seq_of(R, t);
                if (fq < 0) fq = 0;
                fb = fq < R.n_seq ? seq_begin(R, fq) : R.T;
            }
#pragma unroll
            for (int i = 0; i < TB; ++i) {
                const int r = t + i;
                const float* Bt = &s_bc[i][w * NPW];
                const float d = s_dl[i][lane], xu = s_x[i][lane];
                float before[NPW];
#pragma unroll
                for (int n = 0; n < NPW; ++n) before[n] = i == 0 ? h0[n] : h[i > 0 ? i - 1 : 0][n];
                if (!WHOLE) {
                    while (fq < R.n_seq && seq_end(R, fq) <= r) {
                        ++fq;
                        fb = fq < R.n_seq ? seq_begin(R, fq) : R.T;
                    }
                    if (fq < R.n_seq && r == fb) state_in_front(fq, before);
                }
#pragma unroll
                for (int n = 0; n < NPW; ++n) {
                    dec[i][n] = exp2_(d * A2[n]);
                    h[i][n] = fmaf(dec[i][n], before[n], xu * Bt[n]);
                }
                if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
            }
            // and back
            float odd = 0.f, pair1 = 0.f, half1 = 0.f;
#pragma unroll
            for (int i = TB - 1; i >= 0; --i) {
                const int r = t + i;
                bool on = true;
                if (!WHOLE) {
                    while (sq >= 0 && beg > r) {
                        --sq;
                        if (sq >= 0) { beg = seq_begin(R, sq); end = seq_end(R, sq); }
                    }
                    on = r < t1 && sq >= 0 && r < end;
                    if (on && r == end - 1) {
                        const int slot = a.dS_out ? slot_of(R, sq) : -1;
#pragma unroll
                        for (int n = 0; n < NPW; ++n) q[n] = slot >= 0 ? a.dS_out[(size_t)slot * ND + mine + (size_t)n * s.D] : 0.f;
                    }
                }
                float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                if (on) {
                    const float *Bt = &s_bc[i][w * NPW], *Ct = Bt + N;
                    const float d = s_dl[i][lane], xu = s_x[i][lane], dy = s_dy[i][lane];
                    float y = 0.f, s1 = 0.f, s2 = 0.f, before[NPW];
#pragma unroll
                    for (int n = 0; n < NPW; ++n) before[n] = i == 0 ? h0[n] : h[i > 0 ? i - 1 : 0][n];
                    if (!WHOLE && r == beg) state_in_front(sq, before);
#pragma unroll
                    for (int n = 0; n < NPW; ++n) {
                        const float hh = h[i][n], gg = fmaf(Ct[n], dy, q[n]);
                        q[n] = dec[i][n] * gg;
                        const float gp = q[n] * before[n];
                        y = fmaf(Ct[n], hh, y);
                        s1 = fmaf(gg, Bt[n], s1);
                        s2 = fmaf(A[n], gp, s2);
                        tA[n] = fmaf(d, gp, tA[n]);
                        v[n] = gg * xu;
                        v[4 + n] = dy * hh;
                    }
                    s_part[w][0][i][lane] = y;
                    s_part[w][1][i][lane] = s1;
                    s_part[w][2][i][lane] = s2;
                    if (!WHOLE && r == beg && a.dS_in && live) {
                        const int slot = slot_of(R, sq);
                        if (slot >= 0) {
#pragma unroll
                            for (int n = 0; n < NPW; ++n) a.dS_in[(size_t)slot * ND + mine + (size_t)n * s.D] = q[n];
                        }
                    }
                }
                const float x8 = sum8(v, lane);
                if (i & 1) {
                    odd = x8;
                } else {
                    const float pair = deal<XOR1>(x8, odd, lane & 1);
                    if (i % 4 == 2) {
                        pair1 = pair;
                    } else if (i % 8 == 4) {
                        half1 = deal32(pair, pair1);
                    } else {
                        const float sum = deal16(deal32(pair, pair1), half1);
                        const int k = t + i + 4 * ((lane >> 4) & 1) + 2 * (lane >> 5) + (lane & 1);
                        if (k < t1) (part + ((size_t)(t + i) * s.G) * (2 * N))[at + (k - t - i) * s.G * 2 * N] = sum;
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        };
        if (whole) tile(std::true_type{});
        else tile(std::false_type{});
#pragma unroll
        for (int n = 0; n < NPW; ++n) dA[n] += tA[n];          // (a tile's sum first: thousands of rows in one sum would lose digits)
        __syncthreads();
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int k = w + i * W, r = t + k;
            if (!whole) {
                const int sr = r < t1 ? seq_of(R, r) : -1;
                if (sr < 0 || sr >= R.n_seq) continue;
            }
            float y = 0.f, s1 = 0.f, s2 = 0.f;
#pragma unroll
            for (int j = 0; j < W; ++j) { y += s_part[j][0][k][lane]; s1 += s_part[j][1][k][lane]; s2 += s_part[j][2][k][lane]; }
            if (Z && live) row_store(dZ + (size_t)r * s.D, och, from_f<IO>(dz[i] * fmaf(skip, u[i], y)));
            const float dd = fmaf(u[i], s1, s2) * slope[i];
            dD = fmaf(dy[i], u[i], dD);
            dbias += dd;
            if (live) {
                row_store(dU + (size_t)r * s.D, och, from_f<IO>(fmaf(s_dl[k][lane], s1, skip * dy[i])));
                row_store(dDe + (size_t)r * s.D, och, from_f<IO>(dd));
            }
        }
        // (the next tile's step sizes are written over this one's only after every wave has passed the barrier above)
    }
    __syncthreads();
    if (live) {
#pragma unroll
        for (int n = 0; n < NPW; ++n) a.part_A[(size_t)c * ND + mine + (size_t)n * s.D] = dA[n];
    }
    s_part[w][0][0][lane] = dD;
    s_part[w][1][0][lane] = dbias;
    __syncthreads();
    if (w == 0 && live) {
        float x = 0.f, y = 0.f;
#pragma unroll
        for (int j = 0; j < W; ++j) { x += s_part[j][0][0][lane]; y += s_part[j][1][0][lane]; }
        a.part_D[(size_t)(2 * c) * s.D + ch] = x;
        a.part_D[(size_t)(2 * c + 1) * s.D + ch] = y;
    }
}

// The waves' sums over their channels, added up and rounded once; rows of no sequence are left as they are.  R.clear: all gradients of these are
// zeroed here (in the walk that would be 1 % of its time, whether there are any or not).
template <typename IO>
__global__ __launch_bounds__(256) void selscan_bc_kernel(Rows R, const float* __restrict__ part, int nb, int N, int G, IO* __restrict__ dB,
                                                        IO* __restrict__ dC, int D, IO* __restrict__ dU, IO* __restrict__ ddelta,
                                                        IO* __restrict__ dZ)
{
    const long n = (long)R.T * G * 2 * N;
    const int begin = R.n_seq > 0 ? seq_begin(R, 0) : 0, end = R.n_seq > 0 ? seq_end(R, R.n_seq - 1) : 0;
    const long first = (long)begin * G * 2 * N, stop = (long)end * G * 2 * N;
    if (R.clear && (begin > 0 || end < R.T)) {
        const long maps = (long)G * N;
        for (int r = blockIdx.x; r < R.T; r += gridDim.x) {
            if (r >= begin && r < end) continue;
            for (long i = threadIdx.x; i < D; i += 256) {
                dU[(size_t)r * D + i] = ddelta[(size_t)r * D + i] = (IO)0.f;
                if (dZ) dZ[(size_t)r * D + i] = (IO)0.f;
            }
            for (long i = threadIdx.x; i < maps; i += 256) dB[(size_t)r * maps + i] = dC[(size_t)r * maps + i] = (IO)0.f;
        }
    }
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long)gridDim.x * 256) {
        if (i < first || i >= stop) continue;
        float x = 0.f;
        for (int b = 0; b < nb; ++b) x += part[(size_t)b * n + i];
        const int k = (int)(i % (2 * N));
        const long tg = i / (2 * N);
        if (k < N) dB[tg * N + k] = from_f<IO>(x);
        else dC[tg * N + k - N] = from_f<IO>(x);
    }
}

// The chunks' sums of the parameters' gradients: rows 0 .. N-1 are dA's, N dD's and N+1 the bias's.  Sixteen waves share the chunks.
__global__ __launch_bounds__(1024) void selscan_params_kernel(const float* __restrict__ part_A, const float* __restrict__ part_D, int n_chunk,
                                                             int N, int D, float* dA, float* dD, float* dbias)
{
    __shared__ float s_sum[16][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, i = blockIdx.x * 64 + lane, n = blockIdx.y;
    float* to = n < N ? dA + (size_t)n * D : n == N ? dD : dbias;
    if (to == nullptr) return;
    const float* from = (n < N ? part_A + (size_t)n * D : part_D + (size_t)(n - N) * D) + min(i, D - 1);
    const size_t step = n < N ? (size_t)N * D : (size_t)2 * D;
    float x = 0.f;
    for (int c = w; c < n_chunk; c += 16) x += from[(size_t)c * step];
    s_sum[w][lane] = x;
    __syncthreads();
    if (w != 0 || i >= D) return;
    x = 0.f;
#pragma unroll
    for (int j = 0; j < 16; ++j) x += s_sum[j][lane];
    to[i] = x;
}

// ------------------------------------------------------------------------------------------------------------ single tokens
// A wave has 64 channels of `each` requests: what a channel has once (16 decays, 4 KB a wave, as many bytes as its state) is read once.  A request's
// loads all come before its stores.  256 requests of 1536 channels, 16 states: 11.3 us, 4.7 TB/s of states read and written; one request 5.5.
template <typename IO, int N>
__global__ __launch_bounds__(64) void selscan_step_kernel(SelscanArgs a, int each)
{
    const int nb = (a.D + 63) / 64, Dg = a.D / a.G, ch = blockIdx.x % nb * 64 + threadIdx.x;
    const int r0 = blockIdx.x / nb * each, r1 = min(r0 + each, a.rows.T);
    if (ch >= a.D) return;
    const int g = ch / Dg;
    const size_t ND = (size_t)N * a.D;
    float A2[N];
#pragma unroll
    for (int n = 0; n < N; ++n) A2[n] = a.A[(size_t)n * a.D + ch] * kLog2e;
    const float bias = a.delta_bias ? a.delta_bias[ch] : 0.f, skip = a.Dskip ? a.Dskip[ch] : 0.f;
    if (a.rows.clear)
        for (int r = r0; r < r1; ++r)
            if (slot_of(a.rows, r) < 0) ((IO*)a.Y)[(size_t)r * a.D + ch] = (IO)0.f;
    for (int r = r0; r < r1; ++r) {
        const int slot = slot_of(a.rows, r);
        if (slot < 0) continue;
        float* S = a.S_out + (size_t)slot * ND + ch;
        const IO *Bm = (const IO*)a.Bm + (size_t)r * a.ldb + (size_t)g * N, *Cm = (const IO*)a.Cm + (size_t)r * a.ldc + (size_t)g * N;
        float h[N];
        IO b[N], c[N];
#pragma unroll
        for (int n = 0; n < N; ++n) h[n] = S[(size_t)n * a.D];
#pragma unroll
        for (int n = 0; n < N; ++n) { b[n] = Bm[n]; c[n] = Cm[n]; }
        const float u = to_f(((const IO*)a.U)[(size_t)r * a.ldu + ch]);
        const float z = a.Z ? to_f(((const IO*)a.Z)[(size_t)r * a.ldz + ch]) : 0.f;
        float dl = to_f(((const IO*)a.delta)[(size_t)r * a.ldd + ch]) + bias;
        if (a.softplus) dl = softplus_(dl);
        float y = skip * u;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            h[n] = fmaf(exp2_(dl * A2[n]), h[n], dl * u * to_f(b[n]));
            y = fmaf(to_f(c[n]), h[n], y);
        }
#pragma unroll
        for (int n = 0; n < N; ++n) S[(size_t)n * a.D] = h[n];
        if (a.Z) y *= z * sigmoid_(z);
        ((IO*)a.Y)[(size_t)r * a.D + ch] = from_f<IO>(y);
    }
}

// -------------------------------------------------------------------------------------------------------------------- host
bool selscan_states_ok(int N) { return N == 8 || N == 16 || N == 32; }

static int waves_per_group(int D, int G) { return (D / G + 63) / 64; }

// Chunks of whole tiles.  The more there are, the more waves, and the more states to leave, to carry and to begin with (as good as kExtra
// rows each); and what counts is the fullest SIMD.  A kernel: `units`, its workgroups that bring every SIMD as many waves as one brings its
// own; `slots`, how often that fits; `weight`, what its row costs.  kRate: what so many waves issue, of what four do; kUneven: how
// much fuller the fullest SIMD is.
struct ChunkCost { int units, slots; double weight; };
constexpr int kLeastChunk = 24, kExtra = 8;
constexpr double kRate[5] = {1, 0.45, 0.82, 0.93, 1}, kUneven = 0.7;
static void cut_rows(int T, long groups, const ChunkCost (&kernels)[2], int* chunk, int* n_chunk)
{
    double least = 0;
    for (int i = 1; i <= 24; ++i) {
        long n = (long)i * kernels[0].units / groups;
        n = n < 1 ? 1 : n > 1024 ? 1024 : n;
        long len = ((long)T + n - 1) / n;
        len = (len + kSelscanTile - 1) / kSelscanTile * kSelscanTile;
        if (len < kLeastChunk) len = kLeastChunk;
        n = ((long)T + len - 1) / len;
        double cost = 0;
        for (const ChunkCost& k : kernels) {
            const long all = (n * groups + k.units - 1) / k.units;
            cost += k.weight * (double)(len + kExtra) * ((double)all + kUneven) / kRate[all < k.slots ? all : k.slots];
        }
        if (i > 1 && cost >= least) continue;
        least = cost;
        *chunk = (int)len;
        *n_chunk = (int)n;
    }
}

static SelscanPlan plan_of(int T, int D, int N, int G, bool is_bwd, bool has_saved)
{
    SelscanPlan p{};
    const long groups = (long)G * waves_per_group(D, G);
    const int slots = N == 32 ? 3 : 4;
    const ChunkCost forward[2] = {{1024, slots, 1.0}, {1024, slots, 1.2}}, backward[2] = {{N == 32 ? 256 : 1024 / (N / NPW), N == 32 ? 1 : 3, 1.0}, {1024, slots, 1.15}};
    cut_rows(T, groups, is_bwd ? backward : forward, &p.chunk, &p.n_chunk);
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += (bytes + 255) & ~(size_t)255; return here; };
    const size_t ND = (size_t)N * D * sizeof(float);
    p.totals = take(ND * p.n_chunk);
    p.sums = take((size_t)p.n_chunk * D * sizeof(float));
    if (!is_bwd) p.fin = take(ND * p.n_chunk);
    if (is_bwd) {
        p.part_bc = take((size_t)waves_per_group(D, G) * T * G * 2 * N * sizeof(float));
        p.part_A = take(ND * p.n_chunk);
        p.part_D = take((size_t)2 * p.n_chunk * D * sizeof(float));
        if (!has_saved) p.saved = take(((size_t)T + kSelscanTile - 1) / kSelscanTile * ND);
    }
    p.bytes = at;
    return p;
}

SelscanPlan make_selscan_plan(int T, int D, int N, int G, bool is_bwd, bool has_saved)
{
    if (T <= 0) return SelscanPlan{};
    SelscanPlan p = plan_of(T, D, N, G, is_bwd, has_saved);
    // (the states in front of the tiles are worked out by the forward's walk, with its chunks, before the scratch has anything else in it)
    if (is_bwd && !has_saved) {
        const SelscanPlan f = plan_of(T, D, N, G, false, false);
        p.fin = p.bytes;
        p.bytes += f.bytes;
    }
    return p;
}

static ScanShape shape_of(const SelscanArgs& a, int chunk, int n_chunk)
{
    ScanShape s{};
    s.rows = a.rows;
    s.D = a.D; s.N = a.N; s.G = a.G;
    s.Dg = a.D / a.G;
    s.nb = waves_per_group(a.D, a.G);
    s.chunk = chunk; s.n_chunk = n_chunk; s.softplus = a.softplus;
    return s;
}

// Whether there may be sequences without rows whose state behind them is not the one in front already; with one chunk a kernel of its own
// hands them on, else the carries' does.
static bool to_pass_on(const SelscanArgs& a, const float* from, const float* to)
{
    return to != nullptr && to != from && a.rows.n_seq > 0 && (a.rows.cu != nullptr || a.rows.T == 0);
}
static void pass_on(const SelscanArgs& a, const float* from, float* to, int n_chunk, hipStream_t st)
{
    if (n_chunk > 1 || !to_pass_on(a, from, to)) return;
    hipLaunchKernelGGL(selscan_empty_kernel, dim3(a.rows.n_seq < 256 ? a.rows.n_seq : 256), dim3(256), 0, st, a.rows, from, to, (long)a.N * a.D);
}

template <bool BWD>
static void carry(const SelscanArgs& a, float* totals, const float* sums, int n_chunk, const float* from, float* to, hipStream_t st)
{
    const long ND = (long)a.N * a.D;
    const int groups = (int)((ND + 63) / 64), more = to_pass_on(a, from, to) ? (a.rows.n_seq < 256 ? a.rows.n_seq : 256) : 0;
    hipLaunchKernelGGL(selscan_carry_kernel<BWD>, dim3(groups + more), dim3(256), 0, st, a.A, totals, sums, n_chunk, a.D, ND, groups, a.rows, from,
                       to);
}

static ScanFwd fwd_of(const SelscanArgs& a, const SelscanPlan& p, char* ws)
{
    ScanFwd f{};
    f.s = shape_of(a, p.chunk, p.n_chunk);
    f.U = a.U; f.delta = a.delta; f.Z = a.Z;
    f.ldu = a.ldu; f.ldd = a.ldd; f.ldz = a.ldz;
    f.Bm = a.Bm; f.Cm = a.Cm; f.ldb = a.ldb; f.ldc = a.ldc;
    f.A = a.A; f.Dskip = a.Dskip; f.dbias = a.delta_bias;
    f.S_in = a.S_in; f.S_out = a.S_out; f.saved = a.saved;
    f.totals = (float*)(ws + p.totals); f.sums = (float*)(ws + p.sums); f.fin = (float*)(ws + p.fin);
    f.Y = a.Y;
    f.s.same_buffer = a.S_out != nullptr && a.S_out == a.S_in && p.n_chunk > 1;
    return f;
}

template <typename IO, int N>
static void walk(const SelscanArgs& a, const ScanFwd& f, bool out, hipStream_t st)
{
    const unsigned gx = (unsigned)(f.s.G * f.s.nb);
    if (f.s.n_chunk > 1) {
        hipLaunchKernelGGL((selscan_fwd_kernel<IO, N, SCAN_TOTALS>), dim3(gx, f.s.n_chunk - 1), dim3(64), 0, st, f);
        carry<false>(a, f.totals, f.sums, f.s.n_chunk, f.S_in, f.S_out, st);
    }
    if (out) hipLaunchKernelGGL((selscan_fwd_kernel<IO, N, SCAN_OUT>), dim3(gx, f.s.n_chunk), dim3(64), 0, st, f);
    else hipLaunchKernelGGL((selscan_fwd_kernel<IO, N, SCAN_SAVE>), dim3(gx, f.s.n_chunk), dim3(64), 0, st, f);
}

template <typename IO, int N>
static hipError_t fwd(const SelscanArgs& a, const SelscanPlan& p, char* ws, hipStream_t st)
{
    ProfScope prof(KID_SELSCAN, st);
    pass_on(a, a.S_in, a.S_out, p.n_chunk, st);
    if (a.rows.T > 0) {
        const ScanFwd f = fwd_of(a, p, ws);
        walk<IO, N>(a, f, true, st);
        if (f.s.same_buffer)
            hipLaunchKernelGGL(selscan_finish_kernel, dim3((unsigned)(((long)N * a.D + 255) / 256), p.n_chunk), dim3(256), 0, st, f.s,
                               f.fin, a.S_out);
    }
    return hipGetLastError();
}

template <typename IO, int N>
static hipError_t bwd(const SelscanArgs& a, const SelscanPlan& p, char* ws, hipStream_t st)
{
    ProfScope prof(KID_SELSCAN_BWD, st);
    pass_on(a, a.dS_out, a.dS_in, p.n_chunk, st);
    ScanBwd b{};
    b.saved = a.saved;
    if (a.saved == nullptr && a.rows.T > 0) {
        SelscanArgs again = a;
        again.saved = (float*)(ws + p.saved);
        again.S_out = nullptr;
        walk<IO, N>(again, fwd_of(again, plan_of(a.rows.T, a.D, a.N, a.G, false, false), ws + p.fin), false, st);
        b.saved = again.saved;
    }
    b.s = shape_of(a, p.chunk, p.n_chunk);
    b.U = a.U; b.delta = a.delta; b.Z = a.Z; b.dY = a.dY; b.Bm = a.Bm; b.Cm = a.Cm;
    b.ldu = a.ldu; b.ldd = a.ldd; b.ldz = a.ldz; b.lddy = a.lddy; b.ldb = a.ldb; b.ldc = a.ldc;
    b.A = a.A; b.Dskip = a.Dskip; b.dbias = a.delta_bias; b.S_in = a.S_in; b.dS_out = a.dS_out; b.dS_in = a.dS_in;
    b.totals = (float*)(ws + p.totals); b.sums = (float*)(ws + p.sums);
    b.part_bc = (float*)(ws + p.part_bc); b.part_A = (float*)(ws + p.part_A); b.part_D = (float*)(ws + p.part_D);
    b.dU = a.dU; b.ddelta = a.ddelta; b.dZ = a.dZ;
    const unsigned gx = (unsigned)(b.s.G * b.s.nb);
    if (p.n_chunk > 1) {
        hipLaunchKernelGGL((selscan_bwd_totals_kernel<IO, N>), dim3(gx, p.n_chunk - 1), dim3(64), 0, st, b);
        carry<true>(a, b.totals, b.sums, p.n_chunk, a.dS_out, a.dS_in, st);
    }
    if (a.rows.T > 0) {
        hipLaunchKernelGGL((selscan_bwd_kernel<IO, N>), dim3(gx, p.n_chunk), dim3(N / NPW * 64), 0, st, b);
        const long n = (long)a.rows.T * a.G * 2 * N;
        long blocks = (n + 255) / 256;
        if (blocks > 8192) blocks = 8192;
        hipLaunchKernelGGL(selscan_bc_kernel<IO>, dim3((unsigned)blocks), dim3(256), 0, st, a.rows, b.part_bc, b.s.nb, N, a.G, (IO*)a.dB,
                           (IO*)a.dC, a.D, (IO*)a.dU, (IO*)a.ddelta, a.Z ? (IO*)a.dZ : nullptr);
    }
    hipLaunchKernelGGL(selscan_params_kernel, dim3((unsigned)((a.D + 63) / 64), N + 2), dim3(1024), 0, st, b.part_A, b.part_D, p.n_chunk, N,
                       a.D, a.dA, a.dDskip, a.dbias);
    return hipGetLastError();
}

#define CHELA_SCAN(F, ...)                                                                                            \
    if (dtype == 0) switch (a.N) {                                                                                    \
        case 8: return F<bf16, 8>(__VA_ARGS__);                                                                       \
        case 16: return F<bf16, 16>(__VA_ARGS__);                                                                     \
        case 32: return F<bf16, 32>(__VA_ARGS__);                                                                     \
    } else switch (a.N) {                                                                                             \
        case 8: return F<float, 8>(__VA_ARGS__);                                                                      \
        case 16: return F<float, 16>(__VA_ARGS__);                                                                    \
        case 32: return F<float, 32>(__VA_ARGS__);                                                                    \
    }                                                                                                                 \
    return hipErrorInvalidValue;

hipError_t launch_selscan_fwd(const SelscanArgs& a, const SelscanPlan& p, char* ws, int dtype, hipStream_t st) { CHELA_SCAN(fwd, a, p, ws, st) }
hipError_t launch_selscan_bwd(const SelscanArgs& a, const SelscanPlan& p, char* ws, int dtype, hipStream_t st) { CHELA_SCAN(bwd, a, p, ws, st) }

template <typename IO, int N>
static hipError_t step(const SelscanArgs& a, hipStream_t st)
{
    ProfScope prof(KID_SELSCAN_STEP, st);
    const long nb = (a.D + 63) / 64, R = a.rows.T;
    // (256 requests, 1536 channels, for 1, 2, 3 a wave: 12.3, 11.2, 11.9 us; below four waves per SIMD one)
    const int each = nb * R >= 4096 ? 2 : 1;
    hipLaunchKernelGGL((selscan_step_kernel<IO, N>), dim3((unsigned)(nb * ((R + each - 1) / each))), dim3(64), 0, st, a, each);
    return hipGetLastError();
}
hipError_t launch_selscan_step(const SelscanArgs& a, int dtype, hipStream_t st) { CHELA_SCAN(step, a, st) }
#undef CHELA_SCAN

}  // namespace chela
