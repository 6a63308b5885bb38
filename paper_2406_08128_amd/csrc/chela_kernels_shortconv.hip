// Short causal convolution on [tokens, channels] rows, gfx950: sequences, gradient, single tokens.
//
//     u_t = bias + sum_{j<m} w[j] x_{t-j},  y_t = silu(u_t) or u_t;   x in front of a sequence: its state (the last m - 1 inputs), or 0.
// Gradient, with du_t = dy_t silu'(u_t) (u_t is worked out again):
//     dx_t = sum_j w[j] du_{t+j} (rows of the same sequence; the last m - 1 take d(state behind) too, and the state in front is a row like
//     the others),  dw[j] = sum_t du_t x_{t-j},  dbias = sum_t du_t.
//
// Memory-bound: a thread owns two neighbouring channels where the rows allow it and walks a run of rows with the last m - 1 inputs in
// registers, so a row is read once (and m - 1 rows more per run, from the L2).  65536 rows of 1536 channels, 4 taps, bf16: forward 74 us
// (5.5 TB/s), gradient 135 + 8 us (4.3 TB/s); fp32 146 us (5.5 TB/s) and 255 (4.7).  Eight channels per thread, 16 bytes of a row, took
// 107 and 178 in bf16: their weights lie 128 bytes apart from lane to lane, more lines than all the rows have.
#include "chela_rows.h"

namespace chela {

// V neighbouring elements as they lie in memory
template <int BYTES> struct Bits;
template <> struct Bits<2> { typedef unsigned short type; };
template <> struct Bits<4> { typedef unsigned type; };
template <> struct Bits<8> { typedef u32x2 type; };
template <typename IO, int V> using Raw = typename Bits<V * (int)sizeof(IO)>::type;

template <typename IO, int V>
__device__ __forceinline__ void widen(Raw<IO, V> t, float (&x)[V])
{
    struct Elements { IO e[V]; };
    const Elements s = __builtin_bit_cast(Elements, t);
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = to_f(s.e[i]);
}
template <typename IO, int V>
__device__ __forceinline__ Raw<IO, V> narrow(const float (&x)[V])
{
    struct Elements { IO e[V]; } s;
#pragma unroll
    for (int i = 0; i < V; ++i) s.e[i] = from_f<IO>(x[i]);
    return __builtin_bit_cast(Raw<IO, V>, s);
}
template <typename IO, int V>
__device__ __forceinline__ void load_row(const IO* p, float (&x)[V]) { widen<IO, V>(*reinterpret_cast<const Raw<IO, V>*>(p), x); }
template <typename IO, int V>
__device__ __forceinline__ void store_row(IO* p, const float (&x)[V]) { *reinterpret_cast<Raw<IO, V>*>(p) = narrow<IO, V>(x); }

template <int V>
__device__ __forceinline__ void activation(const float (&u)[V], int silu, float (&y)[V])
{
#pragma unroll
    for (int e = 0; e < V; ++e) y[e] = silu ? u[e] * sigmoid_(u[e]) : u[e];
}

// Where in the sequence that row t belongs to: one look-up per run, then by counting.
struct Where {
    int q, beg, end;
    __device__ __forceinline__ void start(const Rows& R, int sequence)
    {
        q = max(sequence, 0);
        set(R);
    }
    __device__ __forceinline__ void set(const Rows& R)
    {
        beg = q < R.n_seq ? seq_begin(R, q) : R.T;
        end = q < R.n_seq ? seq_end(R, q) : R.T;
    }
    // false: row t is in no sequence
    __device__ __forceinline__ bool at(const Rows& R, int t)
    {
        while (q < R.n_seq && end <= t) { ++q; set(R); }
        return q < R.n_seq && t >= beg;
    }
};

// The m - 1 inputs in front of row t of the sequence `at`: rows of it, or of its state, or 0.  back[j]: x_{t-1-j}.
template <typename IO, int V, int M>
__device__ __forceinline__ void history(const ShortConvArgs& a, const Where& at, int t, int ch, float (&back)[M > 1 ? M - 1 : 1][V])
{
    int slot = -2;
#pragma unroll
    for (int j = 0; j < M - 1; ++j) {
        const int r = t - 1 - j;
#pragma unroll
        for (int e = 0; e < V; ++e) back[j][e] = 0.f;
        if (r >= at.beg) {
            load_row<IO, V>((const IO*)a.X + (size_t)r * a.ldx + ch, back[j]);
        } else if (a.S_in) {
            if (slot == -2) slot = slot_of(a.rows, at.q);
            if (slot >= 0) load_row<IO, V>((const IO*)a.S_in + ((size_t)slot * (M - 1) + (M - 1 + r - at.beg)) * a.D + ch, back[j]);
        }
    }
}

// The same where the rows in front of row t are in `back` already, whatever sequence they are of.
template <typename IO, int V, int M>
__device__ __forceinline__ void in_front(const ShortConvArgs& a, const Where& at, int t, int ch, float (&back)[M > 1 ? M - 1 : 1][V])
{
    if (M == 1 || t - (M - 1) >= at.beg) return;
    const int slot = a.S_in ? slot_of(a.rows, at.q) : -1;
#pragma unroll
    for (int j = 0; j < M - 1; ++j) {
        const int r = t - 1 - j;
        if (r >= at.beg) continue;
#pragma unroll
        for (int e = 0; e < V; ++e) back[j][e] = 0.f;
        if (slot >= 0) load_row<IO, V>((const IO*)a.S_in + ((size_t)slot * (M - 1) + (M - 1 + r - at.beg)) * a.D + ch, back[j]);
    }
}
// Row r as it lies in memory; in front of the first and behind the last, where nothing is made of it, the nearest there is.
template <typename IO, int V>
__device__ __forceinline__ Raw<IO, V> load_raw(const void* X, long ld, int r, int T, int ch)
{
    return row_load((const Raw<IO, V>*)((const IO*)X + (size_t)min(max(r, 0), T - 1) * ld), ch * sizeof(IO));
}

template <int V, int M>
__device__ __forceinline__ void weights(const ShortConvArgs& a, int ch, float (&w)[M][V], float (&bias)[V])
{
#pragma unroll
    for (int e = 0; e < V; ++e) {
#pragma unroll
        for (int j = 0; j < M; ++j) w[j][e] = a.w[(size_t)(ch + e) * M + j];
        bias[e] = a.bias ? a.bias[ch + e] : 0.f;
    }
}

// The states behind the sequences, 256 channels of sequence `q`.  A thread reads all m - 1 rows of a channel before it writes one, but the
// rows of the sequences read the states in front too: where these are the same ones, the states come in a launch of their own, behind.
template <typename IO, int M>
__device__ __forceinline__ void state_behind(const ShortConvArgs& a, int q, int block)
{
    const int slot = slot_of(a.rows, q);
    if (slot < 0) return;
    Where at;
    at.q = q;
    at.set(a.rows);
    if (at.end < at.beg) at.end = at.beg;
    for (int ch = block * 256 + (int)threadIdx.x; ch < min(block * 256 + 256, a.D); ch += (int)blockDim.x) {
        float back[M > 1 ? M - 1 : 1][1];
        history<IO, 1, M>(a, at, at.end, ch, back);
#pragma unroll
        for (int j = 0; j < M - 1; ++j) ((IO*)a.S_out)[((size_t)slot * (M - 1) + (M - 2 - j)) * a.D + ch] = from_f<IO>(back[j][0]);
    }
}
template <typename IO, int M>
__global__ __launch_bounds__(256) void short_conv_state_kernel(ShortConvArgs a)
{
    const int nb = (a.D + 255) / 256;
    state_behind<IO, M>(a, blockIdx.x / nb, blockIdx.x % nb);
}

// Rows t0 .. t1 - 1 of no sequence: those in front of `front`, which the walk from t0 began with, and where it has come past the last
// sequence those behind it.  (Behind the walk: a store in it costs registers that it needs.)
template <typename IO, int V>
__device__ __forceinline__ void clear_rows(const Rows& R, int front, const Where& at, void* Y, int D, int t0, int t1, int ch)
{
    if (t0 >= front && at.q < R.n_seq) return;
    const int stop = at.q < R.n_seq ? R.T : R.n_seq > 0 ? seq_end(R, R.n_seq - 1) : 0;
#pragma unroll 1
    for (int t = t0; t < t1; ++t)
        if (t < front || t >= stop) row_store((Raw<IO, V>*)((IO*)Y + (size_t)t * D), ch * sizeof(IO), Raw<IO, V>(0));
}

// Workgroups go to the eight XCDs in turn: the neighbours in memory, which read each other's last rows, to one of them.
__device__ __forceinline__ int xcd_neighbours(int i, int n)
{
    const int per = n / 8;
    return i < per * 8 ? i % 8 * per + i / 8 : i;
}

template <typename IO, int V, int M, int RUN>
__global__ __launch_bounds__(256) void short_conv_kernel(ShortConvArgs a)
{
    const int across = (a.D + V * (int)blockDim.x - 1) / (V * (int)blockDim.x);          // workgroups that a run takes
    const Rows& R = a.rows;
    const int runs = (R.T + RUN - 1) / RUN;
    if ((int)blockIdx.x >= runs * across) {
        const int nb = (a.D + 255) / 256, i = blockIdx.x - runs * across;
        state_behind<IO, M>(a, i / nb, i % nb);
        return;
    }
    const int mine = (blockIdx.x % across * blockDim.x + threadIdx.x) * V, ch = min(mine, a.D - V);
    const int t0 = xcd_neighbours(blockIdx.x / across, runs) * RUN, t1 = min(t0 + RUN, R.T);
    // all rows on their way before the sequence is looked for and the first is looked at
    Raw<IO, V> x[RUN + M - 1];
#pragma unroll
    for (int i = 0; i < RUN + M - 1; ++i) x[i] = load_raw<IO, V>(a.X, a.ldx, t0 - (M - 1) + i, R.T, ch);
    float w[M][V], bias[V], back[M > 1 ? M - 1 : 1][V];
    weights<V, M>(a, ch, w, bias);
    Where at;
    at.start(R, seq_of_wave(R, t0, threadIdx.x & 63));
    if (mine >= a.D) return;
    const bool whole = at.q < R.n_seq && t0 - (M - 1) >= at.beg && t0 + RUN <= at.end;       // within one sequence
#pragma unroll
    for (int j = 0; j < M - 1; ++j) widen<IO, V>(x[M - 2 - j], back[j]);
    auto row = [&](Raw<IO, V> raw, IO* to) {
        float now[V], u[V], y[V];
        widen<IO, V>(raw, now);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            u[e] = fmaf(w[0][e], now[e], bias[e]);
#pragma unroll
            for (int j = 1; j < M; ++j) u[e] = fmaf(w[j][e], back[j - 1][e], u[e]);
        }
        activation<V>(u, a.silu, y);
        if (to) row_store((Raw<IO, V>*)to, ch * sizeof(IO), narrow<IO, V>(y));
#pragma unroll
        for (int j = M - 2; j > 0; --j)
#pragma unroll
            for (int e = 0; e < V; ++e) back[j][e] = back[j - 1][e];
        if (M > 1)
#pragma unroll
            for (int e = 0; e < V; ++e) back[0][e] = now[e];
    };
    if (whole) {
#pragma unroll
        for (int i = 0; i < RUN; ++i) row(x[i + M - 1], (IO*)a.Y + (size_t)(t0 + i) * a.D);
        return;
    }
    int known = -1;                                   // the sequence that `back` is of
    const int front = at.beg;
#pragma unroll 1
    for (int t = t0; t < t1; ++t) {
        const bool on = at.at(R, t);
        if (on && known != at.q) { in_front<IO, V, M>(a, at, t, ch, back); known = at.q; }
        row(x[M - 1], on ? (IO*)a.Y + (size_t)t * a.D : nullptr);
#pragma unroll
        for (int i = M - 1; i < RUN + M - 2; ++i) x[i] = x[i + 1];
    }
    if (R.clear) clear_rows<IO, V>(R, front, at, a.Y, a.D, t0, t1, ch);
}

// One row for each of R requests: the states move on by one.
template <typename IO, int V, int M>
__global__ __launch_bounds__(64) void short_conv_step_kernel(ShortConvArgs a)
{
    const int nb = (a.D + 64 * V - 1) / (64 * V), r = blockIdx.x / nb, ch = (blockIdx.x % nb * 64 + threadIdx.x) * V;
    if (ch >= a.D) return;
    const int slot = slot_of(a.rows, r);
    if (slot < 0) {
        if (a.rows.clear) row_store((Raw<IO, V>*)((IO*)a.Y + (size_t)r * a.D), ch * sizeof(IO), Raw<IO, V>(0));
        return;
    }
    IO* S = (IO*)a.S_out + (size_t)slot * (M - 1) * a.D + ch;
    float w[M][V], bias[V], s[M > 1 ? M - 1 : 1][V], x[V], u[V], y[V];
    load_row<IO, V>((const IO*)a.X + (size_t)r * a.ldx + ch, x);
#pragma unroll
    for (int j = 0; j < M - 1; ++j) load_row<IO, V>(S + (size_t)j * a.D, s[j]);
    weights<V, M>(a, ch, w, bias);
#pragma unroll
    for (int e = 0; e < V; ++e) {
        u[e] = fmaf(w[0][e], x[e], bias[e]);
#pragma unroll
        for (int j = 1; j < M; ++j) u[e] = fmaf(w[j][e], s[M - 1 - j][e], u[e]);
    }
    activation<V>(u, a.silu, y);
    store_row<IO, V>((IO*)a.Y + (size_t)r * a.D + ch, y);
#pragma unroll
    for (int j = 0; j < M - 2; ++j) store_row<IO, V>(S + (size_t)j * a.D, s[j + 1]);
    if (M > 1) store_row<IO, V>(S + (size_t)(M - 2) * a.D, x);
}

// Gradient.  A workgroup walks runs of rows; the sums of dw and dbias stay in its threads' registers and leave once, per workgroup, for
// short_conv_sum_kernel to add up in a fixed order.  pend[k]: what dx of row t - k has so far.
template <typename IO, int V, int M, int RUN>
__global__ __launch_bounds__(256) void short_conv_bwd_kernel(ShortConvArgs a, int runs)
{
    const int ch = (blockIdx.x * blockDim.x + threadIdx.x) * V;
    if (ch >= a.D) return;
    const Rows& R = a.rows;
    float w[M][V], bias[V], dw[M][V], db[V];
    weights<V, M>(a, ch, w, bias);
#pragma unroll
    for (int e = 0; e < V; ++e) {
        db[e] = 0.f;
#pragma unroll
        for (int j = 0; j < M; ++j) dw[j][e] = 0.f;
    }
    // neighbouring runs, so that the rows that two runs share come from the L2
    const int mine = (runs + (int)gridDim.y - 1) / (int)gridDim.y, first = (int)blockIdx.y * mine;
    Where at;                                         // (looked up once: for each run anew, 32 sequences cost 45 of 180 us)
    at.start(R, seq_of(R, first * RUN));
    for (int run = first; run < min(first + mine, runs); ++run) {
        const int t0 = run * RUN, t1 = min(t0 + RUN, R.T);
        // the run and all that it shares with others on their way before the sequence is looked for and the first row is looked at
        Raw<IO, V> xs[RUN + 2 * (M - 1)], dys[RUN + M - 1];
#pragma unroll
        for (int i = 0; i < RUN + 2 * (M - 1); ++i) xs[i] = load_raw<IO, V>(a.X, a.ldx, t0 - (M - 1) + i, R.T, ch);
#pragma unroll
        for (int i = 0; i < RUN + M - 1; ++i) dys[i] = load_raw<IO, V>(a.dY, a.lddy, t0 + i, R.T, ch);
        float back[M > 1 ? M - 1 : 1][V], pend[M][V];
        at.at(R, t0);
        // within one sequence, none of the last m - 1 rows in it?
        const bool whole = at.q < R.n_seq && t0 - (M - 1) >= at.beg && t0 + RUN + M - 1 <= at.end;
#pragma unroll
        for (int j = 0; j < M - 1; ++j) widen<IO, V>(xs[M - 2 - j], back[j]);
#pragma unroll
        for (int k = 0; k < M; ++k)
#pragma unroll
            for (int e = 0; e < V; ++e) pend[k][e] = 0.f;
        // a row's part in pend and, if it is one of the run's, in the sums
        auto row = [&](Raw<IO, V> xr, Raw<IO, V> dyr, bool mine) {
            float x[V], du[V];
            widen<IO, V>(xr, x);
            widen<IO, V>(dyr, du);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                if (a.silu) {
                    float u = fmaf(w[0][e], x[e], bias[e]);
#pragma unroll
                    for (int j = 1; j < M; ++j) u = fmaf(w[j][e], back[j - 1][e], u);
                    const float s = sigmoid_(u);
                    du[e] *= s * fmaf(u, 1.f - s, 1.f);
                }
#pragma unroll
                for (int j = 0; j < M; ++j) pend[j][e] = fmaf(w[j][e], du[e], pend[j][e]);
                if (mine) {
                    db[e] += du[e];
                    dw[0][e] = fmaf(du[e], x[e], dw[0][e]);
#pragma unroll
                    for (int j = 1; j < M; ++j) dw[j][e] = fmaf(du[e], back[j - 1][e], dw[j][e]);
                }
            }
        };
        auto next_x = [&](Raw<IO, V> xr) {
#pragma unroll
            for (int j = M - 2; j > 0; --j)
#pragma unroll
                for (int e = 0; e < V; ++e) back[j][e] = back[j - 1][e];
            if (M > 1) widen<IO, V>(xr, back[0]);
        };
        auto next_pend = [&]() {
#pragma unroll
            for (int j = M - 1; j > 0; --j)
#pragma unroll
                for (int e = 0; e < V; ++e) pend[j][e] = pend[j - 1][e];
#pragma unroll
            for (int e = 0; e < V; ++e) pend[0][e] = 0.f;
        };
        if (whole) {
#pragma unroll
            for (int i = 0; i < RUN + M - 1; ++i) {
                row(xs[i + M - 1], dys[i], i < RUN);
                if (i >= M - 1)
                    row_store((Raw<IO, V>*)((IO*)a.dX + (size_t)(t0 + i - (M - 1)) * a.D), ch * sizeof(IO), narrow<IO, V>(pend[M - 1]));
                next_x(xs[i + M - 1]);
                next_pend();
            }
            continue;
        }
        int known = -1;
        const int front = at.beg;
        // rows t1 .. t1 + m - 2 of the same sequence give to the rows of this run too
#pragma unroll 1
        for (int t = t0; t - t1 < M - 1; ++t) {
            if (t >= R.T || (t >= t1 && (known != at.q || t >= at.end))) break;
            const Raw<IO, V> xr = xs[M - 1], dyr = dys[0];
#pragma unroll
            for (int i = M - 1; i < RUN + 2 * (M - 1) - 1; ++i) xs[i] = xs[i + 1];
#pragma unroll
            for (int i = 0; i < RUN + M - 2; ++i) dys[i] = dys[i + 1];
            if (t < t1 && !at.at(R, t)) { next_x(xr); continue; }
            if (known != at.q) {
                known = at.q;
                in_front<IO, V, M>(a, at, t, ch, back);
#pragma unroll
                for (int k = 0; k < M; ++k)
#pragma unroll
                    for (int e = 0; e < V; ++e) pend[k][e] = 0.f;
            }
            row(xr, dyr, t < t1);
            next_x(xr);
            // what is complete: row t - (m - 1); behind the sequence's last row, all that are left.  (One after the other: this code runs once in
            // a while, and has to come from memory first)
            const int rows = t == at.end - 1 ? M : 1;
#pragma unroll 1
            for (int i = 0; i < rows; ++i, next_pend()) {
                const int r = t + i - (M - 1), behind = r - (at.end - (M - 1));        // place in the state behind the sequence
                if (r >= at.beg ? (r < t0 || r >= t1) : (!a.dS_in || at.beg < t0 || at.beg >= t1 || r < at.beg - (M - 1))) continue;
                float g[V];
#pragma unroll
                for (int e = 0; e < V; ++e) g[e] = pend[M - 1][e];
                const int slot = (r < at.beg || (a.dS_out && behind >= 0)) ? slot_of(R, at.q) : -1;
                if (a.dS_out && behind >= 0 && slot >= 0) {
                    float d[V];
                    load_row<IO, V>((const IO*)a.dS_out + ((size_t)slot * (M - 1) + behind) * a.D + ch, d);
#pragma unroll
                    for (int e = 0; e < V; ++e) g[e] += d[e];
                }
                if (r >= at.beg) store_row<IO, V>((IO*)a.dX + (size_t)r * a.D + ch, g);
                else if (slot >= 0) store_row<IO, V>((IO*)a.dS_in + ((size_t)slot * (M - 1) + (M - 1 + r - at.beg)) * a.D + ch, g);
            }
        }
        if (R.clear) clear_rows<IO, V>(R, front, at, a.dX, a.D, t0, t1, ch);
    }
    float* part = a.part + (size_t)blockIdx.y * (M + 1) * a.D + ch;
#pragma unroll
    for (int e = 0; e < V; ++e) {
#pragma unroll
        for (int j = 0; j < M; ++j) part[(size_t)j * a.D + e] = dw[j][e];
        part[(size_t)M * a.D + e] = db[e];
    }
}

// The workgroups' sums, sixteen waves to 64 channels.
__global__ __launch_bounds__(1024) void short_conv_sum_kernel(ShortConvArgs a, int parts)
{
    __shared__ float s_sum[16][64];
    const int lane = threadIdx.x & 63, ch = blockIdx.x * 64 + lane, j = blockIdx.y, w = threadIdx.x >> 6;
    const float* from = a.part + (size_t)j * a.D + min(ch, a.D - 1);
    float x = 0.f;
#pragma unroll 8
    for (int p = w; p < parts; p += 16) x += from[(size_t)p * (a.m + 1) * a.D];
    s_sum[w][lane] = x;
    __syncthreads();
    if (w != 0 || ch >= a.D) return;
    x = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) x += s_sum[i][lane];
    if (j < a.m) a.dw[(size_t)ch * a.m + j] = x;
    else if (a.dbias) a.dbias[ch] = x;
}

// Sequences without rows hand the state's gradient on.
template <typename IO>
__global__ __launch_bounds__(256) void short_conv_empty_kernel(ShortConvArgs a)
{
    for (int s = blockIdx.x; s < a.rows.n_seq; s += gridDim.x) {
        if (seq_begin(a.rows, s) < seq_end(a.rows, s)) continue;
        const int slot = slot_of(a.rows, s);
        if (slot < 0) continue;
        const size_t n = (size_t)(a.m - 1) * a.D, at = n * slot;
        for (size_t i = threadIdx.x; i < n; i += 256) ((IO*)a.dS_in)[at + i] = a.dS_out ? ((const IO*)a.dS_out)[at + i] : (IO)0.f;
    }
}

// -------------------------------------------------------------------------------------------------------------------- host
// Two neighbouring channels per thread, where every row begins on as many bytes
static bool pairs(const ShortConvArgs& a, int dtype)
{
    const unsigned bytes = dtype == 0 ? 4 : 8;
    return a.D % 2 == 0 && a.ldx % 2 == 0 && a.lddy % 2 == 0 && (((uintptr_t)a.X | (uintptr_t)a.dY) & (bytes - 1)) == 0;
}
static unsigned threads_for(int vectors) { return vectors >= 256 ? 256u : (unsigned)(vectors + 63) / 64 * 64; }

#define CHELA_TAPS(F, IO, V)                                                                                          \
    switch (a.m) {                                                                                                    \
        case 1: F(IO, V, 1); break;                                                                                   \
        case 2: F(IO, V, 2); break;                                                                                   \
        case 3: F(IO, V, 3); break;                                                                                   \
        case 4: F(IO, V, 4); break;                                                                                   \
        case 5: F(IO, V, 5); break;                                                                                   \
        case 6: F(IO, V, 6); break;                                                                                   \
        case 7: F(IO, V, 7); break;                                                                                   \
        case 8: F(IO, V, 8); break;                                                                                   \
        default: return hipErrorInvalidValue;                                                                         \
    }
#define CHELA_TYPES(F)                                                                                                \
    if (dtype == 0) { if (V > 1) { CHELA_TAPS(F, bf16, 2) } else { CHELA_TAPS(F, bf16, 1) } }                         \
    else { if (V > 1) { CHELA_TAPS(F, float, 2) } else { CHELA_TAPS(F, float, 1) } }

// Rows of a run: the fewer, the more rows are read twice, the more, the fewer workgroups there are to read.  Forward, us, runs of 8, 16, 32
// rows: 83, 74, 70 at 65536 rows, 13.7, 15.0, - at 6007 (the short ones below 2048 workgroups).  Gradient, runs of 8 in as many parts as
// make 768 * 768 threads, half and twice as many: 1536 channels 138, 148, 143 us, 4096 channels 133, -, 145 (what the parts leave has to be added
// up); of few channels more of them fill the card: 101 channels, 768 and 1536 parts, 319 and 240.
constexpr int kRun = 16, kShortRun = 8, kBwdRun = 8, kBwdThreads = 768 * 768, kLeastParts = 256, kMostParts = 1536;

hipError_t launch_short_conv_fwd(const ShortConvArgs& a, int dtype, hipStream_t st)
{
    ProfScope prof(KID_SHORT_CONV, st);
    const unsigned states = a.S_out && a.m > 1 ? (unsigned)((a.D + 255) / 256) * (unsigned)a.rows.n_seq : 0;
    const bool apart = a.S_out == a.S_in || a.rows.T == 0;
    if (a.rows.T > 0) {
        const int V = pairs(a, dtype) ? 2 : 1, vectors = (a.D + V - 1) / V;
        const unsigned threads = threads_for(vectors), across = (vectors + threads - 1) / threads;
        const bool few = (long)((a.rows.T + kRun - 1) / kRun) * across < 2048;
        const int run = few ? kShortRun : kRun;
        const dim3 grid(across * (unsigned)((a.rows.T + run - 1) / run) + (apart ? 0 : states));
#define CHELA_F(IO, V, M)                                                                                             \
    if (few) hipLaunchKernelGGL((short_conv_kernel<IO, V, M, kShortRun>), grid, dim3(threads), 0, st, a);             \
    else hipLaunchKernelGGL((short_conv_kernel<IO, V, M, kRun>), grid, dim3(threads), 0, st, a)
        CHELA_TYPES(CHELA_F)
#undef CHELA_F
    }
    if (states > 0 && apart) {
#define CHELA_F(IO, V, M) hipLaunchKernelGGL((short_conv_state_kernel<IO, M>), dim3(states), dim3(256), 0, st, a)
        if (dtype == 0) { CHELA_TAPS(CHELA_F, bf16, 1) } else { CHELA_TAPS(CHELA_F, float, 1) }
#undef CHELA_F
    }
    return hipGetLastError();
}

int short_conv_bwd_parts(int T, int D)
{
    const int threads = (D / (D % 2 ? 1 : 2) + 63) / 64 * 64, runs = (T + kBwdRun - 1) / kBwdRun;
    const int want = kBwdThreads / threads, most = want > kMostParts ? kMostParts : want < kLeastParts ? kLeastParts : want;
    return runs < most ? (runs > 0 ? runs : 1) : most;
}

hipError_t launch_short_conv_bwd(const ShortConvArgs& a, int dtype, hipStream_t st)
{
    ProfScope prof(KID_SHORT_CONV, st);
    const int V = pairs(a, dtype) ? 2 : 1, vectors = (a.D + V - 1) / V;
    const unsigned threads = threads_for(vectors);
    const int runs = (a.rows.T + kBwdRun - 1) / kBwdRun, parts = short_conv_bwd_parts(a.rows.T, a.D);
    const dim3 grid((vectors + threads - 1) / threads, parts);
#define CHELA_F(IO, V, M) hipLaunchKernelGGL((short_conv_bwd_kernel<IO, V, M, kBwdRun>), grid, dim3(threads), 0, st, a, runs)
    CHELA_TYPES(CHELA_F)
#undef CHELA_F
    hipLaunchKernelGGL(short_conv_sum_kernel, dim3((a.D + 63) / 64, a.m + 1), dim3(1024), 0, st, a, parts);
    if (a.dS_in && a.m > 1 && a.rows.n_seq > 0 && (a.rows.cu || a.rows.T == 0)) {
        const dim3 g(a.rows.n_seq < 256 ? a.rows.n_seq : 256);
        if (dtype == 0) hipLaunchKernelGGL(short_conv_empty_kernel<bf16>, g, dim3(256), 0, st, a);
        else hipLaunchKernelGGL(short_conv_empty_kernel<float>, g, dim3(256), 0, st, a);
    }
    return hipGetLastError();
}

hipError_t launch_short_conv_step(const ShortConvArgs& a, int dtype, hipStream_t st)
{
    ProfScope prof(KID_SHORT_CONV, st);
    const int V = pairs(a, dtype) ? 2 : 1, nb = (a.D + 64 * V - 1) / (64 * V);
    const dim3 grid((unsigned)nb * (unsigned)a.rows.T);
#define CHELA_F(IO, V, M) hipLaunchKernelGGL((short_conv_step_kernel<IO, V, M>), grid, dim3(64), 0, st, a)
    CHELA_TYPES(CHELA_F)
#undef CHELA_F
    return hipGetLastError();
}

}  // namespace chela
