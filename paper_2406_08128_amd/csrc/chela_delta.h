// What the kernels of the gated delta rule share: operands of the matrix instructions in either type, tiles in LDS, and the chunks that
// the sequences are cut into.
#pragma once
#include "chela_rows.h"

namespace chela {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(8))) float f32x8;
typedef __attribute__((ext_vector_type(4))) bf16 bf16x4;
typedef __attribute__((ext_vector_type(8))) bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) unsigned u32x2;
typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;

// Tokens of a chunk.  (fp32: a chunk's rows take twice the room in LDS.)
template <typename E> struct DeltaChunk { static constexpr int C = sizeof(E) == 2 ? kDeltaChunkBf16 : kDeltaChunkF32; };
// Elements behind each row of a tile in LDS: 32 bytes (bf16), so that the pieces that a read takes from eight or sixteen rows fall on all banks alike,
// the transposed ones too.  (16 bytes: outputs of 16 heads of 128, 65536 tokens, 342 us, with 32 318; gradients of heads of 64 and 128 311 and 298.)
template <typename E> constexpr int kPad = sizeof(E) == 2 ? 16 : 4;

// A 16 x 32 operand.  All products are 16 x 16 tiles over 32 terms, D[m][n] += sum_k A[m][k] B[n][k]: lane 16 q + c has row c of A (of B)
// at eight k, and of D the column n = c at the rows m = 4 q + i.  Which eight is free as long as A and B agree; here they are
//     k = 16 (j / 4) + 4 q + j % 4,  j = 0..7,
// the rows that two accumulator tiles, one above the other, have in this lane: a result is the next product's operand as it lies in the
// registers, summed over its rows.
// P parts: a value that was worked out in fp32 is rounded to bf16 (P = 1, off by 2^-8 at most) or kept as a sum of two (P = 2, 2^-16).  What the caller
// gave in bf16 has one part.  fp32 operands have all bits, and their products are fp32: eight instructions over four terms each.
// What goes into a state or through the inverse has two parts, and so have the inverse T and the scores P: tokens with keys alike take back most of what
// the one in front wrote, and with T and P in one part what is left was off by 1e-2 to 8e-2 (64 tokens alike; 1e-2 with keys of positive numbers) where
// two leave the output's own rounding, 1.7e-3.  One part have the states that outputs and gradients are made of, N in calls without states in fp32, the
// inner values U, dR and the scores X, Y that only gradients are made of.
template <typename E, int P> struct Op;
template <> struct Op<bf16, 1> { bf16x8 h; };
template <> struct Op<bf16, 2> { bf16x8 h, l; };
template <int P> struct Op<float, P> { f32x8 v; };

template <int PA, int PB>
__device__ __forceinline__ f32x4 mma(const Op<bf16, PA>& a, const Op<bf16, PB>& b, f32x4 c)
{
    if constexpr (PA == 2) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.l, b.h, c, 0, 0, 0);
    if constexpr (PB == 2) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.h, b.l, c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.h, b.h, c, 0, 0, 0);
}
template <int PA, int PB>
__device__ __forceinline__ f32x4 mma(const Op<float, PA>& a, const Op<float, PB>& b, f32x4 c)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[j], b.v[j], c, 0, 0, 0);
    return c;
}

// What has been rounded to bf16, in fp32 again.  (Out of the packed pairs: where the compiler sees the rounding it does it a second time, one by one.)
__device__ __forceinline__ f32x4 widen(bf16x4 x)
{
    const u32x2 u = __builtin_bit_cast(u32x2, x);
    return __builtin_bit_cast(f32x4, u32x4{u[0] << 16, u[0] & 0xffff0000u, u[1] << 16, u[1] & 0xffff0000u});
}
__device__ __forceinline__ f32x8 widen(bf16x8 x)
{
    return __builtin_shufflevector(widen(__builtin_shufflevector(x, x, 0, 1, 2, 3)), widen(__builtin_shufflevector(x, x, 4, 5, 6, 7)), 0, 1, 2, 3, 4, 5, 6, 7);
}

// Two accumulator tiles as an operand.
template <typename E, int P>
__device__ __forceinline__ Op<E, P> operand(f32x4 lo, f32x4 hi)
{
    const f32x8 x = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    Op<E, P> o;
    if constexpr (sizeof(E) == 4) {
        o.v = x;
    } else {
        o.h = __builtin_convertvector(x, bf16x8);
        if constexpr (P == 2) o.l = __builtin_convertvector(x - widen(o.h), bf16x8);
    }
    return o;
}

template <typename E> using Vec4 = typename std::conditional<sizeof(E) == 2, bf16x4, f32x4>::type;
template <typename E> using Vec8 = typename std::conditional<sizeof(E) == 2, bf16x8, f32x8>::type;

// Where column `col` of a tile lies in its row in LDS.  bf16: within 32 columns the two fours that a lane's eight k are come one behind the other, so that
// it reads them at once: 16 bytes of 64 lanes take 8 cycles (6 with 32 bytes behind each row), two times 8 bytes 16.
template <typename E>
__device__ __forceinline__ constexpr int place_of(int col)
{
    return sizeof(E) == 4 ? col : (col & ~31) | (col & 12) * 2 | (col & 16) / 4 | (col & 3);
}
// Four columns beginning with col0 + 4 q, col0 a multiple of 16.
template <typename E>
__device__ __forceinline__ int four_of(int col0, int q) { return sizeof(E) == 4 ? col0 + 4 * q : (col0 & ~31) + (col0 & 16) / 4 + 8 * q; }

// The operand that is X[row0 + c][k0 ..], rows of a tile, summed over its columns.
template <typename E>
__device__ __forceinline__ Op<E, 1> rows_op(const E* X, int ld, int row0, int k0, int lane)
{
    if constexpr (sizeof(E) == 2) {
        return Op<E, 1>{*(const bf16x8*)(X + (row0 + (lane & 15)) * ld + k0 + 8 * (lane >> 4))};
    } else {
        const E* p = X + (row0 + (lane & 15)) * ld + k0 + 4 * (lane >> 4);
        const f32x4 a = *(const f32x4*)p, b = *(const f32x4*)(p + 16);
        return Op<E, 1>{__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7)};
    }
}
// The operand that is X[k0 ..][col0 + c], columns of a tile, summed over its rows.  bf16: within 16 lanes the transposing read hands lane p
// the column p of a 4 x 16 block whose rows the lanes address as p / 4, and 8-byte pieces as p % 4.
template <typename E>
__device__ __forceinline__ Op<E, 1> cols_op(const E* X, int ld, int k0, int col0, int lane)
{
    const int q = lane >> 4, c = lane & 15;
    if constexpr (sizeof(E) == 2) {
        const bf16* p = X + (k0 + 4 * q + (c >> 2)) * ld + four_of<E>(col0, c & 3);
        const bf16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)p);
        const bf16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(p + 16 * ld));
        return Op<E, 1>{__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7)};
    } else {
        const float* p = X + (k0 + 4 * q) * ld + col0 + c;
        Op<E, 1> o;
#pragma unroll
        for (int j = 0; j < 4; ++j) { o.v[j] = p[j * ld]; o.v[4 + j] = p[(16 + j) * ld]; }
        return o;
    }
}

// A matrix of fp32 values in LDS in the form of operands: one part, or two a plane apart.
template <typename E, int P>
struct Planes {
    E* h;
    int ld, plane;                             // (plane: elements from the first parts to the second)
    __device__ __forceinline__ void put(int row, int col, float x) const
    {
        E* p = h + row * ld + place_of<E>(col);
        if constexpr (sizeof(E) == 4) {
            *p = x;
        } else {
            const bf16 a = (bf16)x;
            *p = a;
            if constexpr (P == 2) p[plane] = (bf16)(x - (float)a);
        }
    }
    __device__ __forceinline__ void put4(int row, int col0, int q, f32x4 x) const          // columns col0 + 4 q ..
    {
        E* p = h + row * ld + four_of<E>(col0, q);
        if constexpr (sizeof(E) == 4) {
            *(f32x4*)p = x;
        } else {
            const bf16x4 a = __builtin_convertvector(x, bf16x4);
            *(bf16x4*)p = a;
            if constexpr (P == 2) *(bf16x4*)(p + plane) = __builtin_convertvector(x - widen(a), bf16x4);
        }
    }
    __device__ __forceinline__ Op<E, P> rows(int row0, int k0, int lane) const
    {
        if constexpr (sizeof(E) == 2 && P == 2)
            return Op<E, P>{rows_op(h, ld, row0, k0, lane).h, rows_op(h + plane, ld, row0, k0, lane).h};
        else if constexpr (sizeof(E) == 4)
            return Op<E, P>{rows_op(h, ld, row0, k0, lane).v};
        else
            return rows_op(h, ld, row0, k0, lane);
    }
    __device__ __forceinline__ Op<E, P> cols(int k0, int col0, int lane) const
    {
        if constexpr (sizeof(E) == 2 && P == 2)
            return Op<E, P>{cols_op(h, ld, k0, col0, lane).h, cols_op(h + plane, ld, k0, col0, lane).h};
        else if constexpr (sizeof(E) == 4)
            return Op<E, P>{cols_op(h, ld, k0, col0, lane).v};
        else
            return cols_op(h, ld, k0, col0, lane);
    }
};

// An operand as it lies in memory, lanes next to each other: 16 bytes (bf16) or 32 (fp32) of a lane, the second parts behind the first.
template <typename E, int P> constexpr int kOpElems = 64 * 8 * (sizeof(E) == 2 ? P : 1);
template <typename E, int P>
__device__ __forceinline__ void store_op(E* to, const Op<E, P>& x, int lane)
{
    if constexpr (sizeof(E) == 4) {
        *(f32x8*)(to + 8 * lane) = x.v;
    } else {
        *(bf16x8*)(to + 8 * lane) = x.h;
        if constexpr (P == 2) *(bf16x8*)(to + 512 + 8 * lane) = x.l;
    }
}
template <typename E, int P>
__device__ __forceinline__ Op<E, P> load_op(const E* from, int lane)
{
    if constexpr (sizeof(E) == 4) {
        return Op<E, P>{*(const f32x8*)(from + 8 * lane)};
    } else {
        Op<E, P> o;
        o.h = *(const bf16x8*)(from + 8 * lane);
        if constexpr (P == 2) o.l = *(const bf16x8*)(from + 512 + 8 * lane);
        return o;
    }
}

// LDS is read again behind this: operands that one column group after the other needs would otherwise all be kept in registers.
__device__ __forceinline__ void read_afresh() { asm volatile("" ::: "memory"); }
__device__ __forceinline__ f32x4 zero4() { return f32x4{0.f, 0.f, 0.f, 0.f}; }
__device__ __forceinline__ f32x4 splat4(float x) { return f32x4{x, x, x, x}; }

// ---- chunks.  A sequence's rows are cut into chunks of C, the last one shorter.  The places of all chunks in the scratch: sequence s begins at
// cu[s] / C + s.  (A sequence of n rows has at most floor(n / C) + 1 chunks and the next one begins at least as much further on, so that no
// two chunks share a place, and there are T / C + n_seq places; no prefix sum is needed.)
__device__ __forceinline__ int chunk_key(const Rows& r, int C, int s)
{
    return r.cu == nullptr ? s * ((r.L + C - 1) / C) : seq_begin(r, s) / C + s;
}
__device__ __forceinline__ int chunks_in(const Rows& r, int C, int s)
{
    const int n = r.cu == nullptr ? r.L : seq_end(r, s) - seq_begin(r, s);
    return n > 0 ? (n + C - 1) / C : 0;
}
// The same holds for runs of several chunks: C is then a run's tokens.
struct Chunk { int seq, index, row, n; };      // its sequence, which of that one's chunks, its first row, its rows (0: nothing is here)
// All 64 lanes of a wave together, 64 sequences at a time.
__device__ __forceinline__ Chunk chunk_at(const Rows& r, int C, int place, int lane)
{
    Chunk c{0, 0, 0, 0};
    if (r.cu == nullptr) {
        const int per = (r.L + C - 1) / C;
        if (per == 0) return c;
        c.seq = place / per;
        c.index = place - c.seq * per;
    } else {
        int first = 0, n = r.n_seq;
        while (n > 64) {
            const int step = (n + 63) / 64, i = lane * step;
            const int below = __popcll(__ballot(i < n && chunk_key(r, C, first + min(i, n - 1)) <= place));
            if (below == 0) return c;
            const int skip = min((below - 1) * step, n - 1);
            first += skip;
            n = min(step, n - skip);
        }
        const int below = n > 0 ? __popcll(__ballot(lane < n && chunk_key(r, C, first + min(lane, n - 1)) <= place)) : 0;
        if (below == 0) return c;
        c.seq = first + below - 1;
        c.index = place - chunk_key(r, C, c.seq);
    }
    if (c.seq >= r.n_seq || c.index < 0 || c.index >= chunks_in(r, C, c.seq)) return c;       // (below 0: offsets out of order)
    c.row = (r.cu == nullptr ? c.seq * r.L : seq_begin(r, c.seq)) + c.index * C;
    c.n = min(C, (r.cu == nullptr ? (c.seq + 1) * r.L : seq_end(r, c.seq)) - c.row);
    return c;
}

// The place of the k-th chunk of a run among all chunks, whatever runs there are.
__device__ __forceinline__ int chunk_place(const Rows& r, int C, const Chunk& run, int chunks_to_a_run, int k)
{
    return chunk_key(r, C, run.seq) + run.index * chunks_to_a_run + k;
}

// ---- what a chunk's tokens have of their own: beta, and the running sum of the log decays, gamma.  Sums of 64 bits, held as two floats: two
// tokens' difference has to be good to fp32's last digits behind any number of strong decays.  A log decay below -256 (infinite ones
// too) stands for none of the state being left, which fp32 makes of -104 already.
template <int C>
struct ChunkSteps {
    // (hi + lo: gamma in units of ln 2); up: e^gamma, down: e^(gamma of the last token - gamma), bu: -beta up
    alignas(16) float hi[C], lo[C], beta[C], up[C], down[C], bu[C];
    float whole;                                                       // e^(gamma of the last token)
    // e^(gamma_t - gamma_s) of one token t and four s from s0 on; of four t from t0 on and one s.  (Where s > t it is not wanted and may be infinite: what
    // it is a factor of is chosen away there.  Worked out for all lanes alike: with a branch around each of them, a wave waits for LDS at each.)
    __device__ __forceinline__ f32x4 decays_from(int t, int s0) const
    {
        const f32x4 d = (splat4(hi[t]) - *(const f32x4*)(hi + s0)) + (splat4(lo[t]) - *(const f32x4*)(lo + s0));
        return f32x4{exp2_(d[0]), exp2_(d[1]), exp2_(d[2]), exp2_(d[3])};
    }
    __device__ __forceinline__ f32x4 decays_to(int t0, int s) const
    {
        const f32x4 d = (*(const f32x4*)(hi + t0) - splat4(hi[s])) + (*(const f32x4*)(lo + t0) - splat4(lo[s]));
        return f32x4{exp2_(d[0]), exp2_(d[1]), exp2_(d[2]), exp2_(d[3])};
    }
};
// Sums over the lanes up to each, by DPP: within rows of 16 lanes, then the rows' totals.
template <int CTRL, int ROWS>
__device__ __forceinline__ double plus_dpp(double x)
{
    typedef __attribute__((ext_vector_type(2))) int i32x2;
    const i32x2 v = __builtin_bit_cast(i32x2, x);
    const i32x2 y{__builtin_amdgcn_update_dpp(0, v[0], CTRL, ROWS, 0xf, false), __builtin_amdgcn_update_dpp(0, v[1], CTRL, ROWS, 0xf, false)};
    return x + __builtin_bit_cast(double, y);
}
__device__ __forceinline__ double running_sum(double x)
{
    x = plus_dpp<0x111, 0xf>(x);
    x = plus_dpp<0x112, 0xf>(x);
    x = plus_dpp<0x114, 0xf>(x);
    x = plus_dpp<0x118, 0xf>(x);
    x = plus_dpp<0x142, 0xa>(x);           // lane 15's to the second row, 47's to the fourth
    return plus_dpp<0x143, 0xc>(x);        // lane 31's to the upper two
}
// Four rows of a tile in LDS from row0 + 4 q on, of column col0 + c: as an accumulator tile has them.
template <typename E>
__device__ __forceinline__ f32x4 tile_of(const E* X, int ld, int row0, int col0, int lane)
{
    const int q = lane >> 4, c = lane & 15;
    if constexpr (sizeof(E) == 2) {
        return __builtin_convertvector(__builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(X + (row0 + 4 * q + (c >> 2)) * ld + four_of<E>(col0, c & 3))), f32x4);
    } else {
        const float* p = X + (row0 + 4 * q) * ld + col0 + c;
        return f32x4{p[0], p[ld], p[2 * ld], p[3 * ld]};
    }
}
// The log decay and beta of this lane's token, on their way; n rows there are, the rest are as if they were not (no decay, beta of zero).
struct Steps { float g, beta; };
template <typename E>
__device__ __forceinline__ Steps fetch_steps(const E* g, long ldg, const E* beta, long ldb, int row, int h, int n, int lane)
{
    const size_t t = (size_t)row + min(lane, n - 1);
    return Steps{g != nullptr ? to_f(g[t * ldg + h]) : 0.f, to_f(beta[t * ldb + h])};
}
// By the first wave.
template <int C>
__device__ __forceinline__ void put_steps(ChunkSteps<C>& st, const Steps& x, int n, int tid)
{
    if (tid < 64) {
        const int t = tid;
        const float b = t < n ? x.beta : 0.f, g = t < n ? (x.g < -256.f ? -256.f : x.g) : 0.f;
        const double s = running_sum((double)g) * 1.4426950408889634074;
        typedef __attribute__((ext_vector_type(2))) int i32x2;
        const i32x2 v = __builtin_bit_cast(i32x2, s);
        const double last = __builtin_bit_cast(double, i32x2{__builtin_amdgcn_readlane(v[0], 63), __builtin_amdgcn_readlane(v[1], 63)});
        if (t < C) {
            const float hi = (float)s, up = exp2_(hi);
            st.hi[t] = hi;
            st.lo[t] = (float)(s - (double)hi);
            st.beta[t] = b;
            st.up[t] = up;
            st.bu[t] = -b * up;
            st.down[t] = exp2_((float)(last - s));
            if (t == 0) st.whole = exp2_((float)last);
        }
    }
}

// What a chunk or a run makes of a state is kept as M - w, w times the identity beside it, w = e^Gamma (Gamma the sum of its log decays) where that
// is below 1, so that a state without decay goes through as it is.  Above 1 it is not: keys that replace what grows leave M far below e^Gamma, and what
// is kept would be rounded relative to that, to no digit of M in the end.  w is 1 there, from chunk to chunk w <- min(1, e^gamma w), and what is left of
// e^gamma w comes into M - w.  (What is not a number stays it.)
__device__ __forceinline__ float no_growth(float x) { return x > 1.f ? 1.f : x; }
// x on the diagonal of a tile, added to an accumulator
__device__ __forceinline__ f32x4 plus_diagonal(f32x4 a, float x, int lane)
{
    const int q = lane >> 4, c = lane & 15;
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] += 4 * q + i == c ? x : 0.f;
    return a;
}

// The same operand with each of its eight terms times a factor: f[k0 ..], one for each row of the tile that it was read from.
template <typename E, int P>
__device__ __forceinline__ Op<E, P> scaled(const Op<E, 1>& x, const float* f, int k0, int lane, float by = 1.f)
{
    const f32x4 a = *(const f32x4*)(f + k0 + 4 * (lane >> 4)), b = *(const f32x4*)(f + k0 + 16 + 4 * (lane >> 4));
    f32x8 v;
    if constexpr (sizeof(E) == 4) v = x.v;
    else v = __builtin_convertvector(x.h, f32x8);
    v *= __builtin_shufflevector(a * by, b * by, 0, 1, 2, 3, 4, 5, 6, 7);
    return operand<E, P>(__builtin_shufflevector(v, v, 0, 1, 2, 3), __builtin_shufflevector(v, v, 4, 5, 6, 7));
}

// A chunk's rows of one head, C of D elements, from memory to LDS by way of the registers of NT threads, zeros behind the n there are (the last
// row again is what is read for them: no load waits for a comparison).  Rows begin on an element: loads of global memory need no more.
template <typename E, int C, int D, int NT = 256>
struct Tile {
    static constexpr int W = 16 / sizeof(E), ALL = C * (D / W), M = (ALL + NT - 1) / NT;
    u32x4 x[M];
    __device__ __forceinline__ void fetch(const E* from, long ld, int row, int n, int tid)
    {
        struct __attribute__((packed, aligned(sizeof(E)))) Loose { u32x4 p; };
#pragma unroll
        for (int m = 0; m < M; ++m) {
            const int i = min(m * NT + tid, ALL - 1), t = i / (D / W), k = i % (D / W) * W;
            x[m] = ((const Loose*)(from + (size_t)(row + min(t, n - 1)) * ld + k))->p;
        }
    }
    // (AS_IS: what was written as it lay in LDS)
    template <bool AS_IS = false>
    __device__ __forceinline__ void put(E* to, int ldt, int n, int tid) const
    {
#pragma unroll
        for (int m = 0; m < M; ++m) {
            const int i = m * NT + tid, t = i / (D / W), k = i % (D / W) * W;
            if (ALL % NT != 0 && i >= ALL) break;
            const u32x4 v = t < n ? x[m] : u32x4{0, 0, 0, 0};
            if constexpr (AS_IS || sizeof(E) == 4) {
                *(u32x4*)(to + t * ldt + k) = v;
            } else {
                E* p = to + t * ldt + place_of<E>(k);
                *(u32x2*)p = u32x2{v[0], v[1]};
                *(u32x2*)(p + 8) = u32x2{v[2], v[3]};
            }
        }
    }
};

// Rows of no sequence: zeros in all of `width` elements of each, sixty-four rows to a workgroup.
template <typename E>
__device__ __forceinline__ void clear_rows(const Rows& r, int block, E* to, int width)
{
    if (to == nullptr) return;
    const int lo = r.n_seq > 0 ? seq_begin(r, 0) : r.T, hi = r.n_seq > 0 ? seq_begin(r, r.n_seq) : r.T;
    const int end = min(r.T, 64 * block + 64);
    for (int t = 64 * block; t < end; ++t) {
        if (t >= lo && t < hi) continue;
        E* row = to + (size_t)t * width;
        for (int i = threadIdx.x; i < width; i += blockDim.x) row[i] = (E)0.f;
    }
}

// T between LDS and memory.  Its diagonal is ones and nothing is above it: the C (C - 1) / 2 elements below, as words of both parts (the second in the upper
// half), take what one part of all its elements would.  Pieces of four words, C / 4 to a pair of rows, t behind C - 1 - t, which has as many fours below the
// diagonal's more as t has fewer; the last piece has the three words that the two rows have in the diagonal's fours.  (fp32: all elements as they are.)
template <typename E, int C, int NT>
struct PackedT {
    static constexpr bool PACK = sizeof(E) == 2;
    static constexpr int F = C / 4, W = F - 1, ALL = PACK ? C / 2 * F : C * F, M = (ALL + NT - 1) / NT;
    u32x4 x[M];
    struct Place { int row, four; };                               // (of the last piece: the lower row's four on the diagonal)
    static __device__ __forceinline__ Place place(int i)
    {
        const int r = i / F, p = i % F, a = r / 4;
        if constexpr (!PACK) return Place{r, p};
        return p < W - a ? Place{C - 1 - r, p} : Place{r, p - (W - a)};
    }
    __device__ __forceinline__ void fetch(const E* from, int tid)
    {
#pragma unroll
        for (int m = 0; m < M; ++m) x[m] = ((const u32x4*)from)[ALL % NT == 0 ? m * NT + tid : min(m * NT + tid, ALL - 1)];
    }
    __device__ __forceinline__ void put(const Planes<E, 2>& T, int tid) const
    {
        auto four = [&](int t, int j, u32x4 w) {
            E* p = T.h + t * T.ld + place_of<E>(4 * j);
            *(u32x2*)p = u32x2{w[0] & 0xffffu | w[1] << 16, w[2] & 0xffffu | w[3] << 16};
            *(u32x2*)(p + T.plane) = u32x2{w[0] >> 16 | w[1] & 0xffff0000u, w[2] >> 16 | w[3] & 0xffff0000u};
        };
        constexpr unsigned ONE = 0x3f80u;
#pragma unroll
        for (int m = 0; m < M; ++m) {
            const int i = m * NT + tid, r = i / F, b = r % 4;
            if (ALL % NT != 0 && i >= ALL) break;
            const Place at = place(i);
            u32x4 w = x[m];
            if constexpr (!PACK) {
                *(u32x4*)(T.h + at.row * T.ld + 4 * at.four) = w;
            } else {
                if (i % F == W) {
                    const int o = 3 - b;                           // words of the upper row
                    four(C - 1 - r, W - r / 4, u32x4{o > 0 ? w[0] : ONE, o > 1 ? w[1] : o == 1 ? ONE : 0u, o > 2 ? w[2] : o == 2 ? ONE : 0u, o > 2 ? ONE : 0u});
                    w = u32x4{b > 2 ? w[0] : b > 1 ? w[1] : b > 0 ? w[2] : ONE, b > 2 ? w[1] : b > 1 ? w[2] : b > 0 ? ONE : 0u, b > 2 ? w[2] : b > 1 ? ONE : 0u, b > 2 ? ONE : 0u};
                }
                four(at.row, at.four, w);
            }
        }
        // zeros behind the diagonal's fours, where a product reads them: to the end of the 32 columns; four threads to a row
        if constexpr (PACK)
            if (NT == 4 * C || tid < 4 * C) {
                const int t = tid / 4;
#pragma unroll
                for (int j = tid % 4 + 1; j < 8; j += 4)
                    if (t / 4 % 8 + j < 8) four(t, t / 4 + j, u32x4{0, 0, 0, 0});
            }
    }
    // read(row, four): those words
    template <typename R>
    static __device__ __forceinline__ void store(const R& read, E* to, int tid)
    {
#pragma unroll
        for (int m = 0; m < M; ++m) {
            const int i = m * NT + tid, r = i / F, o = 3 - r % 4;
            if (ALL % NT != 0 && i >= ALL) break;
            const Place at = place(i);
            u32x4 w = read(at.row, at.four);
            if (PACK && i % F == W) {
                const u32x4 u = read(C - 1 - r, W - r / 4);
                w = u32x4{o > 0 ? u[0] : w[0], o > 1 ? u[1] : o > 0 ? w[0] : w[1], o > 2 ? u[2] : o > 1 ? w[0] : o > 0 ? w[1] : w[2], 0u};
            }
            ((u32x4*)to)[i] = w;
        }
    }
};
// ... from its two parts, a plane apart
template <typename E>
struct WordsOfPlanes {
    const Planes<E, 2>& T;
    __device__ __forceinline__ u32x4 operator()(int t, int j) const
    {
        const E* p = T.h + t * T.ld + place_of<E>(4 * j);
        if constexpr (sizeof(E) == 4) return *(const u32x4*)p;
        const u32x2 h = *(const u32x2*)p, l = *(const u32x2*)(p + T.plane);
        return u32x4{h[0] & 0xffffu | l[0] << 16, h[0] >> 16 | l[0] & 0xffff0000u, h[1] & 0xffffu | l[1] << 16, h[1] >> 16 | l[1] & 0xffff0000u};
    }
};
// ... and where it goes nowhere else, as words
template <typename E>
struct Words {
    unsigned* p;
    int ld;
    __device__ __forceinline__ void put(int row, int col, float x) const
    {
        if constexpr (sizeof(E) == 4) {
            p[row * ld + col] = __float_as_uint(x);
        } else {
            const bf16 h = (bf16)x, l = (bf16)(x - (float)h);
            p[row * ld + col] = __builtin_bit_cast(unsigned short, h) | (unsigned)__builtin_bit_cast(unsigned short, l) << 16;
        }
    }
    __device__ __forceinline__ u32x4 operator()(int t, int j) const { return *(const u32x4*)(p + t * ld + 4 * j); }
};

// T = (1 + A)^-1 of a chunk, A_ts = beta_t e^(gamma_t - gamma_s) k_t . k_s below the diagonal, from its keys in LDS; the first 256 threads of a workgroup
// work, all have to call.  sA: room for C (C + 4) floats, where T may be too.  fp32 throughout: blocks of 16 on the diagonal row by row, in place,
// those below by products with them.
template <typename E, int DK, int C, typename O>
__device__ __forceinline__ void chunk_inverse(const E* sK, int LK, const ChunkSteps<C>& st, float* sA, const O& T, int tid)
{
    constexpr int NB = C / 16, LA = C + 4;
    const int lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), q = lane >> 4, c = lane & 15;
    // A, sixteen tokens to a wave
    if (w < NB) {
        const int t = 16 * w + c;
        for (int sb = 0; sb <= w; ++sb) {
            f32x4 x = zero4();
#pragma unroll
            for (int ks = 0; ks < DK / 32; ++ks) x = mma(rows_op(sK, LK, 16 * sb, 32 * ks, lane), rows_op(sK, LK, 16 * w, 32 * ks, lane), x);
            x *= splat4(st.beta[t]) * st.decays_from(t, 16 * sb + 4 * q);
            if (sb == w)
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = 4 * q + i < c ? x[i] : 0.f;
            *(f32x4*)(sA + t * LA + 16 * sb + 4 * q) = x;
        }
    }
    __syncthreads();
    // the inverses of 1 + A's blocks on the diagonal, a lane to a column: x_i = e_i - sum_{j<i} A_ij x_j.  (One wave: a row is written when it has
    // been read for the last time.)
    if (tid < C) {
        float* A = sA + 16 * q * LA + 16 * q;
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float s = i == c ? 1.f : 0.f;
#pragma unroll
            for (int j4 = 0; j4 < (i + 3) / 4; ++j4) {
                const f32x4 r = *(const f32x4*)(A + i * LA + 4 * j4);
#pragma unroll
                for (int j = 0; j < 4; ++j) if (4 * j4 + j < i) s = fmaf(-r[j], x[4 * j4 + j], s);
            }
            x[i] = s;
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < 16; ++i) A[i * LA + c] = x[i];
    }
    __syncthreads();
    // the blocks below it, a wave to a column of blocks: T_rj = -T_rr sum_{j<=b<r} A_rb T_bj, fp32 products
    f32x4 t[NB];
    if (w < NB) {
#pragma unroll
        for (int r = 0; r < NB; ++r) {
            t[r] = zero4();
            if (r == w) {
#pragma unroll
                for (int i = 0; i < 4; ++i) t[r][i] = sA[(16 * r + 4 * q + i) * LA + 16 * r + c];
            } else if (r > w) {
                f32x4 x = zero4();
#pragma unroll
                for (int b = 0; b < r; ++b)
                    if (b >= w) {
                        const f32x4 m = *(const f32x4*)(sA + (16 * r + c) * LA + 16 * b + 4 * q);
#pragma unroll
                        for (int i = 0; i < 4; ++i) x = __builtin_amdgcn_mfma_f32_16x16x4f32(m[i], t[b][i], x, 0, 0, 0);
                    }
                const f32x4 m = *(const f32x4*)(sA + (16 * r + c) * LA + 16 * r + 4 * q);
#pragma unroll
                for (int i = 0; i < 4; ++i) t[r] = __builtin_amdgcn_mfma_f32_16x16x4f32(-m[i], x[i], t[r], 0, 0, 0);
            }
        }
    }
    __syncthreads();
    if (w < NB) {
#pragma unroll
        for (int r = 0; r < NB; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i) T.put(16 * r + 4 * q + i, 16 * w + c, t[r][i]);
    }
    __syncthreads();
}
// Elements behind a row of T where it is worked out (half as many as behind other tiles' rows, so that a fourth workgroup fits in a compute unit), and the
// room, in elements, for either.
template <typename E> constexpr int kPadT = sizeof(E) == 2 ? 8 : 4;
template <typename E> constexpr int inverse_room()
{
    constexpr int C = DeltaChunk<E>::C, t = (sizeof(E) == 2 ? 2 : 1) * C * (C + kPadT<E>), a = C * (C + 4) * 4 / sizeof(E);
    return t > a ? t : a;
}
// Elements of a tile of scores or of T, its two parts.
template <typename E> constexpr int kScores = (sizeof(E) == 2 ? 2 : 1) * DeltaChunk<E>::C * (DeltaChunk<E>::C + kPad<E>);

// RUN(element type, DK, DV) for a call's.
#define CHELA_DELTA(RUN)                                                                                              \
    if (dtype != 0) { if (dk == 64) { if (dv == 64) RUN(float, 64, 64); else RUN(float, 64, 128); }                   \
                      else { if (dv == 64) RUN(float, 128, 64); else RUN(float, 128, 128); } }                        \
    else { if (dk == 64) { if (dv == 64) RUN(bf16, 64, 64); else RUN(bf16, 64, 128); }                                \
           else { if (dv == 64) RUN(bf16, 128, 64); else RUN(bf16, 128, 128); } }

}  // namespace chela
