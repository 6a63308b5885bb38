// Norms before and after a block with its gate and residual, in one pass over the rows, gfx950.
//
//     p = Norm(Y) w_post gate   (w_post null: Y gate),   X' = X + scale p,   N = Norm(X') w_pre;   Norm(x) = x / sqrt(mean x^2 + eps)
// Gradient, from Y, gate and X' (the norms are worked out again), with x^ = Norm(X'), v = dN w_pre, y^ = Norm(Y), s = 1 / sqrt(...):
//     dX = dX' + s (v - x^ mean(v x^)),  dw_pre = sum dN x^;   dp = scale dX,  dgate = dp y^ w_post,  dw_post = sum dp y^ gate,
//     dY = s (v - y^ mean(v y^)) with v = dp w_post gate.
//
// Memory-bound: a row stays in the registers of TPR threads between its two norms, so every tensor is read or written once.  65536 rows of
// 768, bf16: forward 90 us (5.6 TB/s; one row per wave and the gains with every row: 106), gradient 145 us (5.5 TB/s; without the next
// row on its way 271), with the stream in fp32 125 and 219 us (5.6 and 5.1 TB/s); 6007 rows of 1531, fp32: 34 and 53 us (5.5 TB/s).
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

// A workgroup goes over every gridDim.x-th set of rows, the next row on its way while it works on one: the gains, as many bytes as a bf16
// row's tensors have together, are read once.
template <typename IO, typename XT, int TPR, int NV, bool VEC>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void block_norm_kernel(BlockNormArgs a)
{
    typedef RowPart<IO, TPR, NV, VEC> P;
    typedef RowPart<XT, TPR, NV, VEC> PX;
    typedef RowPart<float, TPR, NV, VEC> PW;
    constexpr int E = P::E, RPW = TPR < 256 ? 256 / TPR : 1;
    __shared__ float s_a[TPR / 64][1], s_b[TPR / 64][1];
    const int tid = threadIdx.x % TPR, D = a.D;
    const float inv = 1.f / (float)D;
    float wpost[E], wpre[E];
    typename P::Raw ny, ng;
    typename PX::Raw nx;
    auto load = [&](long r) {
        const size_t o = (size_t)r * D;
        PX::load((const XT*)a.X + o, D, tid, nx);
        if (a.Y) P::load((const IO*)a.Y + o, D, tid, ny);
        if (a.Y && a.gate) P::load((const IO*)a.gate + o, D, tid, ng);
    };
    const long step = (long)gridDim.x * RPW;
    long r = (long)blockIdx.x * RPW + threadIdx.x / TPR;
    if (r < a.rows) load(r);
    if (a.w_post) PW::load(a.w_post, D, tid, wpost);
    if (a.w_pre) PW::load(a.w_pre, D, tid, wpre);
    for (; r < a.rows; r += step) {                            // (with several waves to a row they all have the same rows)
        float x[E], y[E], g[E], sum[1];
        PX::widen(nx, x);
        if (a.Y) P::widen(ny, y);
        if (a.Y && a.gate) P::widen(ng, g);
        if (r + step < a.rows) load(r + step);
        if (a.Y) {
            if (a.w_post) {
                sum[0] = 0.f;
#pragma unroll
                for (int e = 0; e < E; ++e) sum[0] = fmaf(y[e], y[e], sum[0]);
                row_sums<TPR, 1>(sum, s_a);
                const float s = __builtin_amdgcn_rsqf(fmaf(sum[0], inv, a.eps));
#pragma unroll
                for (int e = 0; e < E; ++e) y[e] *= s * wpost[e];
            }
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = fmaf(a.scale, a.gate ? y[e] * g[e] : y[e], x[e]);
            PX::store((XT*)a.X_out + (size_t)r * D, D, tid, x);
        }
        if (a.w_pre) {
            sum[0] = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) sum[0] = fmaf(x[e], x[e], sum[0]);
            row_sums<TPR, 1>(sum, s_b);
            const float s = __builtin_amdgcn_rsqf(fmaf(sum[0], inv, a.eps));
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] *= s * wpre[e];
            P::store((IO*)a.Nrm + (size_t)r * D, D, tid, x);
        }
        // (a wave writes its sums of the next row only after all waves have read those of this one)
        if (TPR > 64) __syncthreads();
    }
}

// The same way over the rows; the sums of the gains' gradients stay in registers and leave once.
template <typename IO, typename XT, int TPR, int NV, bool VEC>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void block_norm_bwd_kernel(BlockNormArgs a)
{
    typedef RowPart<IO, TPR, NV, VEC> P;
    typedef RowPart<XT, TPR, NV, VEC> PX;
    typedef RowPart<float, TPR, NV, VEC> PW;
    constexpr int E = P::E, RPW = TPR < 256 ? 256 / TPR : 1;
    constexpr bool AHEAD = NV < 4 || sizeof(IO) == 2; // (there are registers for the next row)
    __shared__ float s_a[TPR / 64][3], s_b[TPR / 64][1], s_w[2][RPW > 1 ? TPR * E : 1];
    const int tid = threadIdx.x % TPR, D = a.D;
    const float inv = 1.f / (float)D;
    float wpost[E], wpre[E], dwpost[E], dwpre[E];
#pragma unroll
    for (int e = 0; e < E; ++e) { wpost[e] = 1.f; dwpost[e] = dwpre[e] = 0.f; wpre[e] = 0.f; }
    if (a.w_post) PW::load(a.w_post, D, tid, wpost);
    if (a.w_pre) PW::load(a.w_pre, D, tid, wpre);
    typename P::Raw ny, ng, nd;
    typename PX::Raw nx, nu;
    auto load = [&](long r) {
        const size_t o = (size_t)r * D;
        PX::load((const XT*)a.X + o, D, tid, nx);
        if (a.w_pre) P::load((const IO*)a.dN + o, D, tid, nd);
        if (a.Y) P::load((const IO*)a.Y + o, D, tid, ny);
        if (a.Y && a.gate) P::load((const IO*)a.gate + o, D, tid, ng);
        if (a.dX_out) PX::load((const XT*)a.dX_out + o, D, tid, nu);
    };
    const long step = (long)gridDim.x * RPW;
    long r = (long)blockIdx.x * RPW + threadIdx.x / TPR;
    if (AHEAD && r < a.rows) load(r);
    for (; r < a.rows; r += step) {
        if (!AHEAD) load(r);
        float x[E], y[E], g[E], d[E], dx[E], sums[3] = {0.f, 0.f, 0.f}, sum[1] = {0.f};
        PX::widen(nx, x);
        if (a.w_pre) P::widen(nd, d);
        if (a.Y) P::widen(ny, y);
        if (a.Y && a.gate) P::widen(ng, g);
        if (a.dX_out) {
            PX::widen(nu, dx);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) dx[e] = 0.f;
        }
        if (AHEAD && r + step < a.rows) load(r + step);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (a.w_pre) {
                sums[0] = fmaf(x[e], x[e], sums[0]);
                sums[1] = fmaf(d[e] * wpre[e], x[e], sums[1]);
            }
            if (a.Y) sums[2] = fmaf(y[e], y[e], sums[2]);
        }
        row_sums<TPR, 3>(sums, s_a);
        const float sx = __builtin_amdgcn_rsqf(fmaf(sums[0], inv, a.eps)), mx = sums[1] * inv * sx;
        if (a.w_pre) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float n = x[e] * sx;
                dwpre[e] = fmaf(d[e], n, dwpre[e]);
                dx[e] = fmaf(sx, fmaf(-n, mx, d[e] * wpre[e]), dx[e]);
            }
        }
        PX::store((XT*)a.dX + (size_t)r * D, D, tid, dx);
        if (a.Y) {
            const float sy = a.w_post ? __builtin_amdgcn_rsqf(fmaf(sums[2], inv, a.eps)) : 1.f;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float dp = a.scale * dx[e], n = y[e] * sy, gate = a.gate ? g[e] : 1.f;
                dwpost[e] = fmaf(dp * n, gate, dwpost[e]);
                g[e] = dp * n * wpost[e];                        // dgate
                d[e] = dp * wpost[e] * gate;                     // v
                y[e] = n;
                sum[0] = fmaf(d[e], n, sum[0]);
            }
            if (a.gate) P::store((IO*)a.dgate + (size_t)r * D, D, tid, g);
            if (a.w_post) {
                row_sums<TPR, 1>(sum, s_b);
                const float my = sum[0] * inv;
#pragma unroll
                for (int e = 0; e < E; ++e) d[e] = sy * fmaf(-y[e], my, d[e]);
            }
            P::store((IO*)a.dY + (size_t)r * D, D, tid, d);
        }
        // (a wave writes its sums of the next row only after all waves have read those of this one)
        if (TPR > 64) __syncthreads();
    }
    float* part = a.part + (size_t)blockIdx.x * 2 * D;
    if (RPW > 1) {
        // the waves of the workgroup, one after the other
        for (int v = 0; v < RPW; ++v) {
            if ((int)(threadIdx.x / TPR) == v) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    s_w[0][e * TPR + tid] = dwpost[e] + (v ? s_w[0][e * TPR + tid] : 0.f);
                    s_w[1][e * TPR + tid] = dwpre[e] + (v ? s_w[1][e * TPR + tid] : 0.f);
                }
            }
            __syncthreads();
        }
        if (threadIdx.x >= TPR) return;
#pragma unroll
        for (int e = 0; e < E; ++e) { dwpost[e] = s_w[0][e * TPR + tid]; dwpre[e] = s_w[1][e * TPR + tid]; }
    }
    PW::store(part, D, tid, dwpost);
    PW::store(part + D, D, tid, dwpre);
}

// The workgroups' sums, sixteen waves to 64 features.
__global__ __launch_bounds__(1024) void block_norm_sum_kernel(BlockNormArgs a, int parts)
{
    __shared__ float s_sum[16][64];
    const int lane = threadIdx.x & 63, i = blockIdx.x * 64 + lane, k = blockIdx.y, w = threadIdx.x >> 6;
    float* to = k == 0 ? a.dw_post : a.dw_pre;
    if (to == nullptr) return;
    const float* from = a.part + (size_t)k * a.D + min(i, a.D - 1);
    float x = 0.f;
#pragma unroll 8
    for (int p = w; p < parts; p += 16) x += from[(size_t)p * 2 * a.D];
    s_sum[w][lane] = x;
    __syncthreads();
    if (w != 0 || i >= a.D) return;
    x = 0.f;
#pragma unroll
    for (int j = 0; j < 16; ++j) x += s_sum[j][lane];
    to[i] = x;
}

// -------------------------------------------------------------------------------------------------------------------- host
static int rows_per_group(int D) { return D <= 1024 ? 4 : 1; }

// Workgroups.  Gradient, 512, 768, 1024 of them (65536 rows of 768, bf16): 151 us and 5 for their sums, 168 and 7, 154 and 8.  Forward,
// 1024, 2048, 8192: 93, 90, 87 us.
constexpr int kNormParts = 512, kNormGroups = 8192;
int block_norm_bwd_parts(long rows, int D)
{
    const long sets = (rows + rows_per_group(D) - 1) / rows_per_group(D);
    return (int)(sets < 1 ? 1 : sets > kNormParts ? kNormParts : sets);
}

#define CHELA_ROWS(IO, XT, VEC)                                                                                       \
    if (a.D <= 256) CHELA_F(IO, XT, 64, 1, VEC);                                                                      \
    else if (a.D <= 512) CHELA_F(IO, XT, 64, 2, VEC);                                                                 \
    else if (a.D <= 768) CHELA_F(IO, XT, 64, 3, VEC);                                                                 \
    else if (a.D <= 1024) CHELA_F(IO, XT, 64, 4, VEC);                                                                \
    else if (a.D <= 2048) CHELA_F(IO, XT, 256, 2, VEC);                                                               \
    else if (a.D <= 4096) CHELA_F(IO, XT, 256, 4, VEC);                                                               \
    else CHELA_F(IO, XT, 512, 4, VEC);
#define CHELA_TYPES(VEC)                                                                                              \
    if (dtype != 0) { CHELA_ROWS(float, float, VEC) }                                                                 \
    else if (a.x_f32) { CHELA_ROWS(bf16, float, VEC) }                                                                \
    else { CHELA_ROWS(bf16, bf16, VEC) }

hipError_t launch_block_norm_fwd(const BlockNormArgs& a, int dtype, hipStream_t st)
{
    ProfScope prof(KID_BLOCK_NORM, st);
    const long sets = (a.rows + rows_per_group(a.D) - 1) / rows_per_group(a.D);
    const dim3 grid((unsigned)(sets < kNormGroups ? sets : kNormGroups));
#define CHELA_F(IO, XT, TPR, NV, VEC)                                                                                 \
    hipLaunchKernelGGL((block_norm_kernel<IO, XT, TPR, NV, VEC>), grid, dim3(TPR < 256 ? 256 : TPR), 0, st, a)
    if (a.D % 4 == 0) { CHELA_TYPES(true) } else { CHELA_TYPES(false) }
#undef CHELA_F
    return hipGetLastError();
}

hipError_t launch_block_norm_bwd(const BlockNormArgs& a, int dtype, hipStream_t st)
{
    ProfScope prof(KID_BLOCK_NORM, st);
    const int parts = block_norm_bwd_parts(a.rows, a.D);
    const dim3 grid(parts);
#define CHELA_F(IO, XT, TPR, NV, VEC)                                                                                 \
    hipLaunchKernelGGL((block_norm_bwd_kernel<IO, XT, TPR, NV, VEC>), grid, dim3(TPR < 256 ? 256 : TPR), 0, st, a)
    if (a.D % 4 == 0) { CHELA_TYPES(true) } else { CHELA_TYPES(false) }
#undef CHELA_F
    hipLaunchKernelGGL(block_norm_sum_kernel, dim3((a.D + 63) / 64, 2), dim3(1024), 0, st, a, parts);
    return hipGetLastError();
}

}  // namespace chela
