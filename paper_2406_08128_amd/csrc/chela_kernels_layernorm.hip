// Layer norm behind the residual's addition, in one pass over the rows, gfx950.
//
//     X' = X + Y  (Y null: X),   N = n w + b,   n = (X' - m) s,   m = mean X',   s = 1 / sqrt(mean (X' - m)^2 + eps).
// Gradient, from X' (its statistics are worked out again), with v = dN w:
//     dX = dX' + s (v - mean v - n mean(v n)),   dw = sum dN n,   db = sum dN.
// Memory-bound: a row stays in the registers of TPR threads, so every tensor is read or written once; the squares are taken behind the mean, from
// what is left of the row without it (a difference of two sums would lose the digits that a stream far from zero has in common), and what of
// the mean is left there, off as it is by its own rounding, goes with the same sums.
// 65536 rows of 768, bf16: forward 64 us (6.3 TB/s), gradient 77 (5.2), its sums 5; 6007 rows of 1531, fp32: 24 and 25 us (6.0, much of it in
// the cache in front of the memory), the stream in fp32 beside bf16 23.
#include "chela_rowparts.h"

namespace chela {

// Elements of a thread's share that lie in the row: the rest count for nothing in sums of what is zero for no reason of its own.
template <int TPR, int NV, bool VEC>
__device__ __forceinline__ void only_in_row(int D, int tid, float (&x)[NV * 4 + !VEC])
{
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int k = (v * TPR + tid) * 4;
        const bool in = VEC ? k < D : k + 4 <= D;
#pragma unroll
        for (int j = 0; j < 4; ++j) x[4 * v + j] = in ? x[4 * v + j] : 0.f;
    }
    if (!VEC) x[NV * 4] = tid < D % 4 ? x[NV * 4] : 0.f;
}

// A workgroup goes over every gridDim.x-th set of rows, the next row on its way while it works on one.
template <typename IO, typename XT, int TPR, int NV, bool VEC>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void layer_norm_kernel(LayerNormArgs a)
{
    typedef RowPart<IO, TPR, NV, VEC> P;
    typedef RowPart<XT, TPR, NV, VEC> PX;
    typedef RowPart<float, TPR, NV, VEC> PW;
    constexpr int E = P::E, RPW = TPR < 256 ? 256 / TPR : 1;
    __shared__ float s_a[TPR / 64][1], s_b[TPR / 64][2];
    const int tid = threadIdx.x % TPR, D = a.D;
    const float inv = 1.f / (float)D;
    float w[E], b[E];
#pragma unroll
    for (int e = 0; e < E; ++e) { w[e] = 1.f; b[e] = 0.f; }
    typename P::Raw ny;
    typename PX::Raw nx;
    auto load = [&](long r) {
        const size_t o = (size_t)r * D;
        PX::load((const XT*)a.X + o, D, tid, nx);
        if (a.Y) P::load((const IO*)a.Y + o, D, tid, ny);
    };
    const long step = (long)gridDim.x * RPW;
    long r = (long)blockIdx.x * RPW + threadIdx.x / TPR;
    if (r < a.rows) load(r);
    if (a.w) PW::load(a.w, D, tid, w);
    if (a.b) PW::load(a.b, D, tid, b);
    for (; r < a.rows; r += step) {                            // (with several waves to a row they all have the same rows)
        float x[E], sum[1];
        PX::widen(nx, x);
        if (a.Y) {
            float y[E];
            P::widen(ny, y);
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] += y[e];
        }
        if (r + step < a.rows) load(r + step);
        if (a.Y) PX::store((XT*)a.X_out + (size_t)r * D, D, tid, x);
        sum[0] = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) sum[0] += x[e];
        row_sums<TPR, 1>(sum, s_a);
        const float m = sum[0] * inv;
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] -= m;
        only_in_row<TPR, NV, VEC>(D, tid, x);
        float sums[2] = {0.f, 0.f};
#pragma unroll
        for (int e = 0; e < E; ++e) {
            sums[0] += x[e];
            sums[1] = fmaf(x[e], x[e], sums[1]);
        }
        row_sums<TPR, 2>(sums, s_b);
        const float left = sums[0] * inv, s = __builtin_amdgcn_rsqf(fmaxf(fmaf(sums[1], inv, -left * left), 0.f) + a.eps);
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = fmaf((x[e] - left) * s, w[e], b[e]);
        P::store((IO*)a.Nrm + (size_t)r * D, D, tid, x);
        // (a wave writes its sums of the next row only after all waves have read those of this one)
        if (TPR > 64) __syncthreads();
    }
}

// The same way over the rows; the sums of the gains' gradients stay in registers and leave once.
template <typename IO, typename XT, int TPR, int NV, bool VEC>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void layer_norm_bwd_kernel(LayerNormArgs a)
{
    typedef RowPart<IO, TPR, NV, VEC> P;
    typedef RowPart<XT, TPR, NV, VEC> PX;
    typedef RowPart<float, TPR, NV, VEC> PW;
    constexpr int E = P::E, RPW = TPR < 256 ? 256 / TPR : 1;
    constexpr bool AHEAD = NV < 4 || sizeof(IO) == 2; // (there are registers for the next row)
    __shared__ float s_a[TPR / 64][2], s_b[TPR / 64][3], s_w[2][RPW > 1 ? TPR * E : 1];
    const int tid = threadIdx.x % TPR, D = a.D;
    const float inv = 1.f / (float)D;
    float w[E], dw[E], db[E];
#pragma unroll
    for (int e = 0; e < E; ++e) { w[e] = 1.f; dw[e] = db[e] = 0.f; }
    if (a.w) PW::load(a.w, D, tid, w);
    typename P::Raw nd;
    typename PX::Raw nx, nu;
    auto load = [&](long r) {
        const size_t o = (size_t)r * D;
        PX::load((const XT*)a.X + o, D, tid, nx);
        P::load((const IO*)a.dN + o, D, tid, nd);
        if (a.dX_out) PX::load((const XT*)a.dX_out + o, D, tid, nu);
    };
    const long step = (long)gridDim.x * RPW;
    long r = (long)blockIdx.x * RPW + threadIdx.x / TPR;
    if (AHEAD && r < a.rows) load(r);
    for (; r < a.rows; r += step) {
        if (!AHEAD) load(r);
        float x[E], d[E], dx[E], sums[2] = {0.f, 0.f};
        PX::widen(nx, x);
        P::widen(nd, d);
        if (a.dX_out) {
            PX::widen(nu, dx);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) dx[e] = 0.f;
        }
        if (AHEAD && r + step < a.rows) load(r + step);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            sums[0] += x[e];
            sums[1] = fmaf(d[e], w[e], sums[1]);
        }
        row_sums<TPR, 2>(sums, s_a);
        const float m = sums[0] * inv, mv = sums[1] * inv;
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] -= m;
        only_in_row<TPR, NV, VEC>(D, tid, x);
        float three[3] = {0.f, 0.f, 0.f};
#pragma unroll
        for (int e = 0; e < E; ++e) {
            three[0] += x[e];
            three[1] = fmaf(x[e], x[e], three[1]);
            three[2] = fmaf(d[e] * w[e], x[e], three[2]);
        }
        row_sums<TPR, 3>(three, s_b);
        const float left = three[0] * inv, s = __builtin_amdgcn_rsqf(fmaxf(fmaf(three[1], inv, -left * left), 0.f) + a.eps);
        const float mvn = fmaf(three[2], inv, -left * mv) * s;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float n = (x[e] - left) * s;
            dw[e] = fmaf(d[e], n, dw[e]);
            db[e] += d[e];
            dx[e] = fmaf(s, fmaf(-n, mvn, fmaf(d[e], w[e], -mv)), dx[e]);
        }
        PX::store((XT*)a.dX + (size_t)r * D, D, tid, dx);
        // (a wave writes its sums of the next row only after all waves have read those of this one)
        if (TPR > 64) __syncthreads();
    }
    if (a.part == nullptr) return;
    float* part = a.part + (size_t)blockIdx.x * 2 * D;
    if (RPW > 1) {
        // the waves of the workgroup, one after the other
        for (int v = 0; v < RPW; ++v) {
            if ((int)(threadIdx.x / TPR) == v) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    s_w[0][e * TPR + tid] = dw[e] + (v ? s_w[0][e * TPR + tid] : 0.f);
                    s_w[1][e * TPR + tid] = db[e] + (v ? s_w[1][e * TPR + tid] : 0.f);
                }
            }
            __syncthreads();
        }
        if (threadIdx.x >= TPR) return;
#pragma unroll
        for (int e = 0; e < E; ++e) { dw[e] = s_w[0][e * TPR + tid]; db[e] = s_w[1][e * TPR + tid]; }
    }
    PW::store(part, D, tid, dw);
    PW::store(part + D, D, tid, db);
}

// The workgroups' sums, sixteen waves to 64 features.
__global__ __launch_bounds__(1024) void layer_norm_sum_kernel(LayerNormArgs a, int parts)
{
    __shared__ float s_sum[16][64];
    const int lane = threadIdx.x & 63, i = blockIdx.x * 64 + lane, k = blockIdx.y, w = threadIdx.x >> 6;
    float* to = k == 0 ? a.dw : a.db;
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
// A row to a wave where it fits its registers: with 256 threads to a row of 768 (65536 rows, bf16) forward 79 us and gradient 148 instead of 71 and 80, to
// one of 1024 60 and 88 instead of 60 and 65; a wave to 2048 features 92 and 104 instead of 92 and 99.  1024 threads to a row of 8192, bf16,
// 73 and 113 instead of 74 and 84.
static int rows_per_group(int D) { return D <= 1024 ? 4 : 1; }

// Workgroups, of the gradient at most (256, 512, 1024 of them, us): rows of 768 88 80 86, of 1531 37 29 33, of 64 45 29 26, of 8192 78 84 99; of the
// forward (1024, 2048, 8192): 77 76 71, 24 24 25, 15 14 14, 72 73 74.
constexpr int kNormParts = 512, kNormGroups = 8192;
int layer_norm_bwd_parts(long rows, int D)
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

hipError_t launch_layer_norm_fwd(const LayerNormArgs& a, int dtype, hipStream_t st)
{
    ProfScope prof(KID_LAYER_NORM, st);
    const long sets = (a.rows + rows_per_group(a.D) - 1) / rows_per_group(a.D);
    const dim3 grid((unsigned)(sets < kNormGroups ? sets : kNormGroups));
#define CHELA_F(IO, XT, TPR, NV, VEC)                                                                                 \
    hipLaunchKernelGGL((layer_norm_kernel<IO, XT, TPR, NV, VEC>), grid, dim3(TPR < 256 ? 256 : TPR), 0, st, a)
    if (a.D % 4 == 0) { CHELA_TYPES(true) } else { CHELA_TYPES(false) }
#undef CHELA_F
    return hipGetLastError();
}

hipError_t launch_layer_norm_bwd(const LayerNormArgs& a, int dtype, hipStream_t st)
{
    ProfScope prof(KID_LAYER_NORM, st);
    const int parts = layer_norm_bwd_parts(a.rows, a.D);
    const dim3 grid(parts);
#define CHELA_F(IO, XT, TPR, NV, VEC)                                                                                 \
    hipLaunchKernelGGL((layer_norm_bwd_kernel<IO, XT, TPR, NV, VEC>), grid, dim3(TPR < 256 ? 256 : TPR), 0, st, a)
    if (a.D % 4 == 0) { CHELA_TYPES(true) } else { CHELA_TYPES(false) }
#undef CHELA_F
    if (a.part != nullptr)
        hipLaunchKernelGGL(layer_norm_sum_kernel, dim3((a.D + 63) / 64, 2), dim3(1024), 0, st, a, parts);
    return hipGetLastError();
}

}  // namespace chela
