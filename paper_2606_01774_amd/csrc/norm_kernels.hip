// norm_kernels.hip -- the forward of the norms around a mixer: norm behind it, gate, scale, residual,
// norm in front of the next, in one pass over the row (include/bdgdn.h, bdgdn_norm_fwd).
#include "norm.hpp"

namespace bdgdn {

namespace {

constexpr unsigned kMostGroups = 1u << 21;   // (a launch has 2^32 threads)

template <typename X, typename R, typename Y, int LANES, int C, bool WIDE>
__global__ void __launch_bounds__(LANES > 256 ? LANES : 256) bdgdn_norm_fwd_kernel(NormArgs a)
{
    constexpr int THREADS = LANES > 256 ? LANES : 256;
    __shared__ float lds[2 * (THREADS / 64)];
    RowSum<LANES, THREADS, 1> row_sum(lds);
    const int lane = threadIdx.x % LANES;
    for (unsigned row0 = blockIdx.x * (THREADS / LANES); row0 < (unsigned)a.rows; row0 += gridDim.x * (THREADS / LANES)) {
        const unsigned row = row0 + row_of<LANES>();
        const bool there = row < (unsigned)a.rows;   // (sums meet at barriers)
        const int d = there ? a.d : 0, ra = there ? row / (unsigned)a.inner : 0, rb = there ? row - ra * (unsigned)a.inner : 0;
        float x[C][8], z[C][8], r[C][8];
        Ahead<WIDE, LANES, C, X> ax;
        Ahead<WIDE, LANES, C, Y> az;
        Ahead<WIDE, LANES, C, R> ar;
        ax.load(row_at<X>(a.x, a.sx, ra, rb), d, lane);
        if (a.z) az.load(row_at<Y>(a.z, a.sz, ra, rb), d, lane);
        if (a.r) ar.load(row_at<R>(a.r, a.sr, ra, rb), d, lane);
        ax.get(x);
        if (a.z) az.get(z);
        if (a.r) ar.get(r);
        if (a.post) {
            float sum[1] = {0.f};
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[0] = fmaf(x[c][i], x[c][i], sum[0]);
            row_sum(sum);
            const float s1 = 1.f / sqrtf(fmaf(sum[0], a.inv_d, a.eps));
            float w[C][8];
            if (a.w_post) load_row<WIDE, LANES>(w, a.w_post, d, lane);
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) x[c][i] *= a.w_post ? s1 * w[c][i] : s1;
        }
        if (a.z) {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float g = a.act ? sigmoid(z[c][i]) : z[c][i];
                    x[c][i] *= a.act == kActSilu ? z[c][i] * g : g;
                }
        }
        {
            float w[C][8];
            if (a.ls) load_row<WIDE, LANES>(w, a.ls, d, lane);
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x[c][i] *= a.ls ? a.scale * w[c][i] : a.scale;
                    if (a.r) x[c][i] += r[c][i];
                }
        }
        if (a.r_out) store_row<WIDE, LANES>(row_at<R>(a.r_out, a.sro, ra, rb), x, d, lane);
        if (!a.y) continue;
        if (a.pre) {
            float sum[1] = {0.f};
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[0] = fmaf(x[c][i], x[c][i], sum[0]);
            row_sum(sum);
            const float s2 = 1.f / sqrtf(fmaf(sum[0], a.inv_d, a.eps));
            float w[C][8];
            if (a.w_pre) load_row<WIDE, LANES>(w, a.w_pre, d, lane);
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) x[c][i] *= a.w_pre ? s2 * w[c][i] : s2;
        }
        store_row<WIDE, LANES>(row_at<Y>(a.y, a.sy, ra, rb), x, d, lane);
    }
}

template <typename X, typename R, typename Y, int LANES, int C> hipError_t launch(const NormArgs &a, hipStream_t s)
{
    constexpr int THREADS = LANES > 256 ? LANES : 256, ROWS = THREADS / LANES;
    const unsigned groups = ((unsigned)a.rows + ROWS - 1) / ROWS, grid = groups < kMostGroups ? groups : kMostGroups;
    if (a.vec) bdgdn_norm_fwd_kernel<X, R, Y, LANES, C, true><<<grid, THREADS, 0, s>>>(a);
    else bdgdn_norm_fwd_kernel<X, R, Y, LANES, C, false><<<grid, THREADS, 0, s>>>(a);
    return hipGetLastError();
}

template <typename X, typename R, typename Y> hipError_t sized(const NormArgs &a, hipStream_t s)
{
    if (a.d <= 128) return launch<X, R, Y, 16, 1>(a, s);
    if (a.d <= 512) return launch<X, R, Y, 64, 1>(a, s);
    if (a.d <= 2048) return launch<X, R, Y, 256, 1>(a, s);
    if (a.d <= 4096) return launch<X, R, Y, 256, 2>(a, s);
    if (a.d <= 8192) return launch<X, R, Y, 1024, 1>(a, s);
    return launch<X, R, Y, 1024, 2>(a, s);
}

}  // namespace

hipError_t launch_norm_fwd(bool xf, bool rf, bool yf, NormArgs &a, hipStream_t s)
{
    if (yf) return sized<float, float, float>(a, s);
    if (xf) return rf ? sized<float, float, __bf16>(a, s) : sized<float, __bf16, __bf16>(a, s);
    return rf ? sized<__bf16, float, __bf16>(a, s) : sized<__bf16, __bf16, __bf16>(a, s);
}

}  // namespace bdgdn
