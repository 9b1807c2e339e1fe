// norm_kernels.hip -- the forward of the norms around a mixer: norm behind it, gate, scale, residual,
// norm in front of the next, in one pass over the row (include/bdgdn.h, bdgdn_norm_fwd).
//
// Bound by memory: 16384 rows of 4096 with gate and fp32 residual 177 us, 940 MB at 5.3 TB/s (a copy of 512
// MB: 5.4); rows of 8192 5.2, of 1024 5.2, of 4091 4.8, heads of 128 with their gate 5.2, of 100 2.8 (16384 x 16 of
// them in fp32 74 us: the last 4 elements of each go one at a time), of 64 and 256 in bf16 4.2 (rows get as many lanes as they fill: 16 and 64 lanes to them take 1.7 times as long).  One row of 4096 3.5 us,
// of which a launch is two.  Without a bound on registers: one that lets six waves share a SIMD keeps loads
// from overlapping (rows of 1024: 94 us without, 170 with).
#include "norm.hpp"

namespace bdgdn {

namespace {

// Threads of a workgroup whose rows have LANES lanes, and of a compute unit, which keeps them for many rows
// (so the weights are read once, and the next row while this one is worked on).
constexpr int threads_of(int lanes) { return lanes < 256 ? 256 : lanes; }
constexpr int kPerUnit = 1024;

template <typename X, typename R, typename Y, int LANES, int C, bool WHOLE> struct FwdRows {
    Ahead<WHOLE, LANES, C, X> x;
    Ahead<WHOLE, LANES, C, Y> z;
    Ahead<WHOLE, LANES, C, R> r;
    __device__ __forceinline__ void load(const NormArgs &a, unsigned row, int lane)
    {
        const int d = row < (unsigned)a.rows ? a.d : 0;
        const int ra = d ? row / (unsigned)a.inner : 0, rb = d ? row - ra * (unsigned)a.inner : 0;
        x.load(row_at<X>(a.x, a.sx, ra, rb), d, lane);
        if (a.z) z.load(row_at<Y>(a.z, a.sz, ra, rb), d, lane);
        if (a.r) r.load(row_at<R>(a.r, a.sr, ra, rb), d, lane);
    }
};

template <typename X, typename R, typename Y, int LANES, int C, bool WHOLE>
__global__ void __launch_bounds__(threads_of(LANES)) bdgdn_norm_fwd_kernel(NormArgs a)
{
    constexpr int THREADS = threads_of(LANES), ROWS = THREADS / LANES;
    constexpr bool AHEAD = C == 1;   // the next row loaded ahead
    __shared__ float lds[2 * (THREADS / 64)];
    RowSum<LANES, THREADS, 1> row_sum(lds);
    const int lane = threadIdx.x % LANES;
    const unsigned stride = gridDim.x * ROWS, mine = row_of<LANES>();
    FwdRows<X, R, Y, LANES, C, WHOLE> next;
    next.load(a, blockIdx.x * ROWS + mine, lane);
    float w_post[C][8], w_pre[C][8], ls[C][8];
    if (a.w_post) load_row<WHOLE, LANES>(w_post, a.w_post, a.d, lane);
    if (a.ls) load_row<WHOLE, LANES>(ls, a.ls, a.d, lane);
    if (a.w_pre) load_row<WHOLE, LANES>(w_pre, a.w_pre, a.d, lane);
    for (unsigned row0 = blockIdx.x * ROWS; row0 < (unsigned)a.rows; row0 += stride) {
        const unsigned row = row0 + mine;
        const bool there = row < (unsigned)a.rows;   // (sums meet at barriers)
        const int d = there ? a.d : 0, ra = there ? row / (unsigned)a.inner : 0, rb = there ? row - ra * (unsigned)a.inner : 0;
        float x[C][8], z[C][8], r[C][8];
        next.x.get(x, d, lane);
        if (a.z) next.z.get(z, d, lane);
        if (a.r) next.r.get(r, d, lane);
        if (AHEAD) next.load(a, row + stride, lane);
        float s1 = 1.f, s2 = 1.f;
        if (a.post) {
            float sum[1] = {0.f};
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[0] = fmaf(x[c][i], x[c][i], sum[0]);
            row_sum(sum);
            s1 = 1.f / sqrtf(fmaf(sum[0], a.inv_d, a.eps));
        }
        float sum[1] = {0.f};
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float u = a.post ? x[c][i] * s1 : x[c][i];
                if (a.w_post) u *= w_post[c][i];
                if (a.z) {
                    const float g = a.act ? sigmoid(z[c][i]) : z[c][i];
                    u *= a.act == kActSilu ? z[c][i] * g : g;
                }
                u *= a.scale;
                if (a.ls) u *= ls[c][i];
                if (a.r) u += r[c][i];
                x[c][i] = u;
                sum[0] = fmaf(u, u, sum[0]);
            }
        if (a.r_out) store_row<WHOLE, LANES>(row_at<R>(a.r_out, a.sro, ra, rb), x, d, lane);
        if (a.y) {
            if (a.pre) {
                row_sum(sum);
                s2 = 1.f / sqrtf(fmaf(sum[0], a.inv_d, a.eps));
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[c][i] *= a.w_pre ? s2 * w_pre[c][i] : s2;
            }
            store_row<WHOLE, LANES>(row_at<Y>(a.y, a.sy, ra, rb), x, d, lane);
        }
        if (!AHEAD) next.load(a, row + stride, lane);
    }
}

template <typename X, typename R, typename Y, int LANES, int C> hipError_t launch(const NormArgs &a, hipStream_t s)
{
    constexpr int THREADS = threads_of(LANES), ROWS = THREADS / LANES, MOST = 256 * kPerUnit / THREADS;
    const unsigned groups = ((unsigned)a.rows + ROWS - 1) / ROWS, grid = groups < MOST ? groups : MOST;
    if (a.d % 8 == 0) bdgdn_norm_fwd_kernel<X, R, Y, LANES, C, true><<<grid, THREADS, 0, s>>>(a);
    else bdgdn_norm_fwd_kernel<X, R, Y, LANES, C, false><<<grid, THREADS, 0, s>>>(a);
    return hipGetLastError();
}

template <typename X, typename R, typename Y> hipError_t sized(const NormArgs &a, hipStream_t s)
{
    if (a.d <= 64) return launch<X, R, Y, 8, 1>(a, s);
    if (a.d <= 128) return launch<X, R, Y, 16, 1>(a, s);
    if (a.d <= 256) return launch<X, R, Y, 32, 1>(a, s);
    if (a.d <= 512) return launch<X, R, Y, 64, 1>(a, s);
    if (a.d <= 1024) return launch<X, R, Y, 128, 1>(a, s);
    if (a.d <= 2048) return launch<X, R, Y, 256, 1>(a, s);
    if (a.d <= 4096) return launch<X, R, Y, 512, 1>(a, s);
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
