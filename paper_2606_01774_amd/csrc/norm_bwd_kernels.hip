// norm_bwd_kernels.hip -- the backward of the norms around a mixer (include/bdgdn.h, bdgdn_norm_bwd).
//
// With xh = x / rms(x), n = xh w_post, u = n act(z), r' = r + s l u, h = r' / rms(r'), y = h w_pre
// and upstream gradients dy, dr':
//     t = dy w_pre,  g = dr' + (t - h mean(t h)) / rms(r')          dr = g,  dw_pre = sum dy h
//     dl = sum s g u,  du = s l g,  dz = du n act'(z),  dn = du act(z)
//     t = dn w_post,  dx = (t - xh mean(t xh)) / rms(x)             dw_post = sum dn xh
// (without a norm its line is the identity).  A row's lanes hold it in registers through both
// norms; the weights' sums stay in registers over a workgroup's rows, and the workgroups' sums meet
// in a second kernel, in order.
#include "norm.hpp"

namespace bdgdn {

namespace {

constexpr int kThreads = 1024;

template <typename X, typename R, typename Y, int LANES, int C, bool WIDE>
__global__ void __launch_bounds__(kThreads) bdgdn_norm_bwd_kernel(NormArgs a)
{
    constexpr int ROWS = kThreads / LANES;
    constexpr int UNITS = LANES < 64 ? kThreads / 64 : ROWS;   // that hold sums of the same elements
    __shared__ float lds[3 * (kThreads / 64)];
    __shared__ float meet[UNITS > 1 ? UNITS * LANES * 8 : 1];
    const int lane = threadIdx.x % LANES;
    float wp[C][8], wq[C][8], ls[C][8];
    if (a.w_post) load_row<WIDE, LANES>(wp, a.w_post, a.d, lane);
    if (a.w_pre) load_row<WIDE, LANES>(wq, a.w_pre, a.d, lane);
    if (a.ls) load_row<WIDE, LANES>(ls, a.ls, a.d, lane);
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (!a.w_post) wp[c][i] = 1.f;
            if (!a.w_pre) wq[c][i] = 1.f;
            ls[c][i] = a.ls ? a.scale * ls[c][i] : a.scale;
        }
    float acc[3][C][8] = {};   // of w_post, w_pre, layer_scale

    for (unsigned row0 = blockIdx.x * ROWS; row0 < (unsigned)a.rows; row0 += gridDim.x * ROWS) {
        const unsigned row = row0 + threadIdx.x / LANES;
        const bool there = row < (unsigned)a.rows;   // (sums meet at barriers)
        const int d = there ? a.d : 0, ra = there ? row / (unsigned)a.inner : 0, rb = there ? row - ra * (unsigned)a.inner : 0;
        float x[C][8], z[C][8], sum_r[C][8], dy[C][8], g[C][8];
        load_row<WIDE, LANES>(x, row_at<X>(a.x, a.sx, ra, rb), d, lane);
        if (a.z) load_row<WIDE, LANES>(z, row_at<Y>(a.z, a.sz, ra, rb), d, lane);
        if (a.r) load_row<WIDE, LANES>(sum_r, row_at<R>(a.r, a.sro, ra, rb), d, lane);
        load_row<WIDE, LANES>(dy, row_at<Y>(a.dy, a.sdy, ra, rb), a.dy ? d : 0, lane);
        load_row<WIDE, LANES>(g, row_at<R>(a.dr_out, a.sdro, ra, rb), a.dr_out ? d : 0, lane);
        float s1 = 1.f, s2 = 1.f, mean_t = 0.f;
        const bool joint = a.pre && a.r;
        if (a.post || joint) {
            float sum[3] = {0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    sum[0] = fmaf(x[c][i], x[c][i], sum[0]);
                    if (joint) {
                        sum[1] = fmaf(sum_r[c][i], sum_r[c][i], sum[1]);
                        sum[2] = fmaf(dy[c][i] * wq[c][i], sum_r[c][i], sum[2]);
                    }
                }
            row_sum<LANES, kThreads>(sum, lds);
            if (a.post) s1 = 1.f / sqrtf(fmaf(sum[0], a.inv_d, a.eps));
            if (joint) {
                s2 = 1.f / sqrtf(fmaf(sum[1], a.inv_d, a.eps));
                mean_t = sum[2] * s2 * a.inv_d;
            }
        }
        if (a.pre && !a.r) {   // r' = s l u
            float sum[2] = {0.f, 0.f};
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    float u = a.post ? x[c][i] * s1 * wp[c][i] : x[c][i];
                    if (a.z) {
                        const float e = a.act ? sigmoid(z[c][i]) : z[c][i];
                        u *= a.act == kActSilu ? z[c][i] * e : e;
                    }
                    sum_r[c][i] = u * ls[c][i];
                    sum[0] = fmaf(sum_r[c][i], sum_r[c][i], sum[0]);
                    sum[1] = fmaf(dy[c][i] * wq[c][i], sum_r[c][i], sum[1]);
                }
            row_sum<LANES, kThreads>(sum, lds);
            s2 = 1.f / sqrtf(fmaf(sum[0], a.inv_d, a.eps));
            mean_t = sum[1] * s2 * a.inv_d;
        }
        float sum[1] = {0.f};
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (a.pre) {
                    const float h = sum_r[c][i] * s2;
                    if (there) acc[1][c][i] = fmaf(dy[c][i], h, acc[1][c][i]);
                    g[c][i] += s2 * (dy[c][i] * wq[c][i] - h * mean_t);
                } else {
                    g[c][i] += dy[c][i];
                }
                const float xh = a.post ? x[c][i] * s1 : x[c][i], n = a.post ? xh * wp[c][i] : xh;
                float act = 1.f, slope = 0.f;
                if (a.z) {
                    const float e = a.act ? sigmoid(z[c][i]) : z[c][i];
                    act = a.act == kActSilu ? z[c][i] * e : e;
                    slope = a.act == kActSilu ? e * (1.f + z[c][i] * (1.f - e)) : a.act ? e * (1.f - e) : 1.f;
                }
                if (there) acc[2][c][i] = fmaf(a.scale * g[c][i], n * act, acc[2][c][i]);
                const float du = ls[c][i] * g[c][i], dn = du * act;
                z[c][i] = du * n * slope;
                if (there) acc[0][c][i] = fmaf(dn, xh, acc[0][c][i]);
                x[c][i] = xh;
                dy[c][i] = a.post ? dn * wp[c][i] : dn;
                sum[0] = fmaf(dy[c][i], xh, sum[0]);
            }
        if (a.dr) store_row<WIDE, LANES>(row_at<R>(a.dr, a.sdr, ra, rb), g, d, lane);
        if (a.dz) store_row<WIDE, LANES>(row_at<Y>(a.dz, a.sdz, ra, rb), z, d, lane);
        if (!a.dx) continue;
        if (a.post) {
            row_sum<LANES, kThreads>(sum, lds);
            const float mean = sum[0] * a.inv_d;
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) dy[c][i] = s1 * (dy[c][i] - x[c][i] * mean);
        }
        store_row<WIDE, LANES>(row_at<X>(a.dx, a.sdx, ra, rb), dy, d, lane);
    }

    // the workgroup's sums
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        if (!a.dw[k]) continue;
        float *part = a.part + ((long)blockIdx.x * 3 + k) * a.d;
        if constexpr (UNITS == 1) {
            store_row<WIDE, LANES>(part, acc[k], a.d, lane);
        } else {
            static_assert(C == 1, "several rows to a workgroup have one chunk to a lane");
            const int unit = LANES < 64 ? threadIdx.x >> 6 : threadIdx.x / LANES;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float v = acc[k][0][i];
#pragma unroll
                for (int o = LANES; o < 64; o <<= 1) v += __shfl_xor(v, o);
                if (LANES >= 64 || (threadIdx.x & 63) < LANES) meet[unit * LANES * 8 + element<WIDE, LANES>(0, i, lane)] = v;
            }
            __syncthreads();
            for (int e = threadIdx.x; e < a.d; e += kThreads) {
                float v = 0.f;
                for (int u = 0; u < UNITS; ++u) v += meet[u * LANES * 8 + e];
                part[e] = v;
            }
        }
    }
}

// The workgroups' sums of 64 elements, sixteen lanes to an element.
__global__ void __launch_bounds__(1024) bdgdn_norm_weights_kernel(NormArgs a)
{
    __shared__ float lds[16][64];
    const int k = blockIdx.y, e = blockIdx.x * 64 + (threadIdx.x & 63), u = threadIdx.x >> 6;
    if (!a.dw[k]) return;
    float v = 0.f;
    if (e < a.d)
        for (int p = u; p < a.groups; p += 16) v += a.part[((long)p * 3 + k) * a.d + e];
    lds[u][threadIdx.x & 63] = v;
    __syncthreads();
    if (u == 0 && e < a.d) {
        for (int i = 1; i < 16; ++i) v += lds[i][threadIdx.x];
        a.dw[k][e] = v;
    }
}

template <typename X, typename R, typename Y, int LANES, int C> void launch(const NormArgs &a, hipStream_t s)
{
    if (a.vec) bdgdn_norm_bwd_kernel<X, R, Y, LANES, C, true><<<a.groups, kThreads, 0, s>>>(a);
    else bdgdn_norm_bwd_kernel<X, R, Y, LANES, C, false><<<a.groups, kThreads, 0, s>>>(a);
}

template <typename X, typename R, typename Y> hipError_t sized(const NormArgs &a, hipStream_t s)
{
    if (a.groups > 0) {
        if (a.d <= 128) launch<X, R, Y, 16, 1>(a, s);
        else if (a.d <= 512) launch<X, R, Y, 64, 1>(a, s);
        else if (a.d <= 2048) launch<X, R, Y, 256, 1>(a, s);
        else if (a.d <= 4096) launch<X, R, Y, 512, 1>(a, s);
        else if (a.d <= 8192) launch<X, R, Y, 1024, 1>(a, s);
        else launch<X, R, Y, 1024, 2>(a, s);
    }
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && (a.dw[0] || a.dw[1] || a.dw[2])) {
        bdgdn_norm_weights_kernel<<<dim3((a.d + 63) / 64, 3), 1024, 0, s>>>(a);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace

int norm_bwd_groups(int rows, int d)
{
    const int lanes = d <= 128 ? 16 : d <= 512 ? 64 : d <= 2048 ? 256 : d <= 4096 ? 512 : 1024, in_one = kThreads / lanes;
    const int groups = (int)(((long)rows + in_one - 1) / in_one);
    return groups < 512 ? groups : 512;
}

hipError_t launch_norm_bwd(bool xf, bool rf, bool yf, NormArgs &a, hipStream_t s)
{
    if (yf) return sized<float, float, float>(a, s);
    if (xf) return rf ? sized<float, float, __bf16>(a, s) : sized<float, __bf16, __bf16>(a, s);
    return rf ? sized<__bf16, float, __bf16>(a, s) : sized<__bf16, __bf16, __bf16>(a, s);
}

}  // namespace bdgdn
