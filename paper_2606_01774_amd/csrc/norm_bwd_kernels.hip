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
//
// Bound by memory: 16384 rows of 4096 with gate and fp32 residual 273 us, 1476 MB at 5.4 TB/s, and 4.6 for the
// weights' sums (12.6 MB); 16384 x 16 heads of 128 with their gate 96 us, 470 MB at 4.9;
// bf16 heads of 64 and 256 86 us, 335 MB at 3.9, where the vector units are busy in 85 % of the cycles.  The 512 lanes of a
// workgroup take 150 to 180 registers each, so a compute unit has one, and what keeps memory busy is
// the next row, loaded while this one is worked on (443 us without it, in workgroups of 1024).  Twice the
// workgroups leave twice the partial sums, and take 293 us.  Rows of 8192 take two chunks to a lane, none
// ahead: 8192 x 8192 with gate and fp32 residual 361 us, 4.1 TB/s.  Beyond that the sums fill the registers and rows are
// read again from the caches, with spills: 4096 x 16384 1060 us, 1.4 TB/s.
#include "norm.hpp"

namespace bdgdn {

namespace {

constexpr int kThreads = 512;
constexpr int kMostGroups = 256;   // a workgroup to a compute unit

// A lane's parts of the five rows that a row's gradients come from.
template <typename X, typename R, typename Y, int LANES, int C, bool WHOLE> struct BwdRows {
    Ahead<WHOLE, LANES, C, X> x;
    Ahead<WHOLE, LANES, C, Y> z, dy;
    Ahead<WHOLE, LANES, C, R> sum_r, g;
    __device__ __forceinline__ void load(const NormArgs &a, unsigned row, int lane)
    {
        const int d = row < (unsigned)a.rows ? a.d : 0;
        const int ra = d ? row / (unsigned)a.inner : 0, rb = d ? row - ra * (unsigned)a.inner : 0;
        x.load(row_at<X>(a.x, a.sx, ra, rb), d, lane);
        if (a.pre && a.r) sum_r.load(row_at<R>(a.r, a.sro, ra, rb), d, lane);
        dy.load(row_at<Y>(a.dy, a.sdy, ra, rb), a.dy ? d : 0, lane);
        if (a.z) z.load(row_at<Y>(a.z, a.sz, ra, rb), d, lane);
        g.load(row_at<R>(a.dr_out, a.sdro, ra, rb), a.dr_out ? d : 0, lane);
    }
};

template <typename X, typename R, typename Y, int LANES, int C, bool WHOLE>
__global__ void __launch_bounds__(kThreads) bdgdn_norm_bwd_kernel(NormArgs a)
{
    // One or two chunks to a lane stay in registers, and beside one the next row's, loaded ahead; of more
    // each is read again (from the caches) where it is used.
    constexpr bool ONE = C == 1, HOLD = C <= 2;
    constexpr int H = HOLD ? C : 1;
    constexpr auto at = [](int c) { return HOLD ? c : 0; };
    constexpr int ROWS = kThreads / LANES;
    constexpr int UNITS = LANES < 64 ? kThreads / 64 : ROWS;   // that hold sums of the same elements
    __shared__ float lds[2 * 3 * (kThreads / 64)];
    RowSum<LANES, kThreads, 3> row_sum(lds);
    __shared__ float meet[UNITS > 1 ? UNITS * LANES * 8 : 1];
    const int lane = threadIdx.x % LANES;
    float wp[H][8], wq[H][8], ls[H][8];
    auto weights = [&](int c) {
        if (a.w_post) load_chunk<WHOLE, LANES>(wp[at(c)], a.w_post, c, a.d, lane);
        if (a.w_pre) load_chunk<WHOLE, LANES>(wq[at(c)], a.w_pre, c, a.d, lane);
        if (a.ls) load_chunk<WHOLE, LANES>(ls[at(c)], a.ls, c, a.d, lane);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (!a.w_post) wp[at(c)][i] = 1.f;
            if (!a.w_pre) wq[at(c)][i] = 1.f;
            ls[at(c)][i] = a.ls ? a.scale * ls[at(c)][i] : a.scale;
        }
    };
    if (ONE) weights(0);
    // the gate and its slope
    auto gate = [&](float z, float &act, float &slope) {
        float rest;
        const float e = sigmoid(z, rest);
        act = a.act == kActSilu ? z * e : a.act ? e : z;
        slope = a.act == kActSilu ? e * (1.f + z * (1.f - e)) : a.act ? e * rest : 1.f;
    };
    float acc[3][C][8] = {};   // of w_post, w_pre, layer_scale

    const unsigned stride = gridDim.x * ROWS, mine = row_of<LANES>();
    BwdRows<X, R, Y, LANES, H, WHOLE> next;
    if (ONE) next.load(a, blockIdx.x * ROWS + mine, lane);
    for (unsigned row0 = blockIdx.x * ROWS; row0 < (unsigned)a.rows; row0 += stride) {
        const unsigned row = row0 + mine;
        const bool there = row < (unsigned)a.rows;   // (sums meet at barriers)
        const int d = there ? a.d : 0, ra = there ? row / (unsigned)a.inner : 0, rb = there ? row - ra * (unsigned)a.inner : 0;
        const bool joint = a.pre && a.r;
        float x[H][8], z[H][8], sum_r[H][8], dy[H][8], g[H][8], t[C][8];
        auto read_x = [&](int c) { load_chunk<WHOLE, LANES>(x[at(c)], row_at<X>(a.x, a.sx, ra, rb), c, d, lane); };
        auto read_z = [&](int c) { load_chunk<WHOLE, LANES>(z[at(c)], row_at<Y>(a.z, a.sz, ra, rb), c, d, lane); };
        auto read_r = [&](int c) { load_chunk<WHOLE, LANES>(sum_r[at(c)], row_at<R>(a.r, a.sro, ra, rb), c, d, lane); };
        auto read_dy = [&](int c) { load_chunk<WHOLE, LANES>(dy[at(c)], row_at<Y>(a.dy, a.sdy, ra, rb), c, a.dy ? d : 0, lane); };
        auto read_g = [&](int c) { load_chunk<WHOLE, LANES>(g[at(c)], row_at<R>(a.dr_out, a.sdro, ra, rb), c, a.dr_out ? d : 0, lane); };
        if (HOLD) {
            if (!ONE) {
                next.load(a, row, lane);
#pragma unroll
                for (int c = 0; c < C; ++c) weights(c);
            }
            next.x.get(x, d, lane);
            next.dy.get(dy, d, lane);
            next.g.get(g, d, lane);
            if (a.z) next.z.get(z, d, lane);
            if (joint) next.sum_r.get(sum_r, d, lane);
            if (ONE) next.load(a, row + stride, lane);
        }
        float s1 = 1.f, s2 = 1.f, mean_t = 0.f;
        if (a.post || joint) {
            float sum[3] = {0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < C; ++c) {
                if (!HOLD && joint) weights(c);
                if (!HOLD) {
                    read_x(c);
                    if (joint) {
                        read_r(c);
                        read_dy(c);
                    }
                    asm volatile("" ::: "memory");
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    sum[0] = fmaf(x[at(c)][i], x[at(c)][i], sum[0]);
                    if (joint) {
                        sum[1] = fmaf(sum_r[at(c)][i], sum_r[at(c)][i], sum[1]);
                        sum[2] = fmaf(dy[at(c)][i] * wq[at(c)][i], sum_r[at(c)][i], sum[2]);
                    }
                }
            }
            row_sum(sum);
            if (a.post) s1 = 1.f / sqrtf(fmaf(sum[0], a.inv_d, a.eps));
            if (joint) {
                s2 = 1.f / sqrtf(fmaf(sum[1], a.inv_d, a.eps));
                mean_t = sum[2] * s2 * a.inv_d;
            }
        }
        // r' = s l u where there is no residual
        auto sum_again = [&](int c, int i) {
            float act = 1.f, slope;
            if (a.z) gate(z[at(c)][i], act, slope);
            sum_r[at(c)][i] = (a.post ? x[at(c)][i] * s1 * wp[at(c)][i] : x[at(c)][i]) * act * ls[at(c)][i];
        };
        if (a.pre && !a.r) {
            float sum[2] = {0.f, 0.f};
#pragma unroll
            for (int c = 0; c < C; ++c) {
                if (!HOLD) weights(c);
                if (!HOLD) {
                    read_x(c);
                    read_dy(c);
                    if (a.z) read_z(c);
                    asm volatile("" ::: "memory");
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    sum_again(c, i);
                    sum[0] = fmaf(sum_r[at(c)][i], sum_r[at(c)][i], sum[0]);
                    sum[1] = fmaf(dy[at(c)][i] * wq[at(c)][i], sum_r[at(c)][i], sum[1]);
                }
            }
            row_sum(sum);
            s2 = 1.f / sqrtf(fmaf(sum[0], a.inv_d, a.eps));
            mean_t = sum[1] * s2 * a.inv_d;
        }
        float sum[1] = {0.f};
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (!HOLD) weights(c);
            if (!HOLD) {
                read_x(c);
                read_dy(c);
                read_g(c);
                if (a.z) read_z(c);
                if (joint) read_r(c);
                asm volatile("" ::: "memory");
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (a.pre) {
                    if (!HOLD && !a.r) sum_again(c, i);
                    const float h = sum_r[at(c)][i] * s2;
                    if (there) acc[1][c][i] = fmaf(dy[at(c)][i], h, acc[1][c][i]);
                    g[at(c)][i] += s2 * (dy[at(c)][i] * wq[at(c)][i] - h * mean_t);
                } else {
                    g[at(c)][i] += dy[at(c)][i];
                }
                const float xh = a.post ? x[at(c)][i] * s1 : x[at(c)][i], n = a.post ? xh * wp[at(c)][i] : xh;
                float act = 1.f, slope = 0.f;
                if (a.z) gate(z[at(c)][i], act, slope);
                if (there) acc[2][c][i] = fmaf(a.scale * g[at(c)][i], n * act, acc[2][c][i]);
                const float du = ls[at(c)][i] * g[at(c)][i], dn = du * act;
                z[at(c)][i] = du * n * slope;
                if (there) acc[0][c][i] = fmaf(dn, xh, acc[0][c][i]);
                x[at(c)][i] = xh;
                t[c][i] = a.post ? dn * wp[at(c)][i] : dn;
                sum[0] = fmaf(t[c][i], xh, sum[0]);
            }
            if (a.dr) store_chunk<WHOLE, LANES>(row_at<R>(a.dr, a.sdr, ra, rb), g[at(c)], c, d, lane);
            if (a.dz) store_chunk<WHOLE, LANES>(row_at<Y>(a.dz, a.sdz, ra, rb), z[at(c)], c, d, lane);
        }
        if (!a.dx) continue;
        if (a.post) {
            row_sum(sum);
            const float mean = sum[0] * a.inv_d;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                if (!HOLD) {
                    read_x(c);
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[at(c)][i] *= s1;
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) t[c][i] = s1 * (t[c][i] - x[at(c)][i] * mean);
            }
        }
        store_row<WHOLE, LANES>(row_at<X>(a.dx, a.sdx, ra, rb), t, d, lane);
    }

    // the workgroup's sums
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        if (!a.dw[k]) continue;
        float *part = a.part + ((long)blockIdx.x * 3 + k) * a.d;
        if constexpr (UNITS == 1) {
            store_row<WHOLE, LANES>(part, acc[k], a.d, lane);
        } else {
            static_assert(C == 1, "several rows to a workgroup have one chunk to a lane");
            const int unit = LANES < 64 ? threadIdx.x >> 6 : threadIdx.x / LANES;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float v = acc[k][0][i];
#pragma unroll
                for (int o = LANES; o < 64; o <<= 1) v += __shfl_xor(v, o);
                if (LANES >= 64 || (threadIdx.x & 63) < LANES) meet[unit * LANES * 8 + element<LANES>(0, lane) + i] = v;
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
#pragma unroll
    for (int i = 0; i < kMostGroups / 16; ++i) {   // (all of them in flight)
        const int p = u + 16 * i;
        v += p < a.groups && e < a.d ? a.part[((long)p * 3 + k) * a.d + e] : 0.f;
    }
    lds[u][threadIdx.x & 63] = v;
    __syncthreads();
    if (u == 0 && e < a.d) {
        for (int i = 1; i < 16; ++i) v += lds[i][threadIdx.x];
        a.dw[k][e] = v;
    }
}

template <typename X, typename R, typename Y, int LANES, int C> void launch(const NormArgs &a, hipStream_t s)
{
    if (a.d % 8 == 0) bdgdn_norm_bwd_kernel<X, R, Y, LANES, C, true><<<a.groups, kThreads, 0, s>>>(a);
    else bdgdn_norm_bwd_kernel<X, R, Y, LANES, C, false><<<a.groups, kThreads, 0, s>>>(a);
}

template <typename X, typename R, typename Y> hipError_t sized(const NormArgs &a, hipStream_t s)
{
    if (a.groups > 0) {
        if (a.d <= 64) launch<X, R, Y, 8, 1>(a, s);
        else if (a.d <= 128) launch<X, R, Y, 16, 1>(a, s);
        else if (a.d <= 256) launch<X, R, Y, 32, 1>(a, s);
        else if (a.d <= 512) launch<X, R, Y, 64, 1>(a, s);
        else if (a.d <= 1024) launch<X, R, Y, 128, 1>(a, s);
        else if (a.d <= 2048) launch<X, R, Y, 256, 1>(a, s);
        else if (a.d <= 4096) launch<X, R, Y, 512, 1>(a, s);
        else if (a.d <= 8192) launch<X, R, Y, 512, 2>(a, s);
        else launch<X, R, Y, 512, 4>(a, s);
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
    const int lanes = d <= 64 ? 8 : d <= 128 ? 16 : d <= 256 ? 32 : d <= 512 ? 64 : d <= 1024 ? 128 : d <= 2048 ? 256 : 512, in_one = kThreads / lanes;
    const int groups = (int)(((long)rows + in_one - 1) / in_one);
    return groups < kMostGroups ? groups : kMostGroups;
}

hipError_t launch_norm_bwd(bool xf, bool rf, bool yf, NormArgs &a, hipStream_t s)
{
    if (yf) return sized<float, float, float>(a, s);
    if (xf) return rf ? sized<float, float, __bf16>(a, s) : sized<float, __bf16, __bf16>(a, s);
    return rf ? sized<__bf16, float, __bf16>(a, s) : sized<__bf16, __bf16, __bf16>(a, s);
}

}  // namespace bdgdn
