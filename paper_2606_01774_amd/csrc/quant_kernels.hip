// quant_kernels.hip -- products of 8-bit integers with scales for each token and channel
// (include/bdgdn.h, bdgdn_quant_rows, bdgdn_quant_matmul): sums of products are 32-bit integers from
// the matrix cores, exact in any order, and the scales meet them on the way out.
#include "common.hpp"
#include "layer.hpp"

namespace bdgdn {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef const __attribute__((address_space(1))) void *GlobalPtr;
typedef __attribute__((address_space(3))) void *LdsPtr;

// ------------------------------------------------------------------ rows to integers
constexpr int kQuantThreads = 256;

// The largest magnitude as its bits: those of a NaN or an infinity are above every finite one's.
template <typename E> __global__ void __launch_bounds__(kQuantThreads) bdgdn_quant_rows_kernel(QuantArgs a)
{
    __shared__ uint32_t lds[kQuantThreads / 64];
    const int tid = threadIdx.x;
    for (unsigned row = blockIdx.x; row < (unsigned)a.rows; row += gridDim.x) {
        const E *x = static_cast<const E *>(a.x) + row * a.xs;
        uint32_t top = 0;
        for (int e = tid; e < a.cols; e += kQuantThreads) top = max(top, __float_as_uint(to_f(x[e])) & 0x7fffffffu);
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
        __syncthreads();
        if ((tid & 63) == 0) lds[tid >> 6] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kQuantThreads / 64; ++w) top = max(top, lds[w]);
        const bool bad = top > 0x7f7fffffu;
        const float scale = bad ? __uint_as_float(0x7fc00000u) : __uint_as_float(top) / 127.f;
        if (tid == 0) a.scale[row] = scale;
        int8_t *q = a.q + row * a.qs;
        for (int e = tid * 4; e < a.width; e += kQuantThreads * 4) {
            uint32_t word = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (e + i < a.cols && scale > 0.f) {
                    const float t = fminf(fmaxf(rintf(to_f(x[e + i]) / scale), -127.f), 127.f);
                    word |= (uint32_t)(uint8_t)(int8_t)(int)t << (8 * i);
                }
            *reinterpret_cast<uint32_t *>(q + e) = word;
        }
    }
}

// ------------------------------------------------------------------ many tokens
constexpr int kBK = 128;   // bytes of a row to a stage: eight chunks of 16

// Stages rows [row0, row0 + ROWS) x kBK bytes in LDS, straight from memory.  Place c of row r holds
// chunk c ^ (r & 7), so that eight neighbouring lanes, which read one chunk of eight rows, find
// them in different banks.  Rows past the last are the last one again (their results go nowhere).
template <int ROWS, int WAVES>
__device__ __forceinline__ void stage(const int8_t *p, long ld, int row0, int rows, int k0, int8_t *lds, int wave, int lane)
{
#pragma unroll
    for (int i = 0; i < ROWS / 8 / WAVES; ++i) {
        const int block = (i * WAVES + wave) * 8, r = block + (lane >> 3);
        const int8_t *from = p + (long)min(row0 + r, rows - 1) * ld + k0 + (((lane & 7) ^ (r & 7)) << 4);
        __builtin_amdgcn_global_load_lds((GlobalPtr)from, (LdsPtr)(lds + block * kBK), 16, 0, 0);
    }
}

// BM x BN outputs to a workgroup, TM x TN tiles of 32 x 32 to a wave.
template <typename Y, int BM, int BN, int TM, int TN>
__global__ void __launch_bounds__(BM / (32 * TM) * (BN / (32 * TN)) * 64) bdgdn_quant_matmul_kernel(QuantMatmulArgs a)
{
    constexpr int WM = BM / (32 * TM), WN = BN / (32 * TN), WAVES = WM * WN;
    __shared__ __attribute__((aligned(16))) int8_t lds[2][(BM + BN) * kBK];
    const int lane = threadIdx.x & 63, wave = wave_id();
    const int tiles_n = (a.n + BN - 1) / BN;
    const int m0 = (blockIdx.x / tiles_n) * BM, n0 = (blockIdx.x % tiles_n) * BN;
    const int wm = (wave / WN) * TM * 32, wn = (wave % WN) * TN * 32;
    i32x16 acc[TM][TN] = {};
    stage<BM, WAVES>(a.a, a.lda, m0, a.m, 0, lds[0], wave, lane);
    stage<BN, WAVES>(a.w, a.ldw, n0, a.n, 0, lds[0] + BM * kBK, wave, lane);
    const int steps = a.k / kBK;
    for (int t = 0; t < steps; ++t) {
        wait_global_loads();
        __syncthreads();
        if (t + 1 < steps) {
            int8_t *next = lds[(t + 1) & 1];
            stage<BM, WAVES>(a.a, a.lda, m0, a.m, (t + 1) * kBK, next, wave, lane);
            stage<BN, WAVES>(a.w, a.ldw, n0, a.n, (t + 1) * kBK, next + BM * kBK, wave, lane);
        }
        const int8_t *sa = lds[t & 1], *sw = sa + BM * kBK;
#pragma unroll
        for (int s = 0; s < kBK / 32; ++s) {
            const int at = ((2 * s + (lane >> 5)) ^ (lane & 7)) << 4;
            i32x4 fa[TM], fw[TN];
#pragma unroll
            for (int i = 0; i < TM; ++i) fa[i] = *reinterpret_cast<const i32x4 *>(sa + (wm + 32 * i + (lane & 31)) * kBK + at);
#pragma unroll
            for (int j = 0; j < TN; ++j) fw[j] = *reinterpret_cast<const i32x4 *>(sw + (wn + 32 * j + (lane & 31)) * kBK + at);
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fa[i], fw[j], acc[i][j], 0, 0, 0);
        }
    }
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        const int n = n0 + wn + 32 * j + (lane & 31);
        if (n >= a.n) continue;
        const float ws = a.ws[n], bias = a.bias ? a.bias[n] : 0.f;
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int m = m0 + wm + 32 * i + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3);
                if (m < a.m) static_cast<Y *>(a.y)[m * a.ldy + n] = to_e<Y>(fmaf((float)acc[i][j][e], a.as[m] * ws, bias));
            }
    }
}

// ------------------------------------------------------------------ few tokens
constexpr int kFewWaves = 8;

// 16 channels and all tokens (16 MT at most) to a workgroup, whose waves share out k: each weight is
// read once, straight into the matrix cores' registers.
template <typename Y, int MT> __global__ void __launch_bounds__(kFewWaves * 64) bdgdn_quant_few_kernel(QuantMatmulArgs a)
{
    constexpr int U = 4;   // steps of 64 bytes in flight
    __shared__ i32x4 lds[kFewWaves][MT][64];
    const int lane = threadIdx.x & 63, wave = wave_id(), n0 = blockIdx.x * 16;
    const int8_t *w = a.w + (long)min(n0 + (lane & 15), a.n - 1) * a.ldw + (lane >> 4) * 16;
    const int8_t *x[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) x[i] = a.a + (long)min(16 * i + (lane & 15), a.m - 1) * a.lda + (lane >> 4) * 16;
    i32x4 acc[MT] = {};
    int k = wave * 64 * U;
    for (; k + 64 * U <= a.k; k += kFewWaves * 64 * U) {
        i32x4 fw[U], fx[MT][U];
#pragma unroll
        for (int u = 0; u < U; ++u) fw[u] = *reinterpret_cast<const i32x4 *>(w + k + 64 * u);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int u = 0; u < U; ++u) fx[i][u] = *reinterpret_cast<const i32x4 *>(x[i] + k + 64 * u);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int u = 0; u < U; ++u) acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[u], fx[i][u], acc[i], 0, 0, 0);
    }
    for (; k < a.k; k += 64) {   // (k is a multiple of 64: what is left of one wave's last turn)
        const i32x4 fw = *reinterpret_cast<const i32x4 *>(w + k);
#pragma unroll
        for (int i = 0; i < MT; ++i)
            acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw, *reinterpret_cast<const i32x4 *>(x[i] + k), acc[i], 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) lds[wave][i][lane] = acc[i];
    __syncthreads();
    if (wave >= MT) return;
    i32x4 sum = {0, 0, 0, 0};
#pragma unroll
    for (int v = 0; v < kFewWaves; ++v) sum += lds[v][wave][lane];
    const int m = 16 * wave + (lane & 15);
    if (m >= a.m) return;
    const float as = a.as[m];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int n = n0 + 4 * (lane >> 4) + e;
        if (n < a.n)
            static_cast<Y *>(a.y)[m * a.ldy + n] = to_e<Y>(fmaf((float)sum[e], as * a.ws[n], a.bias ? a.bias[n] : 0.f));
    }
}

template <typename Y> hipError_t launch(const QuantPlan &p, const QuantMatmulArgs &a, hipStream_t s)
{
    if (p.kind < 0) {
        const long grid = (long)((a.m + 127) / 128) * ((a.n + 127) / 128);
        bdgdn_quant_matmul_kernel<Y, 128, 128, 2, 2><<<(unsigned)grid, 256, 0, s>>>(a);
    } else {
        const unsigned grid = (a.n + 15) / 16;
        if (p.kind == 1) bdgdn_quant_few_kernel<Y, 1><<<grid, kFewWaves * 64, 0, s>>>(a);
        else if (p.kind == 2) bdgdn_quant_few_kernel<Y, 2><<<grid, kFewWaves * 64, 0, s>>>(a);
        else bdgdn_quant_few_kernel<Y, 4><<<grid, kFewWaves * 64, 0, s>>>(a);
    }
    return hipGetLastError();
}

}  // namespace

QuantPlan quant_plan(int m, int n, int k)
{
    QuantPlan p = {};
    p.split = 1;
    p.kind = m <= 16 ? 1 : m <= 32 ? 2 : m <= 64 ? 4 : -1;
    return p;
}

hipError_t launch_quant_rows(bool bf16, const QuantArgs &a, hipStream_t s)
{
    const unsigned grid = a.rows < (1 << 22) ? a.rows : 1 << 22;
    if (bf16) bdgdn_quant_rows_kernel<__bf16><<<grid, kQuantThreads, 0, s>>>(a);
    else bdgdn_quant_rows_kernel<float><<<grid, kQuantThreads, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_quant_matmul(bool f32_out, const QuantPlan &p, QuantMatmulArgs &a, hipStream_t s)
{
    return f32_out ? launch<float>(p, a, s) : launch<__bf16>(p, a, s);
}

}  // namespace bdgdn
