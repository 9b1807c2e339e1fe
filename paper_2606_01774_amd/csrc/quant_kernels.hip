// quant_kernels.hip -- products of 8-bit integers with scales for each token and channel
// (include/bdgdn.h, bdgdn_quant_rows, bdgdn_quant_matmul): sums of products are 32-bit integers from
// the matrix cores, exact in any order, and the scales meet them on the way out.
//
// 8191 x 8192 x 4096: rows quantised in 23 to 25 us (101 MB at 4.2 TB/s; the vector units are always busy), the
// product in 264 to 276, 2.0 POP/s (a library's product of 8192 x 8192 x 4096 8-bit integers, without scales: 1.9;
// the matrix cores' bound is 5).  The matrix cores are busy in 52 % of the cycles, LDS in 41 %, and a wave spends
// 39 % of its time waiting for loads and at barriers (counters; 508000 cycles in 276 us are 1.85 GHz): neither of the
// two is the bound, the wait between a step and the next is.  512 x 6144 x 2048: 3 to 4 and 14.8 us, 0.9 POP/s, 192
// tiles for 256 compute units, matrix cores busy in 27 % of the cycles.
// 3 x 8192 x 4096: 3 and 10.6 us, 34 MB of weights at 3.2 TB/s, of which the launch and the first loads
// are some 4.
#include "norm.hpp"

namespace bdgdn {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef const __attribute__((address_space(1))) void *GlobalPtr;
typedef __attribute__((address_space(3))) void *LdsPtr;

// ------------------------------------------------------------------ rows to integers
constexpr int kQuantThreads = 256;

// The largest magnitude as its bits: those of a NaN or an infinity are above every finite one's.
template <int LANES> __device__ __forceinline__ uint32_t row_top(uint32_t top, uint32_t *lds)
{
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
    if constexpr (LANES > 64) {
        lds_barrier();   // the last row's has been read
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = top;
        lds_barrier();
#pragma unroll
        for (int w = 0; w < LANES / 64; ++w) top = max(top, lds[w]);
    }
    return top;
}

__device__ __forceinline__ uint32_t four(const float *x, float scale)
{
    uint32_t word = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float t = fminf(fmaxf(rintf(x[i] / scale), -127.f), 127.f);
        word |= (uint32_t)(uint8_t)(int8_t)(int)t << (8 * i);
    }
    return word;
}

// A row to LANES lanes.  HELD chunks of 8 columns to a lane stay in registers between the two passes; longer
// rows are read again (from the caches).
template <typename E, int LANES, int HELD> __global__ void __launch_bounds__(kQuantThreads) bdgdn_quant_rows_kernel(QuantArgs a)
{
    __shared__ uint32_t lds[kQuantThreads / 64];
    const int lane = threadIdx.x % LANES;
    const unsigned row = blockIdx.x * (kQuantThreads / LANES) + row_of<LANES>();
    const int cols = row < (unsigned)a.rows ? a.cols : 0, width = cols ? a.width : 0;
    const E *x = static_cast<const E *>(a.x) + row * a.xs;
    Ahead<false, LANES, HELD, E> in;
    float v[HELD][8];
    uint32_t top = 0;
    auto look = [&](const E *from, int n) {
        in.load(from, n, lane);
        in.get(v, n, lane);
#pragma unroll
        for (int c = 0; c < HELD; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[c][i]) & 0x7fffffffu);
    };
    constexpr int SPAN = HELD * LANES * 8;
    for (int at = SPAN; at < cols; at += SPAN) look(x + at, cols - at);
    look(x, min(cols, SPAN));
    top = row_top<LANES>(top, lds);
    const bool bad = top > 0x7f7fffffu;
    const float scale = bad ? __uint_as_float(0x7fc00000u) : __uint_as_float(top) * (1.f / 127.f);
    if (cols && lane == 0) a.scale[row] = scale;
    int8_t *q = a.q + row * a.qs;
    for (int at = 0; at < width; at += SPAN) {
        if (at) {
            const int n = max(cols - at, 0);
            in.load(x + at, n, lane);
            in.get(v, n, lane);
        }
#pragma unroll
        for (int c = 0; c < HELD; ++c) {
            const int e = at + element<LANES>(c, lane);
            if (e < width) {   // (width is a multiple of 8)
                const bool none = !(scale > 0.f);
                *reinterpret_cast<uint2 *>(q + e) = none ? uint2{0, 0} : uint2{four(v[c], scale), four(v[c] + 4, scale)};
            }
        }
    }
}

template <typename E, int LANES, int HELD> hipError_t launch_rows(const QuantArgs &a, hipStream_t s)
{
    constexpr int ROWS = kQuantThreads / LANES;
    bdgdn_quant_rows_kernel<E, LANES, HELD><<<((unsigned)a.rows + ROWS - 1) / ROWS, kQuantThreads, 0, s>>>(a);
    return hipGetLastError();
}

template <typename E> hipError_t sized_rows(const QuantArgs &a, hipStream_t s)
{
    if (a.cols <= 512) return launch_rows<E, 64, 1>(a, s);
    if (a.cols <= 2048) return launch_rows<E, 256, 1>(a, s);
    if (a.cols <= 4096) return launch_rows<E, 256, 2>(a, s);
    return launch_rows<E, 256, 4>(a, s);
}

// ------------------------------------------------------------------ many tokens
// Stages rows [row0, row0 + ROWS) x kBK bytes in LDS, straight from memory.  A row's chunks of 16 bytes are
// permuted, place c of row r holding chunk c ^ (r & 7), so that eight neighbouring lanes, which read one chunk of
// eight rows, find them in different banks.  Rows past the last are the last one again (their results go
// nowhere).
constexpr int kBK = 128;
template <int ROWS, int WAVES>
__device__ __forceinline__ void stage(const int8_t *p, long ld, int row0, int rows, int k0, int8_t *lds, int wave, int lane)
{
    constexpr int CHUNKS = kBK / 16, AT_ONCE = 64 / CHUNKS;   // rows to a load
#pragma unroll
    for (int i = 0; i < ROWS / AT_ONCE / WAVES; ++i) {
        const int block = (i * WAVES + wave) * AT_ONCE, r = block + lane / CHUNKS;
        const int8_t *from = p + (long)min(row0 + r, rows - 1) * ld + k0 + (((lane % CHUNKS) ^ (r & 7)) << 4);
        __builtin_amdgcn_global_load_lds((GlobalPtr)from, (LdsPtr)(lds + block * kBK), 16, 0, 0);
    }
}

// Waits until at most N of this wave's loads are on their way (s_waitcnt vmcnt(N), the others at their maxima).
template <int N> __device__ __forceinline__ void wait_loads() { __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | (N >> 4) << 14); }

// Between a wave's writes to LDS and its other lanes' reads of them, and back.  The hardware takes a wave's LDS
// operations in order; this keeps the compiler, which sees a lane by itself, to it, and costs no instruction.
__device__ __forceinline__ void wave_exchange()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

template <bool FIRST, typename A, typename B> struct Either { typedef A type; };
template <typename A, typename B> struct Either<false, A, B> { typedef B type; };

// Which tile is this workgroup's.  Workgroups go to the eight dies in turn: each die takes neighbouring tiles,
// in bands of kBand rows of tiles, so that its cache holds what they share.
constexpr int kBand = 8;
__device__ __forceinline__ void tile_of(const QuantMatmulArgs &a, int tiles_m, int tiles_n, int &tm, int &tn)
{
    const int all = tiles_m * tiles_n, id = blockIdx.x, die = id & 7, each = all >> 3, more = all & 7;
    const int at = die * each + min(die, more) + (id >> 3);
    const int band = at / (kBand * tiles_n), first = band * kBand, high = min(kBand, tiles_m - first), in = at - band * kBand * tiles_n;
    tm = first + in % high;
    tn = in / high;
}

// BM x BN outputs to a workgroup, TM x TN tiles of 32 x 32 to a wave; STAGES stages of kBK bytes of k.
// SPLIT: of one part of k, whose integer sums go to the workspace.
template <typename Y, int BM, int BN, int TM, int TN, int STAGES, bool SPLIT>
__global__ void __launch_bounds__(BM / (32 * TM) * (BN / (32 * TN)) * 64) bdgdn_quant_matmul_kernel(QuantMatmulArgs a)
{
    constexpr int WN = BN / (32 * TN), WAVES = BM / (32 * TM) * WN, STEPS = kBK / 32;
    constexpr int STAGE = (BM + BN) * kBK, LOADS = STAGE / 1024 / WAVES;   // a wave's to a stage
    // (one object: of several, the compiler would make every read of the stages wait for all loads into them)
    __shared__ __attribute__((aligned(16))) int8_t lds[STAGES * STAGE + BM * 4];
    float *s_scale = reinterpret_cast<float *>(lds + STAGES * STAGE);
    const int lane = threadIdx.x & 63, wave = wave_id();
    int tm, tn;
    tile_of(a, (a.m + BM - 1) / BM, (a.n + BN - 1) / BN, tm, tn);
    const int m0 = tm * BM, n0 = tn * BN;
    const int wm = (wave / WN) * TM * 32, wn = (wave % WN) * TN * 32;
    float ws[TN], bias[TN];
    if (!SPLIT) {
        for (int i = threadIdx.x; i < BM; i += WAVES * 64) s_scale[i] = a.as[min(m0 + i, a.m - 1)];
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int n = min(n0 + wn + 32 * j + (lane & 31), a.n - 1);
            ws[j] = a.ws[n];
            bias[j] = a.bias ? a.bias[n] : 0.f;
        }
    }
    wait_loads<0>();   // (from here on only the stages' loads are counted)
    i32x16 acc[TM][TN] = {};
    i32x4 fa[2][TM], fw[2][TN];
    const int all = a.k / kBK, from = SPLIT ? (int)((long)all * blockIdx.y / a.split) : 0;
    const int steps = (SPLIT ? (int)((long)all * (blockIdx.y + 1) / a.split) : all) - from;
    auto load = [&](int t) {
        int8_t *to = lds + t % STAGES * STAGE;
        const int k0 = (from + t) * kBK;
        stage<BM, WAVES>(a.a, a.lda, m0, a.m, k0, to, wave, lane);
        stage<BN, WAVES>(a.w, a.ldw, n0, a.n, k0, to + BM * kBK, wave, lane);
    };
    // a wave's operands of 32 bytes of k
    auto fetch = [&](int buf, int s, i32x4 (&ga)[TM], i32x4 (&gw)[TN]) {
        const int8_t *sa = lds + buf * STAGE, *sw = sa + BM * kBK;
        const int at = ((2 * s + (lane >> 5)) ^ (lane & 7)) << 4;
#pragma unroll
        for (int i = 0; i < TM; ++i) ga[i] = *reinterpret_cast<const i32x4 *>(sa + (wm + 32 * i + (lane & 31)) * kBK + at);
#pragma unroll
        for (int j = 0; j < TN; ++j) gw[j] = *reinterpret_cast<const i32x4 *>(sw + (wn + 32 * j + (lane & 31)) * kBK + at);
    };
#pragma unroll
    for (int t = 0; t < STAGES - 1; ++t)
        if (t < steps) load(t);
    int buf = 0;
    for (int t = 0; t < steps; ++t) {
        if (t + STAGES - 2 < steps) wait_loads<(STAGES - 2) * LOADS>();   // stage t has come
        else wait_loads<0>();
        lds_barrier();                                                    // for every wave, and all have read t - 1
        if (t + STAGES - 1 < steps) load(t + STAGES - 1);
        fetch(buf, 0, fa[0], fw[0]);
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            if (s + 1 < STEPS) fetch(buf, s + 1, fa[(s + 1) & 1], fw[(s + 1) & 1]);
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fa[s & 1][i], fw[s & 1][j], acc[i][j], 0, 0, 0);
        }
        buf = buf + 1 == STAGES ? 0 : buf + 1;
    }
    wait_loads<0>();
    lds_barrier();   // nothing comes into the stages, and nobody reads them, any more

    // A wave's results go through its part of the stages (rows of TN * 32), so that they leave as
    // 16-byte pieces of rows.
    typedef typename Either<SPLIT, int32_t, Y>::type Z;
    Z *out = SPLIT ? reinterpret_cast<Z *>(a.part) + (long)blockIdx.y * a.m * a.n : static_cast<Z *>(a.y);
    const long ldy = SPLIT ? a.n : a.ldy;
    constexpr int COLS = TN * 32, UNIT = 16 / sizeof(Z), PIECES = COLS / UNIT, ROOM = STAGES * STAGE / WAVES;
    constexpr int GROUP = ROOM / (32 * COLS * (int)sizeof(Z)) < TM ? ROOM / (32 * COLS * (int)sizeof(Z)) : TM;   // 32-row tiles at once
    static_assert(GROUP >= 1 && TM % GROUP == 0 && 64 % PIECES == 0, "the results fit the stages");
    Z *room = reinterpret_cast<Z *>(lds + wave * ROOM);
#pragma unroll
    for (int g = 0; g < TM; g += GROUP) {
#pragma unroll
        for (int i = g; i < g + GROUP; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int r = 8 * q + 4 * (lane >> 5);
                f32x4 as;
                if (!SPLIT) as = *reinterpret_cast<const f32x4 *>(&s_scale[wm + 32 * i + r]);
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        Z &to = room[(32 * (i - g) + r + e) * COLS + 32 * j + (lane & 31)];
                        if constexpr (SPLIT) to = acc[i][j][4 * q + e];
                        else to = to_e<Y>(fmaf((float)acc[i][j][4 * q + e], as[e] * ws[j], bias[j]));
                    }
            }
        wave_exchange();
#pragma unroll
        for (int it = 0; it < GROUP * 32 * PIECES / 64; ++it) {
            const int r = it * (64 / PIECES) + lane / PIECES, c = (lane % PIECES) * UNIT;
            const int m = m0 + wm + 32 * g + r, n = n0 + wn + c;
            const u32x4 w = *reinterpret_cast<const u32x4 *>(room + r * COLS + c);
            if (m >= a.m) continue;
            Z *to = out + m * ldy + n;
            if (n + UNIT <= a.n) {
                *reinterpret_cast<typename AnyPlace<Z>::type *>(to) = w;
            } else {
                Z v[UNIT];
                __builtin_memcpy(v, &w, 16);
#pragma unroll
                for (int e = 0; e < UNIT; ++e)
                    if (n + e < a.n) to[e] = v[e];
            }
        }
        wave_exchange();   // (the next tiles take the same room)
    }
}

// The parts' sums of four columns to a lane.
template <typename Y> __global__ void __launch_bounds__(256) bdgdn_quant_join_kernel(QuantMatmulArgs a)
{
    const int fours = (a.n + 3) >> 2;
    const long all = (long)a.m * fours, whole = (long)a.m * a.n;
    for (long x = (long)blockIdx.x * 256 + threadIdx.x; x < all; x += (long)gridDim.x * 256) {
        const int m = (int)(x / fours), n = (int)(x - (long)m * fours) * 4, there = min(a.n - n, 4);
        i32x4 sum = {0, 0, 0, 0};
        const int32_t *part = a.part + (long)m * a.n + n;
        for (int p = 0; p < a.split; ++p, part += whole) {
            if (there == 4) {
                const u32x4 w = *reinterpret_cast<const u32x4_e4 *>(part);
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[e] += (int)w[e];
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[e] += e < there ? part[e] : 0;
            }
        }
        const float as = a.as[m];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < there)
                static_cast<Y *>(a.y)[m * a.ldy + n + e] =
                    to_e<Y>(fmaf((float)sum[e], as * a.ws[n + e], a.bias ? a.bias[n + e] : 0.f));
    }
}

// ------------------------------------------------------------------ few tokens
constexpr int kFewWaves = 8;

// 16 channels and up to 16 tokens to a workgroup, whose waves share out k: each weight is read once, straight
// into the matrix cores' registers, and a wave's loads are under way together.  Bound by memory: a token against
// 16384 x 8192 weights 25 us (5.3 TB/s), against 1024 x 16384 ones latency, 8 us.
template <typename Y> __global__ void __launch_bounds__(kFewWaves * 64) bdgdn_quant_few_kernel(QuantMatmulArgs a)
{
    constexpr int U = 8;   // steps of 64 bytes of k
    __shared__ i32x4 lds[kFewWaves][64];
    const int lane = threadIdx.x & 63, wave = wave_id(), n0 = blockIdx.x * 16, m = lane & 15;
    const bool there = m < a.m;   // (what is not there is not read: zeros)
    const int8_t *w = a.w + (long)min(n0 + m, a.n - 1) * a.ldw + (lane >> 4) * 16;
    const int8_t *x = a.a + (long)(there ? m : 0) * a.lda + (lane >> 4) * 16;
    i32x4 acc = {0, 0, 0, 0};
    int k = wave * 64 * U;
    for (; k + 64 * U <= a.k; k += kFewWaves * 64 * U) {
        i32x4 fw[U], fx[U];
#pragma unroll
        for (int u = 0; u < U; ++u) fw[u] = *reinterpret_cast<const i32x4 *>(w + k + 64 * u);
#pragma unroll
        for (int u = 0; u < U; ++u) fx[u] = there ? *reinterpret_cast<const i32x4 *>(x + k + 64 * u) : i32x4{0, 0, 0, 0};
#pragma unroll
        for (int u = 0; u < U; ++u) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[u], fx[u], acc, 0, 0, 0);
    }
    for (; k < a.k; k += 64)   // (k is a multiple of 64: what is left of one wave's last turn)
        acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(*reinterpret_cast<const i32x4 *>(w + k),
                                                    there ? *reinterpret_cast<const i32x4 *>(x + k) : i32x4{0, 0, 0, 0}, acc, 0, 0, 0);
    lds[wave][lane] = acc;
    __syncthreads();
    if (wave > 0 || !there) return;
    i32x4 sum = {0, 0, 0, 0};
#pragma unroll
    for (int v = 0; v < kFewWaves; ++v) sum += lds[v][lane];
    const float as = a.as[m];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int n = n0 + 4 * (lane >> 4) + e;
        if (n < a.n)
            static_cast<Y *>(a.y)[m * a.ldy + n] = to_e<Y>(fmaf((float)sum[e], as * a.ws[n], a.bias ? a.bias[n] : 0.f));
    }
}

// Tiles of side x side outputs to a workgroup.
long tiles(int side, int m, int n) { return (long)((m + side - 1) / side) * ((n + side - 1) / side); }

template <typename Y, int SIDE, int TM, int TN, int STAGES> void launch_tiles(const QuantPlan &p, const QuantMatmulArgs &a, hipStream_t s)
{
    constexpr int THREADS = SIDE / (32 * TM) * (SIDE / (32 * TN)) * 64;
    const dim3 grid((unsigned)tiles(SIDE, a.m, a.n), p.split);
    if (p.split == 1) {
        bdgdn_quant_matmul_kernel<Y, SIDE, SIDE, TM, TN, STAGES, false><<<grid, THREADS, 0, s>>>(a);
        return;
    }
    bdgdn_quant_matmul_kernel<Y, SIDE, SIDE, TM, TN, STAGES, true><<<grid, THREADS, 0, s>>>(a);
    const long groups = ((long)a.m * ((a.n + 3) / 4) + 255) / 256;
    bdgdn_quant_join_kernel<Y><<<(unsigned)(groups < 65536 ? groups : 65536), 256, 0, s>>>(a);
}

template <typename Y> hipError_t launch(const QuantPlan &p, const QuantMatmulArgs &a, hipStream_t s)
{
    const unsigned strips = (a.n + 15) / 16;
    switch (p.kind) {
    case 16: bdgdn_quant_few_kernel<Y><<<strips, kFewWaves * 64, 0, s>>>(a); break;
    case 64: launch_tiles<Y, 64, 1, 1, 4>(p, a, s); break;
    case 128: launch_tiles<Y, 128, 2, 2, 2>(p, a, s); break;
    default: launch_tiles<Y, 256, 4, 2, 2>(p, a, s);
    }
    return hipGetLastError();
}

}  // namespace

// How a product is cut.  Up to 16 tokens go by strips of 16 channels.  Others by tiles of 64, 128 or 256 on a side,
// whose 128-byte steps of k take a workgroup 0.33, 0.61 and 2.0 us when every compute unit has one (0.47 for two of 64;
// two of 128 take twice as long): the least of steps x rounds over the chip x that.  m, n, k in us, with 64 / 128 / 256:
//     128, 8192, 4096: 13.4 / 22.9 / 50.3     512, 6144, 2048: 16.7 / 14.3 / 29.5     1024, 8192, 4096: 64.8 / 41.1 / 54.2
//     8191, 8192, 4096: 480 / 315 / 261
// Few tiles of 64 and a long k: parts of k, whose sums a second kernel joins (4 us): 128, 1024, 16384 takes 39.3 us in
// one part, 13.0 in eight.
QuantPlan quant_plan(int m, int n, int k)
{
    QuantPlan p = {};
    p.split = 1;
    if (m <= 16) {
        p.kind = 16;
        return p;
    }
    const double steps = k / 128;
    const long t64 = tiles(64, m, n), t128 = tiles(128, m, n), t256 = tiles(256, m, n);
    const double c64 = steps * (t64 <= 256 ? 0.33 : 0.47 * ((t64 + 511) / 512)), c128 = steps * 0.61 * ((t128 + 255) / 256);
    const double c256 = steps * 2.0 * ((t256 + 255) / 256);
    p.kind = c64 <= c128 && c64 <= c256 ? 64 : c128 <= c256 ? 128 : 256;
    if (p.kind == 64) {
        int split = 1;
        while (t64 * split * 2 <= 256 && steps / (split * 2) >= 8) split *= 2;
        if (steps * 0.33 * (split - 1) / split > 8.0) p.split = split;
    }
    if (p.split > 1) p.bytes = (size_t)p.split * m * n * 4;
    return p;
}

hipError_t launch_quant_rows(bool bf16, const QuantArgs &a, hipStream_t s)
{
    return bf16 ? sized_rows<__bf16>(a, s) : sized_rows<float>(a, s);
}

hipError_t launch_quant_matmul(bool f32_out, const QuantPlan &p, QuantMatmulArgs &a, hipStream_t s)
{
    return f32_out ? launch<float>(p, a, s) : launch<__bf16>(p, a, s);
}

}  // namespace bdgdn
