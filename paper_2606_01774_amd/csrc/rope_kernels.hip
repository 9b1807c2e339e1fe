// rope_kernels.hip -- rotary positions of queries and keys.
//
// A pair (a, b) of a head's elements turns by t = 2 pi frac(p F / 2^64), F the pair's turns a
// position in units of 2^-64, p the row's position: (a cos t - b sin t, a sin t + b cos t).
// p F modulo 2^64 is one integer product and exact, so far positions lose nothing.  cos and
// sin of a head's pairs are the same in every head: a thread computes those of its pairs once
// and takes them through several heads.
//
// Bound by memory: q and k of 4 x 4096 tokens (40 heads of 128, bf16) 70 us, 335 MB at 4.8 TB/s (a copy of 512
// MB: 5.4); 8 heads of 64 of 32749 fp32 rows, 16 elements turned, 29 us, 134 MB at 4.6.  One token 3.4 us, a
// launch and a load.
#include "anywhere.hpp"
#include "layer.hpp"

namespace bdgdn {

namespace {

constexpr int kThreads = 256;
constexpr unsigned kMostBlocks = 1u << 22;   // (a launch has 2^32 threads)

// cos and sin of 2 pi w / 2^64.  The nearest quarter turn is taken off as an integer; what is left
// lies within an eighth of a turn, where the Taylor series of degree 9 and 10 are exact to 2e-9.
__device__ __forceinline__ void turn(uint64_t w, float &c, float &s)
{
    const uint32_t f = (uint32_t)((w + 0x80000000ull) >> 32);
    const uint32_t quarter = (f + 0x20000000u) >> 30;
    const float x = (float)(int32_t)(f - (quarter << 30)) * 1.46291807926715968e-9f;   // 2 pi / 2^32
    const float z = x * x;
    const float sn = fmaf(x * z, fmaf(z, fmaf(z, fmaf(z, 2.75573192e-6f, -1.98412698e-4f), 8.33333333e-3f), -1.66666667e-1f), x);
    const float cs = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -2.75573192e-7f, 2.48015873e-5f), -1.38888889e-3f), 4.16666667e-2f), -0.5f), 1.f);
    const float a = quarter & 1 ? sn : cs, b = quarter & 1 ? cs : sn;
    c = (quarter + 1) & 2 ? -a : a;
    s = quarter & 2 ? -b : b;
}

// 16 bytes of consecutive elements, of which the first n are there.
template <typename E> struct Chunk {
    static constexpr int CH = 16 / sizeof(E);
    E e[CH];
    template <bool RAGGED> __device__ __forceinline__ void load(const unsigned char *p, int n)
    {
        if (!RAGGED || n >= CH) {
            const u32x4 w = *reinterpret_cast<const typename AnyPlace<E>::type *>(p);
            __builtin_memcpy(e, &w, 16);
        } else {
#pragma unroll
            for (int i = 0; i < CH; ++i)
                if (i < n) e[i] = reinterpret_cast<const E *>(p)[i];
        }
    }
    template <bool RAGGED> __device__ __forceinline__ void store(unsigned char *p, int n) const
    {
        if (!RAGGED || n >= CH) {
            u32x4 w;
            __builtin_memcpy(&w, e, 16);
            *reinterpret_cast<typename AnyPlace<E>::type *>(p) = w;
        } else {
#pragma unroll
            for (int i = 0; i < CH; ++i)
                if (i < n) reinterpret_cast<E *>(p)[i] = e[i];
        }
    }
};

// A piece of a head is two chunks: HALF: elements and their partners; PAIRS, and behind the rotated
// elements those that stay: neighbours.  RAGGED: some chunks are not whole.
template <typename E, bool PAIRS, bool RAGGED> __global__ void __launch_bounds__(kThreads) bdgdn_rope_kernel(RopeArgs a)
{
    constexpr int CH = Chunk<E>::CH, U = 2;   // pairs of a piece; heads in flight
    const int row_l = threadIdx.x >> (a.item_log + a.sub_log);
    const int sub = (threadIdx.x >> a.item_log) & ((1 << a.sub_log) - 1);
    const int first = sub + (blockIdx.y << a.sub_log), step = gridDim.y << a.sub_log;
    const int half = a.rot >> 1;
    const unsigned rows = (unsigned)a.R * (unsigned)a.N;
    for (unsigned row = (blockIdx.x << a.row_log) + row_l; row < rows; row += gridDim.x << a.row_log) {
        const int r = row / (unsigned)a.N, n = row - r * (unsigned)a.N;
        if (a.count && n >= a.count[r]) continue;
        long p = a.pos ? a.pos[row] : n;
        if (a.len) {
            const int slot = a.slot ? a.slot[r] : r;
            if ((unsigned)slot < (unsigned)a.n_slots) p += max(a.len[slot], 0);
        }
        for (int item = threadIdx.x & ((1 << a.item_log) - 1); item < a.items; item += 1 << a.item_log) {
            const bool stays = item >= a.turned;
            // the elements of the two chunks, and how many there are
            int e0 = stays ? a.rot + (item - a.turned) * 2 * CH : PAIRS ? item * 2 * CH : item * CH;
            int e1 = stays || PAIRS ? e0 + CH : e0 + half;
            const int end = stays ? a.d : PAIRS ? a.rot : half;
            if (stays && a.d - a.rot >= CH) {   // (what lies past the end is moved back: copied twice)
                e0 = min(e0, a.d - CH);
                e1 = min(e1, a.d - CH);
            }
            const int n0 = end - e0, n1 = stays ? end - e1 : PAIRS ? n0 - CH : n0;
            float c[CH], s[CH];
            if (!stays) {
#pragma unroll
                for (int i = 0; i < CH; ++i) {
                    const int pair = item * CH + i;
                    turn((uint64_t)p * a.turns[RAGGED ? min(pair, half - 1) : pair], c[i], s[i]);
                    c[i] *= a.scale;
                    s[i] *= a.sine;
                }
            }
            for (int h0 = first; h0 < a.h; h0 += U * step) {
                Chunk<E> lo[U], hi[U];
                unsigned char *to[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int h = h0 + u * step;
                    if (h >= a.h) break;
                    const int w = h >= a.h_q, hh = w ? h - a.h_q : h;
                    const unsigned char *from = a.x[w] + r * a.xs[w][0] + n * a.xs[w][1] + hh * a.xs[w][2];
                    to[u] = a.y[w] + r * a.ys[w][0] + n * a.ys[w][1] + hh * a.ys[w][2];
                    lo[u].template load<RAGGED>(from + e0 * (int)sizeof(E), n0);
                    if (!RAGGED || n1 > 0) hi[u].template load<RAGGED>(from + e1 * (int)sizeof(E), n1);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (h0 + u * step >= a.h) break;
                    if (!stays) {
#pragma unroll
                        for (int i = 0; i < CH; ++i) {
                            // PAIRS: the first half of a piece's pairs lies in lo, the second in hi
                            E &ea = !PAIRS ? lo[u].e[i] : i < CH / 2 ? lo[u].e[2 * i % CH] : hi[u].e[2 * i % CH];
                            E &eb = !PAIRS ? hi[u].e[i] : i < CH / 2 ? lo[u].e[(2 * i + 1) % CH] : hi[u].e[(2 * i + 1) % CH];
                            const float x = to_f(ea), y = to_f(eb);
                            ea = to_e<E>(x * c[i] - y * s[i]);
                            eb = to_e<E>(x * s[i] + y * c[i]);
                        }
                    }
                    lo[u].template store<RAGGED>(to[u] + e0 * (int)sizeof(E), n0);
                    if (!RAGGED || n1 > 0) hi[u].template store<RAGGED>(to[u] + e1 * (int)sizeof(E), n1);
                }
            }
        }
    }
}

int log_up(int x)
{
    int l = 0;
    while ((1 << l) < x) ++l;
    return l;
}

template <typename E, bool PAIRS> hipError_t launch(RopeArgs &a, hipStream_t s)
{
    constexpr int CH = Chunk<E>::CH;
    const int half = a.rot / 2, stay = a.in_place ? 0 : a.d - a.rot;
    a.turned = (half + CH - 1) / CH;   // (of either layout: a piece has CH pairs)
    a.items = a.turned + (stay + 2 * CH - 1) / (2 * CH);
    a.item_log = log_up(a.items);
    if (a.item_log > 8) a.item_log = 8;
    const unsigned rows = (unsigned)a.R * (unsigned)a.N;
    // head-lanes: all heads at once, fewer as long as there are four lanes to every place the chip has
    // for one.  q and k of 16384 tokens (40 heads of 128, bf16): 84 us with one, 69 with four, 72 with eight,
    // 93 with all heads at once
    int heads_log = log_up(a.h);
    while (heads_log > 0 && ((long)rows << (a.item_log + heads_log - 1)) >= 4 * 524288) --heads_log;
    // (or one to every place, where a quarter of them or more would have no head.  22270 rows of 18 heads of 64: 41 us, 34 with
    // half the lanes, of 24 42 and 37.  Fewer idle ones: 28 heads of 64 43 and 40, of 128 68 and 70; 40 of 64 54 and 55)
    if (4 * a.h <= 3 << heads_log && ((long)rows << (a.item_log + heads_log - 1)) >= 524288) --heads_log;
    a.sub_log = heads_log < 8 - a.item_log ? heads_log : 8 - a.item_log;
    a.row_log = 8 - a.item_log - a.sub_log;
    if (heads_log > a.sub_log + 15) heads_log = a.sub_log + 15;   // (a grid's second dimension)
    const unsigned blocks = (rows + (1u << a.row_log) - 1) >> a.row_log;
    const unsigned parts = 1u << (heads_log - a.sub_log);
    const dim3 grid(blocks * (long)parts < kMostBlocks ? blocks : kMostBlocks / parts, parts);
    if (half % CH || (stay && stay < CH)) bdgdn_rope_kernel<E, PAIRS, true><<<grid, kThreads, 0, s>>>(a);
    else bdgdn_rope_kernel<E, PAIRS, false><<<grid, kThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(bool bf16, bool pairs, RopeArgs &a, hipStream_t s)
{
    if (bf16) return pairs ? launch<__bf16, true>(a, s) : launch<__bf16, false>(a, s);
    return pairs ? launch<float, true>(a, s) : launch<float, false>(a, s);
}

}  // namespace bdgdn
