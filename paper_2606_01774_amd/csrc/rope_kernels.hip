// rope_kernels.hip -- rotary positions of queries and keys.
//
// A pair (a, b) of a head's elements turns by t = 2 pi frac(p F / 2^64), F the pair's turns a
// position in units of 2^-64, p the row's position: (a cos t - b sin t, a sin t + b cos t).
// p F modulo 2^64 is one integer product and exact, so far positions lose nothing.  cos and
// sin of a head's pairs are the same in every head: a thread computes those of its pairs once
// and takes them through several heads.
#include "common.hpp"
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

// CH consecutive elements, 16 bytes of them at once.
template <typename E, int CH> struct Chunk {
    E e[CH];
    template <int N = CH> __device__ __forceinline__ void load(const unsigned char *p)
    {
        if constexpr (N * sizeof(E) == 16) {
            const u32x4 w = *reinterpret_cast<const u32x4 *>(p);
            __builtin_memcpy(e, &w, 16);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) e[i] = reinterpret_cast<const E *>(p)[i];
        }
    }
    template <int N = CH> __device__ __forceinline__ void store(unsigned char *p) const
    {
        if constexpr (N * sizeof(E) == 16) {
            u32x4 w;
            __builtin_memcpy(&w, e, 16);
            *reinterpret_cast<u32x4 *>(p) = w;
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) reinterpret_cast<E *>(p)[i] = e[i];
        }
    }
};

// Elements that stay, to a piece.
template <typename E, int CH> constexpr int staying() { return CH * sizeof(E) == 16 ? CH : 1; }

// A piece of a head: HALF: CH elements and their partners; PAIRS: CH elements, CH / 2 pairs; behind
// the rotated ones some elements that stay.
template <typename E, bool PAIRS, int CH> __global__ void __launch_bounds__(kThreads) bdgdn_rope_kernel(RopeArgs a)
{
    constexpr int P = PAIRS ? CH / 2 : CH, S = staying<E, CH>();   // pairs of a piece
    constexpr int U = 2;                                           // heads in flight
    const int row_l = threadIdx.x >> (a.item_log + a.sub_log);
    const int sub = (threadIdx.x >> a.item_log) & ((1 << a.sub_log) - 1);
    const int first = sub + (blockIdx.y << a.sub_log), step = gridDim.y << a.sub_log;
    const int turned = a.rot / (PAIRS ? CH : 2 * CH);
    const long half = (a.rot >> 1) * (long)sizeof(E);
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
            const bool stays = item >= turned;
            const long e0 = (stays ? a.rot + (item - turned) * S : item * CH) * (long)sizeof(E);
            float c[P], s[P];
            if (!stays) {
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    turn((uint64_t)p * a.turns[item * P + i], c[i], s[i]);
                    c[i] *= a.scale;
                    s[i] *= a.sine;
                }
            }
            for (int h0 = first; h0 < a.h; h0 += U * step) {
                Chunk<E, CH> lo[U], hi[U];
                unsigned char *to[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int h = h0 + u * step;
                    if (h >= a.h) break;
                    const int w = h >= a.h_q, hh = w ? h - a.h_q : h;
                    const unsigned char *from = a.x[w] + r * a.xs[w][0] + n * a.xs[w][1] + hh * a.xs[w][2] + e0;
                    to[u] = a.y[w] + r * a.ys[w][0] + n * a.ys[w][1] + hh * a.ys[w][2] + e0;
                    if (stays) {
                        lo[u].template load<S>(from);
                    } else {
                        lo[u].load(from);
                        if (!PAIRS) hi[u].load(from + half);
                    }
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (h0 + u * step >= a.h) break;
                    if (stays) {
                        lo[u].template store<S>(to[u]);
                        continue;
                    }
#pragma unroll
                    for (int i = 0; i < P; ++i) {
                        E &ea = lo[u].e[PAIRS ? 2 * i : i], &eb = PAIRS ? lo[u].e[PAIRS ? 2 * i + 1 : 0] : hi[u].e[i];
                        const float x = to_f(ea), y = to_f(eb);
                        ea = to_e<E>(x * c[i] - y * s[i]);
                        eb = to_e<E>(x * s[i] + y * c[i]);
                    }
                    lo[u].store(to[u]);
                    if (!PAIRS) hi[u].store(to[u] + half);
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

template <typename E, bool PAIRS, int CH> hipError_t launch(RopeArgs &a, hipStream_t s)
{
    const int piece = PAIRS ? CH : 2 * CH;
    a.items = a.rot / piece + (a.in_place ? 0 : (a.d - a.rot) / staying<E, CH>());
    a.item_log = log_up(a.items);
    if (a.item_log > 8) a.item_log = 8;
    const unsigned rows = (unsigned)a.R * (unsigned)a.N;
    // head-lanes: all heads at once, fewer as long as the chip stays full
    int heads_log = log_up(a.h);
    while (heads_log > 0 && ((long)rows << (a.item_log + heads_log - 1)) >= 524288) --heads_log;
    a.sub_log = heads_log < 8 - a.item_log ? heads_log : 8 - a.item_log;
    a.row_log = 8 - a.item_log - a.sub_log;
    const unsigned blocks = (rows + (1u << a.row_log) - 1) >> a.row_log;
    const unsigned parts = 1u << (heads_log - a.sub_log);
    const dim3 grid(blocks * (long)parts < kMostBlocks ? blocks : kMostBlocks / parts, parts);
    bdgdn_rope_kernel<E, PAIRS, CH><<<grid, kThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(bool bf16, bool pairs, bool wide, RopeArgs &a, hipStream_t s)
{
    if (bf16) {
        if (pairs) return wide ? launch<__bf16, true, 8>(a, s) : launch<__bf16, true, 2>(a, s);
        return wide ? launch<__bf16, false, 8>(a, s) : launch<__bf16, false, 1>(a, s);
    }
    if (pairs) return wide ? launch<float, true, 4>(a, s) : launch<float, true, 2>(a, s);
    return wide ? launch<float, false, 4>(a, s) : launch<float, false, 1>(a, s);
}

}  // namespace bdgdn
