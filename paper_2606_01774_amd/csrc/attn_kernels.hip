// attn_kernels.hip -- attention of a block of nodes over a paged cache and over the nodes
// themselves.
//
// The rows that share a key head (N nodes x G query heads, M in all) are taken together, 16 MT
// of them by one wave, which streams 32 keys at a time from memory to registers and needs no
// LDS.  Both products are formed transposed, S^T = K Q^T and O^T = V^T P^T, so that a lane
// holds one row's scores (row = lane & 15) and the accumulators of the first product are the
// operand of the second as they stand.  The keys of a request are cut into splits, one wave
// each; a second kernel joins the splits' (maximum, sum, output).
#include <type_traits>

#include "common.hpp"
#include "round.hpp"

namespace bdgdn {

namespace {

constexpr int kTile = 32;          // keys of a step
constexpr int kMinTiles = 4;       // of a split, at least
constexpr int kWaves = 4;          // of a workgroup
typedef unsigned int u32x2v __attribute__((ext_vector_type(2)));

template <typename T, int D> struct Geo {
    static constexpr int kRow = D * sizeof(T);          // bytes of a row
    static constexpr int NK = kRow / 64;                // 16-byte chunks of a key row in a lane
    static constexpr int VB = kRow < 256 ? 8 : 16;      // bytes of a chunk of a value row in a lane
    static constexpr int NV = kRow / (16 * VB);         // such chunks
    static constexpr int EV = VB / sizeof(T);           // elements of such a chunk
    static constexpr int NT = D / 16;                   // accumulator tiles of a row group
};

__device__ __forceinline__ float max_over_groups(float x)
{
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}

// What a wave works on: request, split of its tiles, key head, row group.
struct Item {
    int r, split, splits, base;    // base: the request's first (request, split) pair
    int len, tiles;                // cached tokens and tiles
    bool valid;
};

__device__ __forceinline__ int length_of(const AttnArgs &a, int r)
{
    const int slot = a.slot ? a.slot[r] : r;
    if ((unsigned)slot >= (unsigned)a.n_slots) return 0;
    return min(max(a.len[slot], 0), a.max_pages * a.page);
}

// Tiles of a split: what spreads all requests' tiles over the pairs that the call aims at.
__device__ __forceinline__ int split_tiles(const AttnArgs &a, int lane)
{
    int sum = 0;
    for (int r = lane; r < a.R; r += 64) sum += (length_of(a, r) + kTile - 1) / kTile;
#pragma unroll
    for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
    return max(kMinTiles, (sum + a.items - 1) / a.items);
}

// The (request, split) pair number `pair`, or with pair < 0 the pairs of request `req`.
__device__ __forceinline__ Item find_item(const AttnArgs &a, int pair, int req, int lane)
{
    const int per = split_tiles(a, lane);
    Item it = {};
    int before = 0;
    for (int r0 = 0; r0 < a.R; r0 += 64) {
        const int r = r0 + lane;
        const int len = r < a.R ? length_of(a, r) : 0;
        const int tiles = (len + kTile - 1) / kTile;
        const int n = r < a.R ? max(1, (tiles + per - 1) / per) : 0;
        int inc = n;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int y = __shfl_up(inc, o);
            if (lane >= o) inc += y;
        }
        const int start = before + inc - n;
        const unsigned long long hit = __ballot(pair >= 0 ? (n > 0 && pair >= start && pair < start + n) : r == req);
        if (hit) {
            const int src = __ffsll(hit) - 1;
            it.r = r0 + src;
            it.base = __shfl(start, src);
            it.splits = __shfl(n, src);
            it.len = __shfl(len, src);
            it.tiles = __shfl(tiles, src);
            it.split = pair - it.base;
            it.valid = true;
            return it;
        }
        before += __shfl(inc, 63);
    }
    return it;
}

// One step of 32 keys for MT groups of 16 rows.
template <typename T, int D, int MT, bool SPLITP> struct Wave {
    typedef Geo<T, D> G;
    u32x4 q[MT][G::NK];
    f32x4 o[MT][G::NT];
    float l[MT];           // this lane's share of the weights' sum
    float m[MT];           // in units of the scaled scores' base-2 exponents
    float c;

    __device__ __forceinline__ void init(float scale)
    {
        c = scale;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            m[i] = -INFINITY;
            l[i] = 0.f;
#pragma unroll
            for (int t = 0; t < G::NT; ++t) o[i][t] = f32x4{0, 0, 0, 0};
        }
    }

    // s[mt][half] of lane (g, r): keys 16 half + 4 g + i against row r
    __device__ __forceinline__ void scores(f32x4 (&s)[MT][2], const u32x4 (&k)[2][G::NK])
    {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                f32x4 x = {0, 0, 0, 0};
#pragma unroll
                for (int j = 0; j < G::NK; ++j) {
                    if constexpr (sizeof(T) == 2) {
                        x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[h][j]),
                                                                    __builtin_bit_cast(bf16x8, q[mt][j]), x, 0, 0, 0);
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            x = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[h][j][i]),
                                                                     __uint_as_float(q[mt][j][i]), x, 0, 0, 0);
                    }
                }
                s[mt][h] = x;
            }
    }

    // s -> weights exp2(c s - m); the running maximum grows only when a score passes it by
    // more than 2^8, so that the accumulators are seldom rescaled.
    __device__ __forceinline__ void weigh(f32x4 (&s)[MT][2])
    {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            float top = s[mt][0][0];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) top = fmaxf(top, s[mt][h][i]);
            top = c * max_over_groups(top);
            if (__any(top > m[mt] + 8.f)) {
                const float now = fmaxf(m[mt], top);
                const float f = m[mt] == -INFINITY ? 0.f : fexp2(m[mt] - now);
                m[mt] = now;
                l[mt] *= f;
#pragma unroll
                for (int t = 0; t < G::NT; ++t) o[mt][t] *= f;
            }
            const float base = m[mt] == -INFINITY ? 0.f : m[mt];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[mt][h][i] = fexp2(fmaf(s[mt][h][i], c, -base));
                    l[mt] += s[mt][h][i];
                }
        }
    }

    // o += V^T P^T; v[e] is the lane's part of value row
    // 16 (e / 4) + 4 g + e % 4.
    __device__ __forceinline__ void values(const f32x4 (&p)[MT][2], const u32x4 (&v)[8][G::NV])
    {
        if constexpr (sizeof(T) == 2) {
            bf16x8 hi[MT], lo[MT];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float x = p[mt][e >> 2][e & 3];
                    hi[mt][e] = (__bf16)x;
                    if (SPLITP) lo[mt][e] = (__bf16)(x - (float)hi[mt][e]);
                }
            }
#pragma unroll
            for (int j = 0; j < G::NV; ++j)
#pragma unroll
                for (int w = 0; w < G::VB / 4; ++w) {
                    u32x4 even, odd;
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        even[x] = __builtin_amdgcn_perm(v[2 * x + 1][j][w], v[2 * x][j][w], 0x05040100u);
                        odd[x] = __builtin_amdgcn_perm(v[2 * x + 1][j][w], v[2 * x][j][w], 0x07060302u);
                    }
                    const bf16x8 a0 = __builtin_bit_cast(bf16x8, even), a1 = __builtin_bit_cast(bf16x8, odd);
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) {
                        f32x4 &o0 = o[mt][j * G::EV + 2 * w], &o1 = o[mt][j * G::EV + 2 * w + 1];
                        o0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a0, hi[mt], o0, 0, 0, 0);
                        o1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a1, hi[mt], o1, 0, 0, 0);
                        if (SPLITP) {
                            o0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a0, lo[mt], o0, 0, 0, 0);
                            o1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a1, lo[mt], o1, 0, 0, 0);
                        }
                    }
                }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    const float x = p[mt][e >> 2][e & 3];
#pragma unroll
                    for (int j = 0; j < G::NV; ++j)
#pragma unroll
                        for (int w = 0; w < 4; ++w)
                            o[mt][j * 4 + w] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[e][j][w]), x,
                                                                                    o[mt][j * 4 + w], 0, 0, 0);
                }
        }
    }
};

template <int NK> __device__ __forceinline__ void load_key(u32x4 (&k)[NK], const unsigned char *row, int g)
{
#pragma unroll
    for (int j = 0; j < NK; ++j) k[j] = *reinterpret_cast<const u32x4 *>(row + 64 * j + 16 * g);
}

template <int VB, int NV> __device__ __forceinline__ void load_value(u32x4 (&v)[NV], const unsigned char *row, int r)
{
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if constexpr (VB == 16) {
            v[j] = *reinterpret_cast<const u32x4 *>(row + 256 * j + 16 * r);
        } else {
            const u32x2v x = *reinterpret_cast<const u32x2v *>(row + 128 * j + 8 * r);
            v[j] = u32x4{x[0], x[1], 0, 0};
        }
    }
}

template <int N> __device__ __forceinline__ void zero(u32x4 (&x)[N])
{
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = u32x4{0, 0, 0, 0};
}

__device__ __forceinline__ bool finite_words(u32x4 x, bool wide)
{
    bool ok = true;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        ok &= wide ? (x[i] & 0x7f800000u) != 0x7f800000u
                   : (x[i] & 0x7f80u) != 0x7f80u && (x[i] & 0x7f800000u) != 0x7f800000u;
    return ok;
}

// Infinities and NaNs of a word of values set to zero.
__device__ __forceinline__ uint32_t finite_part(uint32_t x, bool wide)
{
    if (wide) return (x & 0x7f800000u) == 0x7f800000u ? 0u : x;
    const uint32_t lo = (x & 0x7f80u) == 0x7f80u ? 0u : x & 0xffffu;
    return lo | ((x & 0x7f800000u) == 0x7f800000u ? 0u : x & 0xffff0000u);
}

template <typename T, int D, int MT, bool SPLITP>
__global__ void __launch_bounds__(64 * kWaves) bdgdn_tree_attn_kernel(AttnArgs a)
{
    typedef Geo<T, D> G;
    const int lane = threadIdx.x & 63, g = lane >> 4, rr = lane & 15;
    const int heads = a.h_kv * a.RG;
    const int wave = __builtin_amdgcn_readfirstlane(blockIdx.x * kWaves + (threadIdx.x >> 6));
    const int pair = wave / heads, rest = wave - pair * heads;
    const int kvh = rest / a.RG, rg = rest - kvh * a.RG;
    const Item it = find_item(a, pair, -1, lane);
    if (!it.valid) return;
    const int r = __builtin_amdgcn_readfirstlane(it.r);
    const int M = a.N * a.G, count = a.count ? min(max(a.count[r], 0), a.N) : a.N;

    Wave<T, D, MT, SPLITP> w;
    w.init(a.c);
    int node[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int row = min((rg * MT + mt) * 16 + rr, M - 1);
        node[mt] = row / a.G;
        load_key(w.q[mt], static_cast<const unsigned char *>(a.q) + ((long)r * a.N + node[mt]) * a.q_stride +
                              (long)(kvh * a.G + row - node[mt] * a.G) * G::kRow, g);
#pragma unroll
        for (int j = 0; j < G::NK; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) w.q[mt][j][i] = (w.q[mt][j][i] & a.q_and) ^ a.q_xor;
    }

    // the split's share of the request's tiles
    const int t0 = (int)((long)it.tiles * it.split / it.splits), t1 = (int)((long)it.tiles * (it.split + 1) / it.splits);
    const int slot = a.slot ? a.slot[r] : r;
    const int32_t *table = a.table + (long)slot * a.max_pages;
    const unsigned char *kp = static_cast<const unsigned char *>(a.kp) + (long)kvh * a.head_stride;
    const unsigned char *vp = static_cast<const unsigned char *>(a.vp) + (long)kvh * a.head_stride;
    for (int t = t0; t < t1; ++t) {
        // lane x (and x + 32) finds key x of the tile
        const int tok = t * kTile + (lane & 31);
        const int col = tok / a.page;
        const int page = tok < it.len ? table[col] : -1;
        const bool there = (unsigned)page < (unsigned)a.n_pages;
        const uint32_t at = there ? page * a.page16 + (tok - col * a.page) * a.token16 : 0;
        const uint32_t seen = (uint32_t)__ballot(there);
        if (!seen) continue;
        u32x4 k[2][G::NK], v[8][G::NV];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t off = __shfl(at, 16 * h + rr);
            if (seen >> (16 * h + rr) & 1) load_key(k[h], kp + (long)off * 16, g);
            else zero(k[h]);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int key = 16 * (e >> 2) + 4 * g + (e & 3);
            const uint32_t off = __shfl(at, key);
            if (seen >> key & 1) load_value<G::VB>(v[e], vp + (long)off * 16, rr);
            else zero(v[e]);
        }
        f32x4 s[MT][2];
        w.scores(s, k);
        if (seen != 0xffffffffu) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (!(seen >> (16 * (e >> 2) + 4 * g + (e & 3)) & 1)) s[mt][e >> 2][e & 3] = -INFINITY;
        }
        w.weigh(s);
        w.values(s, v);
    }

    // the nodes themselves, with the last split
    if (it.split == it.splits - 1) {
        const unsigned char *kn = static_cast<const unsigned char *>(a.k) + (long)r * a.N * a.k_stride + (long)kvh * G::kRow;
        const unsigned char *vn = static_cast<const unsigned char *>(a.v) + (long)r * a.N * a.v_stride + (long)kvh * G::kRow;
        const uint64_t live = count >= 64 ? ~0ull : (1ull << count) - 1;
        uint64_t sees[MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            sees[mt] = live;
            if (a.mask_kind == 1) sees[mt] &= node[mt] == 63 ? ~0ull : (1ull << (node[mt] + 1)) - 1;
            if (a.mask_kind == 2) sees[mt] &= a.mask[(long)r * a.N + node[mt]];
        }
        for (int n0 = 0; n0 < count; n0 += kTile) {
            u32x4 k[2][G::NK], v[8][G::NV];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int key = n0 + 16 * h + rr;
                if (key < count) load_key(k[h], kn + key * a.k_stride, g);
                else zero(k[h]);
            }
            bool fine = true;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int key = n0 + 16 * (e >> 2) + 4 * g + (e & 3);
                if (key < count) load_value<G::VB>(v[e], vn + key * a.v_stride, rr);
                else zero(v[e]);
#pragma unroll
                for (int j = 0; j < G::NV; ++j) fine &= finite_words(v[e][j], sizeof(T) == 4);
            }
            f32x4 s[MT][2];
            w.scores(s, k);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (!(sees[mt] >> (n0 + 16 * (e >> 2) + 4 * g + (e & 3)) & 1)) s[mt][e >> 2][e & 3] = -INFINITY;
            w.weigh(s);
            if (__any(!fine)) {
                // Values that are not finite: a weight of zero does not take them out of a
                // product, so they are left out of it and added where they are seen.
#pragma unroll
                for (int e = 0; e < 8; ++e)
#pragma unroll
                    for (int j = 0; j < G::NV; ++j)
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[e][j][i] = finite_part(v[e][j][i], sizeof(T) == 4);
            }
            w.values(s, v);
            if (__any(!fine)) {
                for (int x = 0; x < kTile && n0 + x < count; ++x) {
                    const T *row = reinterpret_cast<const T *>(vn + (n0 + x) * a.v_stride);
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) {
                        f32x4 mine = s[mt][0];
                        if (x >= 16) mine = s[mt][1];
                        const int from = ((x & 15) >> 2) * 16 + rr;
                        const float p0 = __shfl(mine[0], from), p1 = __shfl(mine[1], from), p2 = __shfl(mine[2], from),
                                    p3 = __shfl(mine[3], from);
                        const float p = (x & 3) == 0 ? p0 : (x & 3) == 1 ? p1 : (x & 3) == 2 ? p2 : p3;
                        if (sees[mt] >> (n0 + x) & 1) {
#pragma unroll
                            for (int j = 0; j < G::NV; ++j)
#pragma unroll
                                for (int i = 0; i < 4; ++i)
#pragma unroll
                                    for (int e = 0; e < G::EV; ++e) {
                                        const float y = to_f(row[j * 16 * G::EV + (4 * g + i) * G::EV + e]);
                                        if (!(fabsf(y) < INFINITY)) w.o[mt][j * G::EV + e][i] += p * y;
                                    }
                        }
                    }
                }
            }
        }
    }

    // the wave's part: rows of [d] and (maximum, sum)
    float *po = a.part_o + (long)wave * 16 * MT * D, *pml = a.part_ml + (long)wave * 16 * MT * 2;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int row = mt * 16 + rr;
        float sum = w.l[mt];
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if ((rg * MT + mt) * 16 + rr >= M) continue;
        if (g == 0) {
            pml[2 * row] = w.m[mt];
            pml[2 * row + 1] = sum;
        }
#pragma unroll
        for (int j = 0; j < G::NV; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < G::EV; ++e)
                    po[row * D + j * 16 * G::EV + (4 * g + i) * G::EV + e] = w.o[mt][j * G::EV + e][i];
    }
}

// One wave per (request, node, query head): o = sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s.
template <typename Out, int D> __global__ void __launch_bounds__(256) bdgdn_tree_attn_join_kernel(AttnArgs a, int mt)
{
    const int lane = threadIdx.x & 63;
    const long row = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= (long)a.R * a.N * a.h_q) return;
    const int hq = (int)(row % a.h_q);
    const int rn = (int)(row / a.h_q), n = rn % a.N, r = rn / a.N;
    const Item it = find_item(a, -1, r, lane);
    const int count = a.count ? min(max(a.count[r], 0), a.N) : a.N;
    const int kvh = hq / a.G, m0 = n * a.G + hq - kvh * a.G, rg = m0 / (16 * mt), at = m0 - rg * 16 * mt;
    constexpr int E = D / 64;
    float top = -INFINITY;
    for (int s = 0; s < it.splits; ++s) {
        const long wave = ((long)(it.base + s) * a.h_kv + kvh) * a.RG + rg;
        top = fmaxf(top, a.part_ml[(wave * 16 * mt + at) * 2]);
    }
    const float base = top == -INFINITY ? 0.f : top;
    float o[E] = {}, l = 0.f;
    for (int s = 0; s < it.splits; ++s) {
        const long wave = ((long)(it.base + s) * a.h_kv + kvh) * a.RG + rg;
        const float m = a.part_ml[(wave * 16 * mt + at) * 2];
        if (m == -INFINITY) continue;   // a split without a key
        const float f = fexp2(m - base);
        l += f * a.part_ml[(wave * 16 * mt + at) * 2 + 1];
        const float *po = a.part_o + (wave * 16 * mt + at) * D + lane * E;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] += f * po[e];
    }
    const bool none = n >= count || l == 0.f;
    Out *out = static_cast<Out *>(a.o) + row * D + lane * E;
#pragma unroll
    for (int e = 0; e < E; ++e) out[e] = to_e<Out>(none ? 0.f : o[e] / l);
    if (a.lse && lane == 0) a.lse[row] = none ? -INFINITY : (top + __log2f(l)) * 0.6931471805599453f;
}

__global__ void __launch_bounds__(64) bdgdn_tree_mask_kernel(int N, const int32_t *parent, uint64_t *mask, int32_t *depth)
{
    // one wave per request, lane n for node n: a node's word takes in its parent's when that is done
    const int n = threadIdx.x, r = blockIdx.x;
    const int p = n < N ? parent[(long)r * N + n] : -1;
    const bool root = p < 0 || p >= n;
    uint64_t w = n < N ? 1ull << n : 0;
    int up = root ? n : p;
    for (int i = 0; i < 6; ++i) {   // after i steps a word holds the 2^i nearest ancestors
        const uint32_t lo = __shfl((uint32_t)w, up), hi = __shfl((uint32_t)(w >> 32), up);
        w |= (uint64_t)hi << 32 | lo;
        up = __shfl(up, up);
    }
    if (n < N) {
        mask[(long)r * N + n] = w;
        if (depth) depth[(long)r * N + n] = __popcll(w) - 1;
    }
}

// Row groups of a wave at most: what its registers hold (512 a lane).
constexpr int most_mt(bool bf16, int d) { return bf16 ? (d == 256 ? 2 : 4) : (d == 256 ? 1 : 2); }

template <typename T, int D, bool F32OUT> hipError_t launch_d(int mt, const AttnArgs &a, hipStream_t s)
{
    constexpr bool SP = sizeof(T) == 2 && F32OUT;
    constexpr int most = most_mt(sizeof(T) == 2, D);
    typedef typename std::conditional<F32OUT, float, __bf16>::type Out;
    if (mt == 1) bdgdn_tree_attn_kernel<T, D, 1, SP><<<a.grid, 64 * kWaves, 0, s>>>(a);
    else if (mt == 2) bdgdn_tree_attn_kernel<T, D, (most < 2 ? 1 : 2), SP><<<a.grid, 64 * kWaves, 0, s>>>(a);
    else bdgdn_tree_attn_kernel<T, D, most, SP><<<a.grid, 64 * kWaves, 0, s>>>(a);
    const long rows = (long)a.R * a.N * a.h_q;
    bdgdn_tree_attn_join_kernel<Out, D><<<(unsigned)((rows + 3) / 4), 256, 0, s>>>(a, mt);
    return hipGetLastError();
}

}  // namespace

AttnPlan attn_plan(bool bf16, int d, int R, int N, int h_q, int h_kv)
{
    AttnPlan p;
    const int M = N * (h_q / h_kv);
    const int groups = M <= 16 ? 1 : M <= 32 ? 2 : 4, most = most_mt(bf16, d);
    p.mt = groups < most ? groups : most;
    p.RG = (M + 16 * p.mt - 1) / (16 * p.mt);
    const long heads = (long)h_kv * p.RG;
    const long items = 2048 / heads;
    p.items = (int)(items < 1 ? 1 : items);
    p.items_max = p.items + R;
    const size_t rows = (size_t)p.items_max * heads * 16 * p.mt;
    p.part_bytes = ((rows * 8 + 255) & ~(size_t)255) + rows * d * 4;
    return p;
}

hipError_t launch_tree_attn(bool bf16, bool f32_out, int d, const AttnPlan &p, AttnArgs &a, hipStream_t s)
{
    a.RG = p.RG;
    a.items = p.items;
    a.grid = (int)(((long)p.items_max * a.h_kv * p.RG + kWaves - 1) / kWaves);
#define BDGDN_ATTN(T, F) \
    (d == 64 ? launch_d<T, 64, F>(p.mt, a, s) : d == 128 ? launch_d<T, 128, F>(p.mt, a, s) : launch_d<T, 256, F>(p.mt, a, s))
    if (!bf16) return BDGDN_ATTN(float, true);
    return f32_out ? BDGDN_ATTN(__bf16, true) : BDGDN_ATTN(__bf16, false);
#undef BDGDN_ATTN
}

hipError_t launch_tree_mask(int R, int N, const int32_t *parent, uint64_t *mask, int32_t *depth, hipStream_t s)
{
    bdgdn_tree_mask_kernel<<<R, 64, 0, s>>>(N, parent, mask, depth);
    return hipGetLastError();
}

}  // namespace bdgdn
