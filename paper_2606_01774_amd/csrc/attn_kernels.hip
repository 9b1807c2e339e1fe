// attn_kernels.hip -- attention of a block of nodes over a paged cache and over the nodes
// themselves.
//
// The rows that share a key head (N nodes x G query heads, M in all) are taken together: 16 MT
// of them by one wave, which streams 32 keys at a time from memory to registers, the next keys
// requested when the scores are done with these and the next values when the output is.  Both
// products are formed transposed, S^T = K Q^T and O^T = V^T P^T, so that a lane holds one row's
// scores (row = lane & 15) and the accumulators of the first product are the operand of the
// second as they stand; the transposed values are made from 16-byte loads by byte permutes.
// Four waves are a workgroup: those with different rows take the same keys, those with the
// same rows every KW-th tile, and are joined through LDS.  The keys of a request are cut into
// as many splits as fill the chip, balanced over requests of different lengths; where a
// request has more than one, a second kernel joins the splits' (maximum, sum, output).
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

// What a workgroup works on: a request and one split of its tiles.
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

// The (request, split) pair number `pair`.  A split has the tiles that spread all requests'
// over the pairs that the call aims at.
__device__ __forceinline__ Item find_item(const AttnArgs &a, int pair, int lane)
{
    const int len0 = lane < a.R ? length_of(a, lane) : 0;
    int sum = (len0 + kTile - 1) / kTile;
    for (int r = lane + 64; r < a.R; r += 64) sum += (length_of(a, r) + kTile - 1) / kTile;
#pragma unroll
    for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
    const int per = max(kMinTiles, (sum + a.items - 1) / a.items);
    Item it = {};
    int before = 0;
    for (int r0 = 0; r0 < a.R; r0 += 64) {
        const int r = r0 + lane;
        const int len = r0 == 0 ? len0 : r < a.R ? length_of(a, r) : 0;
        const int tiles = (len + kTile - 1) / kTile;
        const int n = r < a.R ? max(1, (tiles + per - 1) / per) : 0;
        int inc = n;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int y = __shfl_up(inc, o);
            if (lane >= o) inc += y;
        }
        const int start = before + inc - n;
        const unsigned long long hit = __ballot(pair >= start && pair < start + n);
        if (hit) {
            const int src = __ffsll(hit) - 1;
            it.r = r0 + src;
            it.base = __builtin_amdgcn_readlane(start, src);
            it.splits = __builtin_amdgcn_readlane(n, src);
            it.len = __builtin_amdgcn_readlane(len, src);
            it.tiles = __builtin_amdgcn_readlane(tiles, src);
            it.split = pair - it.base;
            it.valid = true;
            return it;
        }
        before += __builtin_amdgcn_readlane(inc, 63);
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

// Where the keys of a tile of cached tokens lie.  WHOLE: a page holds whole tiles, so a tile
// is one base address; otherwise lane x finds key x & 31 and the others ask it.  A key that is
// not there reads the pool's first token instead and is left out by `seen`.
template <bool WHOLE> struct Tiles {
    const int32_t *table;
    const unsigned char *kp, *vp;
    int len, page, n_pages, lane;
    uint32_t page16, token16;
    uint32_t at;          // WHOLE: of the tile's first token, else of this lane's, in 16 bytes
    uint32_t seen;        // keys that are there

    // the page of a tile (WHOLE) or of this lane's key, ahead of its use
    __device__ __forceinline__ int page_of(int t) const
    {
        if (WHOLE) return table[t * kTile / page];
        const int tok = t * kTile + (lane & 31);
        return tok < len ? table[tok / page] : -1;
    }
    __device__ __forceinline__ void go(int t, int p)
    {
        const int tok = t * kTile + (WHOLE ? 0 : lane & 31);
        const bool there = (unsigned)p < (unsigned)n_pages;
        at = there ? p * page16 + (uint32_t)(tok % page) * token16 : 0;
        if (WHOLE) {
            const int left = len - tok;
            seen = !there ? 0u : left >= kTile ? ~0u : (1u << left) - 1;
        } else {
            seen = (uint32_t)__ballot(there);
        }
    }
    __device__ __forceinline__ uint32_t offset(int key) const { return WHOLE ? 0 : __shfl(at, key); }
    template <int NK> __device__ __forceinline__ void keys(u32x4 (&k)[2][NK], int g, int rr) const
    {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (WHOLE) load_key(k[h], kp + (long)at * 16 + (uint32_t)(h * 16 * token16) * 16 + (uint32_t)(rr * token16 * 16), g);
            else load_key(k[h], kp + (long)offset(16 * h + rr) * 16, g);
        }
    }
    template <int VB, int NV> __device__ __forceinline__ void values(u32x4 (&v)[8][NV], int g, int rr) const
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t key = 16 * (e >> 2) + (e & 3);
            if (WHOLE) load_value<VB>(v[e], vp + (long)at * 16 + (long)key * token16 * 16 + (uint32_t)(4 * g * token16 * 16), rr);
            else load_value<VB>(v[e], vp + (long)offset(key + 4 * g) * 16, rr);
        }
    }
};

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

template <typename T, int D, int MT, bool SPLITP, bool WHOLE, typename Out>
__global__ void __launch_bounds__(64 * kWaves) bdgdn_tree_attn_kernel(AttnArgs a)
{
    typedef Geo<T, D> G;
    __shared__ f32x4 s_o[2][G::NT][64];
    __shared__ float s_ml[2][2][64];
    const int lane = threadIdx.x & 63, g = lane >> 4, rr = lane & 15;
    const int wave = wave_id(), kw = wave / a.RW, rw = wave - kw * a.RW, KW = kWaves / a.RW;
    // workgroups with the same keys and other rows are neighbours on one XCD (their numbers
    // are equal modulo 8)
    const int x = blockIdx.x & 7, y = blockIdx.x >> 3;
    const int unit = y / a.RG * 8 + x, rg = y % a.RG;
    const int pair = unit / a.h_kv, kvh = unit - pair * a.h_kv;
    const Item it = find_item(a, pair, lane);
    if (!it.valid) return;
    const int r = it.r;
    const int M = a.N * a.G, count = a.count ? min(max(a.count[r], 0), a.N) : a.N;
    if (it.split == 0 && kvh == 0 && rg == 0 && threadIdx.x == 0) {
        a.info[2 * r] = it.base;
        a.info[2 * r + 1] = it.splits;
    }

    Wave<T, D, MT, SPLITP> w;
    w.init(a.c);
    const int row0 = (rg * a.RW + rw) * 16 * MT;   // of this wave's rows
    int node[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int row = min(row0 + mt * 16 + rr, M - 1);
        node[mt] = row / a.G;
        load_key(w.q[mt], static_cast<const unsigned char *>(a.q) + ((long)r * a.N + node[mt]) * a.q_stride +
                              (long)(kvh * a.G + row - node[mt] * a.G) * G::kRow, g);
    }

    // the split's share of the request's tiles, every KW-th for this wave
    const int t0 = (int)((long)it.tiles * it.split / it.splits) + kw, t1 = (int)((long)it.tiles * (it.split + 1) / it.splits);
    const int slot = a.slot ? a.slot[r] : r;
    Tiles<WHOLE> tl;
    tl.table = a.table + (long)slot * a.max_pages;
    tl.kp = static_cast<const unsigned char *>(a.kp) + (long)kvh * a.head_stride;
    tl.vp = static_cast<const unsigned char *>(a.vp) + (long)kvh * a.head_stride;
    tl.len = it.len; tl.page = a.page; tl.n_pages = a.n_pages; tl.lane = lane;
    tl.page16 = a.page16; tl.token16 = a.token16;
    u32x4 k[2][G::NK], v[8][G::NV];
    int next_page = -1;
    if (t0 < t1) {
        tl.go(t0, tl.page_of(t0));
        tl.keys(k, g, rr);
        tl.template values<G::VB>(v, g, rr);
        if (t0 + KW < t1) next_page = tl.page_of(t0 + KW);
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int j = 0; j < G::NK; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) w.q[mt][j][i] = (w.q[mt][j][i] & a.q_and) ^ a.q_xor;
    for (int t = t0; t < t1; t += KW) {
        f32x4 s[MT][2];
        w.scores(s, k);
        const uint32_t seen = tl.seen;
        const bool more = t + KW < t1;
        if (more) {
            tl.go(t + KW, next_page);
            tl.keys(k, g, rr);
            if (t + 2 * KW < t1) next_page = tl.page_of(t + 2 * KW);
        }
        if (seen != ~0u) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (!(seen >> (16 * (e >> 2) + 4 * g + (e & 3)) & 1)) {
                    zero(v[e]);
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) s[mt][e >> 2][e & 3] = -INFINITY;
                }
        }
        w.weigh(s);
        w.values(s, v);
        if (more) tl.template values<G::VB>(v, g, rr);
    }

    // the nodes themselves, with the last split
    if (it.split == it.splits - 1 && kw == KW - 1) {
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
#pragma unroll
            for (int h = 0; h < 2; ++h) load_key(k[h], kn + min(n0 + 16 * h + rr, count - 1) * a.k_stride, g);
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
                        // (every weight of a lane is asked for, so that none is held by a varying index)
                        const int from = ((x & 15) >> 2) * 16 + rr;
                        float p = 0.f;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float pe = __shfl(s[mt][e >> 2][e & 3], from);
                            if (e == (x >> 4) * 4 + (x & 3)) p = pe;
                        }
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

    // waves with the same rows, joined two by two
    for (int step = KW >> 1; step; step >>= 1) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            const int at = (kw & (step - 1)) * a.RW + rw;
            if (kw >= step && kw < 2 * step) {
                s_ml[at][0][lane] = w.m[mt];
                s_ml[at][1][lane] = w.l[mt];
#pragma unroll
                for (int t = 0; t < G::NT; ++t) s_o[at][t][lane] = w.o[mt][t];
            }
            __syncthreads();
            if (kw < step) {
                const float m = s_ml[at][0][lane], top = fmaxf(w.m[mt], m), base = top == -INFINITY ? 0.f : top;
                const float f0 = fexp2(w.m[mt] - base), f1 = fexp2(m - base);
                w.m[mt] = top;
                w.l[mt] = w.l[mt] * f0 + s_ml[at][1][lane] * f1;
#pragma unroll
                for (int t = 0; t < G::NT; ++t) w.o[mt][t] = w.o[mt][t] * f0 + s_o[at][t][lane] * f1;
            }
            __syncthreads();
        }
    }
    if (kw) return;

#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int row = row0 + mt * 16 + rr;
        float sum = w.l[mt];
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (row >= M) continue;
        if (it.splits == 1) {   // the result
            const bool none = node[mt] >= count || sum == 0.f;
            const float inv = none ? 0.f : 1.f / sum;
            const long at = ((long)r * a.N + node[mt]) * a.h_q + kvh * a.G + row - node[mt] * a.G;
            Out *out = static_cast<Out *>(a.o) + at * D;
#pragma unroll
            for (int j = 0; j < G::NV; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    Out *p = out + j * 16 * G::EV + (4 * g + i) * G::EV;
                    float y[G::EV];
#pragma unroll
                    for (int e = 0; e < G::EV; ++e) y[e] = none ? 0.f : w.o[mt][j * G::EV + e][i] * inv;
#pragma unroll
                    for (int e = 0; e < G::EV; e += 4) st4(p + e, y[e], y[e + 1], y[e + 2], y[e + 3]);
                }
            if (a.lse && g == 0) a.lse[at] = none ? -INFINITY : (w.m[mt] + __log2f(sum)) * 0.6931471805599453f;
        } else {                // the split's part: rows of [d] and (maximum, sum)
            const long at = ((long)pair * a.h_kv + kvh) * a.rows_padded + row;
            float *po = a.part_o + at * D;
            if (g == 0) {
                a.part_ml[2 * at] = w.m[mt];
                a.part_ml[2 * at + 1] = sum;
            }
#pragma unroll
            for (int j = 0; j < G::NV; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int e = 0; e < G::EV; e += 4)
                        st4(po + j * 16 * G::EV + (4 * g + i) * G::EV + e, w.o[mt][j * G::EV + e][i], w.o[mt][j * G::EV + e + 1][i],
                            w.o[mt][j * G::EV + e + 2][i], w.o[mt][j * G::EV + e + 3][i]);
        }
    }
}

// One workgroup per (request, key head, 16 rows), 16 lanes to a row:
// o = sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s.
template <typename Out, int D> __global__ void __launch_bounds__(256) bdgdn_tree_attn_join_kernel(AttnArgs a, int row_tiles)
{
    constexpr int C = D / 64;   // float4s of a lane
    const int tile = blockIdx.x % row_tiles, rest = blockIdx.x / row_tiles, kvh = rest % a.h_kv, r = rest / a.h_kv;
    const int base = a.info[2 * r], splits = a.info[2 * r + 1];
    if (splits == 1) return;   // written by its one split
    const int c = threadIdx.x & 15, lane = threadIdx.x & 63, row = tile * 16 + (threadIdx.x >> 4);
    if (row >= a.N * a.G) return;
    const long stride = (long)a.h_kv * a.rows_padded;   // rows from one split to the next
    const long at0 = ((long)base * a.h_kv + kvh) * a.rows_padded + row;
    float top = -INFINITY;
    for (int s = c; s < splits; s += 16) top = fmaxf(top, a.part_ml[2 * (at0 + s * stride)]);
#pragma unroll
    for (int o = 8; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    const float ref = top == -INFINITY ? 0.f : top;
    f32x4 o[C] = {};
    float l = 0.f;
    for (int s0 = 0; s0 < splits; s0 += 16) {
        float f = 0.f;
        if (s0 + c < splits) {
            const long at = at0 + (s0 + c) * stride;
            f = fexp2(a.part_ml[2 * at] - ref);
            l += f * a.part_ml[2 * at + 1];
        }
        const int n = min(16, splits - s0);
#pragma unroll 8
        for (int i = 0; i < n; ++i) {
            const float fi = __shfl(f, (lane & 48) + i);
            const f32x4 *po = reinterpret_cast<const f32x4 *>(a.part_o + (at0 + (s0 + i) * stride) * D) + c;
#pragma unroll
            for (int x = 0; x < C; ++x) o[x] += fi * po[16 * x];
        }
    }
#pragma unroll
    for (int x = 8; x; x >>= 1) l += __shfl_xor(l, x);
    const int n = row / a.G, count = a.count ? min(max(a.count[r], 0), a.N) : a.N;
    const bool none = n >= count || l == 0.f;
    const long at = ((long)r * a.N + n) * a.h_q + kvh * a.G + row - n * a.G;
    Out *out = static_cast<Out *>(a.o) + at * D + 4 * c;
    const float inv = none ? 0.f : 1.f / l;
#pragma unroll
    for (int x = 0; x < C; ++x) {
        const f32x4 y = none ? f32x4{0, 0, 0, 0} : o[x] * inv;
        st4(out + 64 * x, y[0], y[1], y[2], y[3]);
    }
    if (a.lse && c == 0) a.lse[at] = none ? -INFINITY : (top + __log2f(l)) * 0.6931471805599453f;
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

template <typename T, int D, int MT, bool F32OUT> void launch_m(const AttnPlan &p, const AttnArgs &a, hipStream_t s)
{
    constexpr bool SP = sizeof(T) == 2 && F32OUT;
    typedef typename std::conditional<F32OUT, float, __bf16>::type Out;
    if (a.page % kTile == 0) bdgdn_tree_attn_kernel<T, D, MT, SP, true, Out><<<p.grid, 64 * kWaves, 0, s>>>(a);
    else bdgdn_tree_attn_kernel<T, D, MT, SP, false, Out><<<p.grid, 64 * kWaves, 0, s>>>(a);
    const int row_tiles = (a.N * a.G + 15) / 16;
    bdgdn_tree_attn_join_kernel<Out, D><<<a.R * a.h_kv * row_tiles, 256, 0, s>>>(a, row_tiles);
}

template <typename T, int D, bool F32OUT> hipError_t launch_d(const AttnPlan &p, const AttnArgs &a, hipStream_t s)
{
    constexpr int most = most_mt(sizeof(T) == 2, D);
    if (p.mt == 1) launch_m<T, D, 1, F32OUT>(p, a, s);
    else if (p.mt == 2) launch_m<T, D, (most < 2 ? 1 : 2), F32OUT>(p, a, s);
    else launch_m<T, D, most, F32OUT>(p, a, s);
    return hipGetLastError();
}

}  // namespace

AttnPlan attn_plan(bool bf16, int d, int R, int N, int h_q, int h_kv)
{
    AttnPlan p;
    const int M = N * (h_q / h_kv);
    const int groups = M <= 16 ? 1 : M <= 32 ? 2 : 4, most = most_mt(bf16, d);
    p.mt = groups < most ? groups : most;
    const int waves = (M + 16 * p.mt - 1) / (16 * p.mt);
    p.RW = waves <= 1 ? 1 : waves <= 2 ? 2 : 4;
    p.RG = (waves + p.RW - 1) / p.RW;
    p.rows_padded = p.RG * p.RW * 16 * p.mt;
    const long heads = (long)h_kv * p.RG;
    const long items = (p.mt == 4 ? 512 : 768) / heads;
    p.items = (int)(items < 1 ? 1 : items);
    const long units = ((long)p.items + R) * h_kv;   // (request, split, key head) triples at most
    p.grid = (int)((units + 7) / 8 * 8 * p.RG);
    const size_t rows = (size_t)units * p.rows_padded;
    p.ml_at = ((size_t)R * 8 + 255) & ~(size_t)255;
    p.o_at = p.ml_at + ((rows * 8 + 255) & ~(size_t)255);
    p.bytes = p.o_at + rows * d * 4;
    return p;
}

hipError_t launch_tree_attn(bool bf16, bool f32_out, int d, const AttnPlan &p, AttnArgs &a, void *workspace, hipStream_t s)
{
    a.RW = p.RW;
    a.RG = p.RG;
    a.items = p.items;
    a.rows_padded = p.rows_padded;
    char *ws = static_cast<char *>(workspace);
    a.info = reinterpret_cast<int32_t *>(ws);
    a.part_ml = reinterpret_cast<float *>(ws + p.ml_at);
    a.part_o = reinterpret_cast<float *>(ws + p.o_at);
#define BDGDN_ATTN(T, F) (d == 64 ? launch_d<T, 64, F>(p, a, s) : d == 128 ? launch_d<T, 128, F>(p, a, s) : launch_d<T, 256, F>(p, a, s))
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
