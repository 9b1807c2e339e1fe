// attn.hpp -- attention of a block of nodes over a paged cache: the parts that its kernels share.
//
// The rows that share a key head (N nodes x G query heads, M in all) are taken together: 16 MT
// of them by one wave, 32 keys at a time.  Both
// products are formed transposed, S^T = K Q^T and O^T = V^T P^T, so that a lane holds one row's
// scores (row = lane & 15) and the accumulators of the first product are the operand of the
// second as they stand; the transposed values are made from 16-byte loads by byte permutes.
#pragma once

#include "common.hpp"
#include "round.hpp"

namespace bdgdn {

namespace {

constexpr int kTile = 32;          // keys of a step
typedef unsigned int u32x2v __attribute__((ext_vector_type(2)));

template <typename T, int D> struct Geo {
    static constexpr int kRow = D * sizeof(T);          // bytes of a row
    static constexpr int NK = kRow / 64;                // 16-byte chunks of a key row in a lane
    static constexpr int VB = kRow < 256 ? 8 : 16;      // bytes of a chunk of a value row in a lane
    static constexpr int NV = kRow / (16 * VB);         // such chunks
    static constexpr int EV = VB / sizeof(T);           // elements of such a chunk
    static constexpr int NT = D / 16;                   // accumulator tiles of a row group
};

// The lane's number, as new to the compiler: what follows from it is worked out again in each
// turn of a loop, not once before it and kept in registers that the loop needs.
__device__ __forceinline__ int lane_anew()
{
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
    return lane;
}

// Registers without a value that nothing has to be kept for (a variable that is set under a
// condition in a loop would otherwise hold the last turn's).
template <int M, int N> __device__ __forceinline__ void undefine(u32x4 (&x)[M][N])
{
#pragma unroll
    for (int i = 0; i < M; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) asm volatile("" : "=v"(x[i][j]));
}

// Tables that a kernel reads at addresses common to a wave, through the scalar cache: such a
// read is not counted among the vector loads, so waiting for it leaves those in flight.
typedef __attribute__((address_space(4))) const int32_t *TablePtr;

__device__ __forceinline__ TablePtr table_of(const AttnArgs &a, int r)
{
    const int slot = a.slot ? ((TablePtr)(uintptr_t)a.slot)[r] : r;
    return (TablePtr)(uintptr_t)(a.table + (long)slot * a.max_pages);
}

__device__ __forceinline__ float max_over_groups(float x)
{
    // the swaps leave a value and its partner's in the two results
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// The work of all requests in one row, a request's cached tiles followed by its nodes, is cut
// into equal ranges, one to a workgroup (of each key head and row group), whatever the requests'
// lengths.  A range holds the end of one request, whole ones and the beginning of another.  The
// nodes, with the queries and the output, count as a.node_units tiles: what a request costs
// whatever its length.
struct Range {
    int pos, end;              // what is left of the range
    int size;                  // of every range
    int r, off, len, tiles;    // the request at pos, its tile there, its cached tokens and tiles
};

__device__ __forceinline__ int length_of(const AttnArgs &a, int r)
{
    const int slot = a.slot ? a.slot[r] : r;
    if ((unsigned)slot >= (unsigned)a.n_slots) return 0;
    return min(max(a.len[slot], 0), a.max_pages * a.page);
}

__device__ __forceinline__ int tiles_of(int len) { return (len + kTile - 1) / kTile; }

// The length of request g.r, its tiles.
__device__ __forceinline__ void go_to(const AttnArgs &a, Range &g)
{
    const int slot = a.slot ? ((TablePtr)(uintptr_t)a.slot)[g.r] : g.r;
    g.len = (unsigned)slot < (unsigned)a.n_slots ? min(max(((TablePtr)(uintptr_t)a.len)[slot], 0), a.max_pages * a.page) : 0;
    g.tiles = tiles_of(g.len);
}

__device__ __forceinline__ Range find_range(const AttnArgs &a, int w, int lane)
{
    Range g = {};
    if (a.uncut) {
        if (w >= a.R) return g;
        g.r = w;
        go_to(a, g);
        g.end = g.size = g.tiles + a.node_units;
        return g;
    }
    const int len0 = lane < a.R ? length_of(a, lane) : 0;
    int sum = lane < a.R ? tiles_of(len0) + a.node_units : 0;
    for (int r = lane + 64; r < a.R; r += 64) sum += tiles_of(length_of(a, r)) + a.node_units;
#pragma unroll
    for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
    sum = __builtin_amdgcn_readfirstlane(sum);
    g.size = max(a.least, (sum + a.ranges - 1) / a.ranges);
    // (in 64 bits: ranges past the end may lie beyond 2^31)
    const long pos = (long)w * g.size;
    if (pos >= sum) return g;
    g.pos = (int)pos;
    g.end = (int)min(pos + g.size, (long)sum);
    int before = 0;
    for (int r0 = 0; r0 < a.R; r0 += 64) {
        const int r = r0 + lane;
        const int len = r0 == 0 ? len0 : r < a.R ? length_of(a, r) : 0;
        const int n = r < a.R ? tiles_of(len) + a.node_units : 0;
        int inc = n;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int y = __shfl_up(inc, o);
            if (lane >= o) inc += y;
        }
        const int start = before + inc - n;
        const unsigned long long hit = __ballot(g.pos >= start && g.pos < start + n);
        if (hit) {
            const int src = __ffsll(hit) - 1;
            g.r = r0 + src;
            g.off = g.pos - __builtin_amdgcn_readlane(start, src);
            g.len = __builtin_amdgcn_readlane(len, src);
            g.tiles = tiles_of(g.len);
            return g;
        }
        before += __builtin_amdgcn_readlane(inc, 63);
    }
    return g;
}

// What a workgroup does with one request: tiles t0 .. t1 - 1, the nodes where `nodes` (they are
// done where the first of their units lies); nothing where only later units are left.
struct Piece {
    int r, len, t0, t1;
    bool nodes, none, whole;   // whole: the request's only piece
    int part;                  // else its place among the parts: 2 w for a range's first piece, 2 w + 1
};

__device__ __forceinline__ Piece piece_of(const AttnArgs &a, const Range &g, int w)
{
    Piece p;
    const int end = g.off + min(g.tiles + a.node_units - g.off, g.end - g.pos);
    p.r = g.r;
    p.len = g.len;
    p.t0 = min(g.off, g.tiles);
    p.t1 = min(end, g.tiles);
    p.none = g.off > g.tiles;
    p.nodes = !p.none && end > g.tiles;
    p.whole = p.nodes && g.off == 0;
    p.part = 2 * w + (g.pos != (long)w * g.size);
    return p;
}

__device__ __forceinline__ void next_piece(const AttnArgs &a, Range &g)
{
    g.pos += min(g.tiles + a.node_units - g.off, g.end - g.pos);
    if (g.pos >= g.end) return;
    ++g.r;
    g.off = 0;
    go_to(a, g);
}

// What the joining kernel needs to know of a request that a range begins.
__device__ __forceinline__ void note_request(const AttnArgs &a, const Range &g)
{
    a.info[1 + 2 * g.r] = g.pos;
    a.info[2 + 2 * g.r] = g.tiles + 1;
    if (g.pos == 0) a.info[0] = g.size;
}

// One step of 32 keys for MT groups of 16 rows.
template <typename T, int D, int MT> struct Wave {
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

    // keys that are not there: their scores, their values
    __device__ __forceinline__ void hide(f32x4 (&s)[MT][2], uint32_t seen, int g)
    {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (!(seen >> (16 * (e >> 2) + 4 * g + (e & 3)) & 1))
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) s[mt][e >> 2][e & 3] = -INFINITY;
    }
    __device__ __forceinline__ void hide(u32x4 (&v)[8][G::NV], uint32_t seen, int g)
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t there = seen >> (16 * (e >> 2) + 4 * g + (e & 3)) & 1 ? ~0u : 0u;
#pragma unroll
            for (int j = 0; j < G::NV; ++j) v[e][j] &= there;
        }
    }

    // s -> weights exp2(c s - m), for TP tiles at once; the running maximum grows only when a
    // score passes it by more than 2^8, so that the accumulators are seldom rescaled.
    template <int TP> __device__ __forceinline__ void weigh(f32x4 (&s)[TP][MT][2])
    {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            float top = s[0][mt][0][0];
#pragma unroll
            for (int t = 0; t < TP; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i) top = fmaxf(top, s[t][mt][h][i]);
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
            for (int t = 0; t < TP; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        s[t][mt][h][i] = fexp2(fmaf(s[t][mt][h][i], c, -base));
                        l[mt] += s[t][mt][h][i];
                    }
        }
    }

    // o += V^T P^T; v[e] is the lane's part of value row
    // 16 (e / 4) + 4 g + e % 4.  With bf16 inputs the weights go to the matrix units in two bf16 parts
    // (16 bits), so that a bf16 result is an fp32 one rounded: with one part it is off by
    // 2.2e-3 in the mean square, with two by its own 1.65e-3.  Where memory bounds a call that costs
    // 0.5 to 6 % (64 requests of up to 4096 tokens, 32 heads on 8 of 128, 8 nodes: 126.8 for 126.1 us),
    // where the products do 8 to 17 (32 nodes 171 for 158, 64 nodes 285 for 243, trees of 24 over
    // 128k 221 for 191).  Their sum is of the whole ones.
    __device__ __forceinline__ void values(const f32x4 (&p)[MT][2], const u32x4 (&v)[8][G::NV])
    {
        if constexpr (sizeof(T) == 2) {
            bf16x8 hi[MT], lo[MT];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float x = p[mt][e >> 2][e & 3];
                    // The first part is cut off, not rounded, and the second is more than zero by
                    // the 2^-23 of x: of one sign, they take an infinite value over as it is.
                    const uint32_t top = __float_as_uint(x) & 0xffff0000u;
                    hi[mt][e] = __builtin_bit_cast(__bf16, (unsigned short)(top >> 16));
                    lo[mt][e] = (__bf16)__builtin_fmaf(x, 0x1.000002p0f, -__uint_as_float(top));
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
                    for (int part = 0; part < 2; ++part)
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) {
                            f32x4 &o0 = o[mt][j * G::EV + 2 * w], &o1 = o[mt][j * G::EV + 2 * w + 1];
                            o0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a0, part ? lo[mt] : hi[mt], o0, 0, 0, 0);
                            o1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a1, part ? lo[mt] : hi[mt], o1, 0, 0, 0);
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

// tok / page.
__device__ __forceinline__ int column(const AttnArgs &a, int tok)
{
    return a.page_mul ? (int)(__umulhi((unsigned)tok, a.page_mul) >> a.page_shift) : tok;
}

// Where the keys of a tile of cached tokens lie.  HALVES: a page holds whole runs of 16
// tokens, so a tile is two base addresses; otherwise lane x finds key x & 31 and the others
// ask it.  A key that is not there reads the pool's first tokens instead and is left out by
// `seen`.
template <bool HALVES> struct Tiles {
    const AttnArgs &a;
    TablePtr table;
    const unsigned char *kp, *vp;
    int len, lane;
    uint32_t at[2];       // HALVES: of the halves' first tokens, else of this lane's, in 16 bytes
    uint32_t seen;        // keys that are there
    int pages[2];         // the next tile's, ahead of its use

    __device__ __forceinline__ Tiles(const AttnArgs &args, int r, int kvh, int len_, int lane_) : a(args), len(len_), lane(lane_)
    {
        table = table_of(a, r);
        kp = static_cast<const unsigned char *>(a.kp) + (long)kvh * a.head_stride;
        vp = static_cast<const unsigned char *>(a.vp) + (long)kvh * a.head_stride;
    }
    __device__ __forceinline__ void look_up(int t)
    {
        if (HALVES) {
#pragma unroll
            for (int h = 0; h < 2; ++h) pages[h] = t * kTile + 16 * h < len ? table[column(a, t * kTile + 16 * h)] : -1;
        } else {
            const int tok = t * kTile + (lane & 31);
            pages[0] = tok < len ? ((const int32_t *)(uintptr_t)table)[column(a, tok)] : -1;
        }
    }
    __device__ __forceinline__ bool place(int tok, int page, uint32_t &where) const
    {
        const bool there = (unsigned)page < (unsigned)a.n_pages;
        where = there ? page * a.page16 + (uint32_t)(tok - column(a, tok) * a.page) * a.token16 : 0;
        return there;
    }
    // on to the tile that was looked up
    __device__ __forceinline__ void go(int t)
    {
        if (HALVES) {
            seen = 0;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int tok = t * kTile + 16 * h, left = len - tok;
                if (place(tok, pages[h], at[h])) seen |= (left >= 16 ? 0xffffu : (1u << left) - 1) << (16 * h);
            }
        } else {
            seen = (uint32_t)__ballot(place(t * kTile + (lane & 31), pages[0], at[0]));
        }
    }
    __device__ __forceinline__ const unsigned char *row(const unsigned char *p, int h, int i, int lane_key) const
    {
        // key 16 h + i + lane_key, of which 16 h + i is the same for all lanes
        if (HALVES) return p + (long)at[h] * 16 + (long)(i * a.token16) * 16 + (uint32_t)(lane_key * a.token16 * 16);
        return p + (long)__shfl(at[0], 16 * h + i + lane_key) * 16;
    }
    template <int NK> __device__ __forceinline__ void keys(u32x4 (&k)[2][NK], int g, int rr) const
    {
#pragma unroll
        for (int h = 0; h < 2; ++h) load_key(k[h], row(kp, h, 0, rr), g);
    }
    template <int VB, int NV> __device__ __forceinline__ void values(u32x4 (&v)[8][NV], int g, int rr) const
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) load_value<VB>(v[e], row(vp, e >> 2, e & 3, 4 * g), rr);
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

// The queries of a wave's 16 MT rows from row0 on, and the nodes that they belong to.
template <typename T, int D, int MT>
__device__ __forceinline__ void load_rows(Wave<T, D, MT> &w, const AttnArgs &a, int r, int kvh, int row0, int (&node)[MT],
                                          int g, int rr)
{
    typedef Geo<T, D> G;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int row = min(row0 + mt * 16 + rr, a.N * a.G - 1);
        node[mt] = row / a.G;
        load_key(w.q[mt], static_cast<const unsigned char *>(a.q) + ((long)r * a.N + node[mt]) * a.q_stride +
                              (long)(kvh * a.G + row - node[mt] * a.G) * G::kRow, g);
    }
}

template <typename T, int D, int MT> __device__ __forceinline__ void sign_rows(Wave<T, D, MT> &w, const AttnArgs &a)
{
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int j = 0; j < Geo<T, D>::NK; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) w.q[mt][j][i] = (w.q[mt][j][i] & a.q_and) ^ a.q_xor;
}

// The nodes themselves as keys and values, for the rows of one wave.
template <typename T, int D, int MT>
__device__ __forceinline__ void attend_nodes(Wave<T, D, MT> &w, const AttnArgs &a, int r, int kvh, int count,
                                             const int (&node)[MT], int g, int rr)
{
    typedef Geo<T, D> G;
    u32x4 k[2][G::NK], v[8][G::NV];
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
            load_value<G::VB>(v[e], vn + min(key, count - 1) * a.v_stride, rr);
            const uint32_t live_bits = key < count ? ~0u : 0u;
#pragma unroll
            for (int j = 0; j < G::NV; ++j) {
                v[e][j] &= live_bits;
                fine &= finite_words(v[e][j], sizeof(T) == 4);
            }
        }
        f32x4 st[1][MT][2];
        f32x4(&s)[MT][2] = st[0];
        w.scores(s, k);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (!(sees[mt] >> (n0 + 16 * (e >> 2) + 4 * g + (e & 3)) & 1)) s[mt][e >> 2][e & 3] = -INFINITY;
        w.weigh(st);
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

// Waves with the same rows (RW apart, KW of them) joined two by two; the first of them holds
// the result.  s_o and s_ml have room for KW / 2 * RW waves.
template <typename T, int D, int MT>
__device__ __forceinline__ void join_waves(Wave<T, D, MT> &w, f32x4 (*s_o)[Geo<T, D>::NT][64], float (*s_ml)[2][64],
                                           int kw, int rw, int KW, int RW, int lane)
{
    typedef Geo<T, D> G;
    for (int step = KW >> 1; step; step >>= 1) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            const int at = (kw & (step - 1)) * RW + rw;
            if (kw >= step && kw < 2 * step) {
                s_ml[at][0][lane] = w.m[mt];
                s_ml[at][1][lane] = w.l[mt];
#pragma unroll
                for (int t = 0; t < G::NT; ++t) s_o[at][t][lane] = w.o[mt][t];
            }
            lds_barrier();
            if (kw < step) {
                const float m = s_ml[at][0][lane], top = fmaxf(w.m[mt], m), base = top == -INFINITY ? 0.f : top;
                const float f0 = fexp2(w.m[mt] - base), f1 = fexp2(m - base);
                w.m[mt] = top;
                w.l[mt] = w.l[mt] * f0 + s_ml[at][1][lane] * f1;
#pragma unroll
                for (int t = 0; t < G::NT; ++t) w.o[mt][t] = w.o[mt][t] * f0 + s_o[at][t][lane] * f1;
            }
            lds_barrier();
        }
    }
}

// The rows of one wave: the result where the request is one piece, else the piece's part.
template <typename Out, typename T, int D, int MT>
__device__ __forceinline__ void write_rows(const Wave<T, D, MT> &w, const AttnArgs &a, const Piece &it, int kvh,
                                           int count, int row0, const int (&node)[MT], int g, int rr)
{
    typedef Geo<T, D> G;
    const int r = it.r, M = a.N * a.G;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int row = row0 + mt * 16 + rr;
        float sum = w.l[mt];
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (row >= M) continue;
        if (it.whole) {          // the result
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
        } else {                // rows of [d] and (maximum, sum)
            const long at = ((long)it.part * a.h_kv + kvh) * a.rows_padded + row;
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

}  // namespace

}  // namespace bdgdn
