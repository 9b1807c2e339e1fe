// attn_kernels.hip -- attention of a block of nodes over a paged cache and over the nodes
// themselves: the kernel for fp32, and for few rows over pages of any size, the joining kernel,
// tree masks, dispatch.  (bf16 over pages of whole runs of 16 tokens takes the kernel of
// attn_staged_kernels.hip, which is as fast or faster: one node on 64 requests of up to 4096 tokens
// 110.5 against 115 us, four 122.5 against 122, eight 126 against 134, 32 174 against 231.)
//
// One wave streams its tiles from memory to registers, the next keys requested when the scores
// are done with these and the next values when the output is.  Four waves are a workgroup:
// those with different rows take the same keys, those with the same rows every KW-th tile,
// and are joined through LDS.  Latency bounds it: a wave has one tile on its way at a time.  3 requests of up to 1003
// tokens in fp32, 15 rows of 64 to a key head: 9 us, and 4 to join them.
#include <type_traits>

#include "attn.hpp"

namespace bdgdn {

namespace {

constexpr int kWaves = 4;          // of a workgroup

// Waves of a SIMD that a kernel's registers allow (two of up to 256, one of more).
constexpr int waves_per_simd(bool bf16, int d) { return d == 64 || (bf16 && d == 128) ? 2 : 1; }

template <typename T, int D, int MT, bool HALVES, typename Out>
__global__ void __launch_bounds__(64 * kWaves, waves_per_simd(sizeof(T) == 2, D)) bdgdn_tree_attn_kernel(AttnArgs a)
{
    typedef Geo<T, D> G;
    __shared__ f32x4 s_o[2][G::NT][64];
    __shared__ float s_ml[2][2][64];
    const int wave = wave_id(), kw = wave / a.RW, rw = wave - kw * a.RW, KW = kWaves / a.RW;
    // workgroups with the same keys and other rows are neighbours on one XCD (their numbers
    // are equal modulo 8)
    const int x = blockIdx.x & 7, y = blockIdx.x >> 3;
    const int unit = y / a.RG * 8 + x, rg = y % a.RG;
    const int range = unit / a.h_kv, kvh = unit - range * a.h_kv;
    Range span = find_range(a, range, threadIdx.x & 63);
    Wave<T, D, MT> w;
    const int row0 = (rg * a.RW + rw) * 16 * MT;   // of this wave's rows
    for (; span.pos < span.end; next_piece(a, span)) {
        const int lane = lane_anew(), g = lane >> 4, rr = lane & 15;
        const Piece it = piece_of(a, span, range);
        if (it.none) continue;
        const int count = a.count ? min(max(a.count[it.r], 0), a.N) : a.N;
        if (!a.uncut && span.off == 0 && kvh == 0 && rg == 0 && threadIdx.x == 0) note_request(a, span);
        w.init(a.c);
        int node[MT];
        load_rows(w, a, it.r, kvh, row0, node, g, rr);

        // every KW-th tile for this wave
        const int t0 = it.t0 + kw, t1 = it.t1;
        Tiles<HALVES> tl(a, it.r, kvh, it.len, lane);
        u32x4 k[2][G::NK], v[8][G::NV];
        undefine(k);
        undefine(v);
        if (t0 < t1) {
            tl.look_up(t0);
            tl.go(t0);
            tl.keys(k, g, rr);
            tl.template values<G::VB>(v, g, rr);
            if (t0 + KW < t1) tl.look_up(t0 + KW);
        }
        sign_rows(w, a);
        for (int t = t0; t < t1; t += KW) {
            f32x4 st[1][MT][2];
            f32x4(&s)[MT][2] = st[0];
            w.scores(s, k);
            const uint32_t seen = tl.seen;
            const bool more = t + KW < t1;
            if (more) {
                tl.go(t + KW);
                tl.keys(k, g, rr);
                if (t + 2 * KW < t1) tl.look_up(t + 2 * KW);
            }
            if (seen != ~0u) {
                w.hide(s, seen, g);
                w.hide(v, seen, g);
            }
            w.weigh(st);
            w.values(s, v);
            if (more) tl.template values<G::VB>(v, g, rr);
        }
        if (it.nodes && kw == KW - 1) attend_nodes(w, a, it.r, kvh, count, node, g, rr);
        join_waves(w, s_o, s_ml, kw, rw, KW, a.RW, lane);
        if (kw == 0) write_rows<Out>(w, a, it, kvh, count, row0, node, g, rr);
    }
}

// Threads of a joining workgroup, lanes to a row (16 where the pieces are few and a lane has to
// ask for more of each: 64 x 32 nodes 13.4 us, 17.8 with 32 lanes), and rows of a workgroup; W waves
// share the pieces of one wave's rows.
constexpr int join_threads(int W) { return W > 4 ? 64 * W : 256; }
constexpr int join_lanes(int d, int W) { return W == 1 ? 16 : d / 4; }
constexpr int join_rows(int d, int W) { return join_threads(W) / W / join_lanes(d, W); }

// One workgroup per (request, key head, some rows):
// o = sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s over the pieces s of a request.
// Bound by memory where there are many requests (64 in two pieces each, 128 rows of 128 to a
// key head: 13.4 us, 70 MB), by latency where there are few.
template <typename Out, int D, int W> __global__ void __launch_bounds__(join_threads(W)) bdgdn_tree_attn_join_kernel(AttnArgs a, int row_tiles)
{
    constexpr int LANES = join_lanes(D, W), ROWS = join_rows(D, W), C = D / 4 / LANES;   // C float4s of a lane
    const int tile = blockIdx.x % row_tiles, rest = blockIdx.x / row_tiles, kvh = rest % a.h_kv, r = rest / a.h_kv;
    const int size = a.info[0], pos = a.info[1 + 2 * r], w0 = pos / size, splits = (pos + a.info[2 + 2 * r] - 1) / size - w0 + 1;
    if (splits == 1) return;   // one piece, whose workgroup wrote the result
    const int lane = threadIdx.x & 63, wave = wave_id(), part = wave % W, c = lane % LANES;
    const int row = tile * ROWS + wave / W * (64 / LANES) + lane / LANES;
    const bool there = row < a.N * a.G;
    // the first piece ends its range unless it begins there too, the others begin theirs
    const int second = pos % size != 0;
    const auto place = [&](int s) {
        return ((long)(2 * (w0 + s) + (s == 0 ? second : 0)) * a.h_kv + kvh) * a.rows_padded + row;
    };
    // this wave's pieces
    const int per = (splits + W - 1) / W, first = part * per, last = min(first + per, splits);
    float top = -INFINITY, l = 0.f;
    f32x4 o[C] = {};
    if (there) {
        for (int s = first + c; s < last; s += LANES) top = fmaxf(top, a.part_ml[2 * place(s)]);
#pragma unroll
        for (int x = LANES / 2; x; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
        const float ref = top == -INFINITY ? 0.f : top;
        for (int s0 = first; s0 < last; s0 += LANES) {
            float f = 0.f;
            if (s0 + c < last) {
                const long at = place(s0 + c);
                f = fexp2(a.part_ml[2 * at] - ref);
                l += f * a.part_ml[2 * at + 1];
            }
            const int n = min(LANES, last - s0);
#pragma unroll 8
            for (int i = 0; i < n; ++i) {
                const float fi = __shfl(f, lane - c + i);
                const f32x4 *po = reinterpret_cast<const f32x4 *>(a.part_o + place(s0 + i) * D) + c;
#pragma unroll
                for (int x = 0; x < C; ++x) o[x] += fi * po[LANES * x];
            }
        }
#pragma unroll
        for (int x = LANES / 2; x; x >>= 1) l += __shfl_xor(l, x);
    }
    if constexpr (W > 1) {
        static_assert(C == 1, "");
        __shared__ f32x4 s_o[W][64];
        __shared__ float s_ml[W][2][64];
        s_o[part][lane] = o[0];
        s_ml[part][0][lane] = top;
        s_ml[part][1][lane] = l;
        __syncthreads();
        if (part) return;
        for (int w = 1; w < W; ++w) top = fmaxf(top, s_ml[w][0][lane]);
        const float ref = top == -INFINITY ? 0.f : top;
        o[0] = f32x4{0, 0, 0, 0};
        l = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float f = fexp2(s_ml[w][0][lane] - ref);
            o[0] += f * s_o[w][lane];
            l += f * s_ml[w][1][lane];
        }
    }
    if (!there) return;
    const int n = row / a.G, count = a.count ? min(max(a.count[r], 0), a.N) : a.N;
    const bool none = n >= count || l == 0.f;
    const long at = ((long)r * a.N + n) * a.h_q + kvh * a.G + row - n * a.G;
    const float inv = none ? 0.f : 1.f / l;
#pragma unroll
    for (int x = 0; x < C; ++x) {
        const f32x4 y = none ? f32x4{0, 0, 0, 0} : o[x] * inv;
        st4(static_cast<Out *>(a.o) + at * D + 4 * (c + LANES * x), y[0], y[1], y[2], y[3]);
    }
    if (a.lse && c == 0) a.lse[at] = none ? -INFINITY : (top + __log2f(l)) * 0.6931471805599453f;
}

template <typename Out, int D, int W> void launch_join(const AttnArgs &a, hipStream_t s)
{
    const int row_tiles = (a.N * a.G + join_rows(D, W) - 1) / join_rows(D, W);
    bdgdn_tree_attn_join_kernel<Out, D, W><<<a.R * a.h_kv * row_tiles, join_threads(W), 0, s>>>(a, row_tiles);
}

__global__ void __launch_bounds__(64) bdgdn_tree_mask_kernel(int N, const int32_t *parent, uint64_t *mask, int32_t *depth)
{
    // one wave per request, lane n for node n; 2 to 5 us, a launch's own
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

// 16-row groups of a wave at most: what its registers hold, 512 a lane.
constexpr int most_mt(int d) { return d == 256 ? 1 : 2; }

template <typename T, int D, int MT, bool F32OUT> hipError_t launch_m(const AttnPlan &p, const AttnArgs &a, hipStream_t s)
{
    typedef typename std::conditional<F32OUT, float, __bf16>::type Out;
    constexpr bool HALVES = sizeof(T) == 4;   // (bf16 over such pages is the staged kernel's)
    if (HALVES && a.page % 16 == 0) bdgdn_tree_attn_kernel<T, D, MT, HALVES, Out><<<p.grid, 64 * kWaves, 0, s>>>(a);
    else bdgdn_tree_attn_kernel<T, D, MT, false, Out><<<p.grid, 64 * kWaves, 0, s>>>(a);
    return hipGetLastError();
}

template <typename T, int D, bool F32OUT> hipError_t launch_d(const AttnPlan &p, const AttnArgs &a, hipStream_t s)
{
    constexpr int most = most_mt(D);
    hipError_t e = p.staged ? launch_tree_attn_staged(F32OUT, D, p.grid, a, s)
                   : p.mt == 1 ? launch_m<T, D, 1, F32OUT>(p, a, s)
                               : launch_m<T, D, most, F32OUT>(p, a, s);
    if (e != hipSuccess || p.uncut) return e;
    typedef typename std::conditional<F32OUT, float, __bf16>::type Out;
    // Four waves to a row's pieces where requests have eight or more, sixteen from 64 on.  One node of
    // 4 heads of 64 over 57078 tokens, in 446 pieces: the call 24 us, 57 with four; 2 requests in 32
    // pieces each, 96 rows of 128: the joining 10 us, 19 with one.  With two pieces to a request most of
    // them would have nothing to do.
    if (p.ranges >= 64 * a.R) launch_join<Out, D, 16>(a, s);
    else if (p.ranges >= 8 * a.R) launch_join<Out, D, 4>(a, s);
    else launch_join<Out, D, 1>(a, s);
    return hipGetLastError();
}

}  // namespace

AttnPlan attn_plan(bool bf16, int d, int page, long most, int R, int N, int h_q, int h_kv)
{
    AttnPlan p;
    const int M = N * (h_q / h_kv);
    // Pages of other sizes: a staged wave's rows have an address to a lane, which pays from 33 rows to a
    // key head on.  16 requests of 100 to 4000 tokens, pages of 24 and 8 key heads of 256: 96 rows 126 us
    // staged and 196 streamed, 36 rows 81 and 106, but 24 rows 76 and 65, four 73 and 52; pages of 100, 4 heads of
    // 128: 48 rows 28.4 and 29.4, but 32 rows 25 and 28, two (one head of four) 23 and 24.
    p.staged = bf16 && (page % 16 == 0 || M > 32);
    // a staged wave always has 32 rows, idle ones load for the others; a streaming wave has as
    // many 16-row groups as the rows fill, and waves without rows take tiles instead
    p.mt = p.staged ? 2 : M <= 16 ? 1 : most_mt(d);
    const int waves = (M + 16 * p.mt - 1) / (16 * p.mt);
    p.RW = waves <= 1 && !p.staged ? 1 : waves <= 2 ? 2 : 4;
    p.RG = (waves + p.RW - 1) / p.RW;
    p.rows_padded = p.RG * p.RW * 16 * p.mt;
    // one range for every workgroup that the chip holds at once (one or two to a compute unit)
    const long heads = (long)h_kv * p.RG, ranges = 256 * (p.staged ? (d == 256 ? 1 : 2) : waves_per_simd(bf16, d)) / heads;
    // A table of few columns holds no long request: one workgroup (of a key head) takes each, and
    // nothing is joined.  Room for 128 tokens, 32 query heads on 8 of 128: 64 requests of 8 nodes 13.0 us where
    // cutting takes 23.7, of 64 nodes 42 for 59.5, one of one node 10.5 for 13.5 (one of 64 nodes on
    // one head of 256 21.9 for 22.3).  For 256: 18.0 for 26.9, 13.6 for 13.5; but with heads of 256 one
    // of one node 21.2 for 17.3, and with 192 rows in fp32 51 for 32.  For 512: one of one node 20 for
    // 13.6.  It goes by the table, which the host knows: short requests in a table with room for a
    // long context are cut.
    p.uncut = most <= 128 || (most <= 256 && M <= 64 && d <= 128);
    p.ranges = p.uncut ? R : (int)(ranges < 1 ? 1 : ranges);
    p.least = 4;   // tiles of a range, one to a wave
    p.grid = (int)(((long)p.ranges * h_kv + 7) / 8 * 8 * p.RG);
    const size_t rows = p.uncut ? 0 : 2 * (size_t)p.ranges * h_kv * p.rows_padded;
    p.ml_at = ((size_t)(1 + 2 * (size_t)R) * 4 + 255) & ~(size_t)255;
    p.o_at = p.ml_at + ((rows * 8 + 255) & ~(size_t)255);
    p.bytes = p.o_at + rows * d * 4;
    return p;
}

hipError_t launch_tree_attn(bool bf16, bool f32_out, int d, const AttnPlan &p, AttnArgs &a, void *workspace, hipStream_t s)
{
    a.RW = p.RW;
    a.RG = p.RG;
    a.ranges = p.ranges;
    a.least = p.least;
    a.uncut = p.uncut;
    a.node_units = 4 + p.RW * p.mt / 2;
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
