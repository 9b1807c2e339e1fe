// attn_staged_kernels.hip -- attention of a block of nodes over a paged cache: the kernel for bf16
// over pages of whole runs of 16 tokens (HALVES: a tile is two runs of rows), and for many rows
// over pages of any size (each lane asks the one that has looked a key's page up).
//
// Four waves are a workgroup of RW x KW: RW (two or four) have 32 rows each and read the same
// tiles, KW take different tiles.  Tiles go from memory to LDS without passing through
// registers, S stages of two tiles (one where heads of 256 and four row waves need the room),
// one barrier a stage; the softmax takes a wave's tiles of a stage in one turn.  Two workgroups
// share a compute unit (one with heads of 256, whose accumulators need the registers), so that
// the ends of one's pieces and its barriers pass while the other computes.  A row of D elements
// is D / 8 chunks of 16 bytes; chunk c of key x lies at place c ^ (x & 15) of its row
// (c ^ (x / 2 & 7) in rows of 8 chunks), so that the 16 lanes that read one chunk of 16 keys, and
// those that read 16 chunks of one key, meet different banks.
//
// What bounds it: memory, up to 16 nodes or so (32 query heads on 8 of 128): one node on 64 requests of up
// to 4096 tokens takes 110.5 us, 5.0 TB/s, 16 take 142.  From 32 nodes on the products and the softmax do: 64
// requests of 2048 tokens and 32 nodes take 147.5 us, of which the loads alone (the products taken out of a
// copy) 116; 64 nodes on up to 4096 take 285, 510 TFLOP/s of the formula's operations (a value's product
// is done twice), the vector units busy 54 % of the time and the matrix units 37.
#include <mutex>
#include <type_traits>

#include "attn.hpp"

namespace bdgdn {

namespace {

typedef __attribute__((address_space(1))) const void *GlobalPtr;
typedef __attribute__((address_space(3))) void *LdsPtr;

template <int D, int RW> struct Staged {
    static constexpr int CH = D / 8;                    // chunks of a row
    static constexpr int W = 4;                         // waves
    static constexpr int KW = W / RW;
    static constexpr int TP = D == 256 ? 1 : 2 / KW;    // tiles that a wave takes at once
    static constexpr int TILES = KW * TP;               // of a stage
    static constexpr int STAGE = TILES * 64 * CH;       // chunks of a stage: tiles x (keys, values) x 32 rows
    static constexpr int LOADS = TILES * CH / W;        // of a wave for a stage, 64 chunks each
    static constexpr int S = (D == 256 ? 131072 : 65536) / (STAGE * 16);
    static constexpr int JOIN = (KW / 2) * RW * (D / 16 * 1024 + 512);
    static constexpr int LDS = S * STAGE * 16 > JOIN ? S * STAGE * 16 : JOIN;
    static __device__ __forceinline__ int place(int c, int key) { return c ^ (CH == 8 ? (key >> 1) & 7 : key & 15); }
};

template <int N> __device__ __forceinline__ void wait_loads_barrier()
{
    // the memory clobber keeps reads and writes of LDS on their side of the barrier
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

template <int D, int RW, bool HALVES, typename Out>
__global__ void __launch_bounds__(256, D == 256 ? 1 : 2) bdgdn_tree_attn_staged_kernel(AttnArgs a)
{
    typedef __bf16 T;
    typedef Geo<T, D> G;
    typedef Staged<D, RW> X;
    constexpr int CH = X::CH, KW = X::KW, TP = X::TP, S = X::S, LOADS = X::LOADS, ROWS = 64 / CH;   // rows of one load
    extern __shared__ u32x4 lds[];
    __shared__ uint32_t s_seen[S][X::TILES][2];
    const int wave = wave_id(), kw = wave / RW, rw = wave % RW;
    // workgroups with the same keys and other rows are neighbours on one XCD (their numbers
    // are equal modulo 8)
    const int x = blockIdx.x & 7, y = blockIdx.x >> 3;
    const int unit = y / a.RG * 8 + x, rg = y % a.RG;
    const int range = unit / a.h_kv, kvh = unit - range * a.h_kv;
    Range span = find_range(a, range, threadIdx.x & 63);
    Wave<T, D, 2> w;
    const int row0 = (rg * RW + rw) * 32;   // of this wave's rows
    const bool idle = row0 >= a.N * a.G;    // it has none, and only loads

    // this wave's share of a stage: rows [first, first + LOADS ROWS) of the keys or the values of one tile
    const int block = wave * LOADS, ltile = block / CH, first = block % (CH / 2) * ROWS;
    const bool is_value = block / (CH / 2) & 1;
    const unsigned char *pool = static_cast<const unsigned char *>(is_value ? a.vp : a.kp) + (long)kvh * a.head_stride;
    for (; span.pos < span.end; next_piece(a, span)) {
        const int lane = lane_anew(), g = lane >> 4, rr = lane & 15;
        // HALVES (a page holds whole runs of 16 tokens): this lane's chunks behind the first of their run
        uint32_t off[HALVES ? LOADS : 1];
        if (HALVES)
#pragma unroll
            for (int l = 0; l < LOADS; ++l) {
                const int key = first + l * ROWS + lane / CH;
                off[HALVES ? l : 0] = (key & 15) * a.token16 * 16 + X::place(lane % CH, key) * 16;
            }
        // where this lane's chunks of keys and values lie in a tile
        int ko[G::NK], vo[4];
#pragma unroll
        for (int j = 0; j < G::NK; ++j) ko[j] = rr * CH + X::place(4 * j + g, rr);
#pragma unroll
        for (int i = 0; i < 4; ++i) vo[i] = CH == 8 ? ((4 * g + i) * CH + X::place(rr >> 1, 4 * g + i)) * 16 + (rr & 1) * 8
                                                    : ((4 * g + i) * CH + X::place(rr, 4 * g + i)) * 16;
        const Piece it = piece_of(a, span, range);
        if (it.none) continue;
        const int count = a.count ? min(max(a.count[it.r], 0), a.N) : a.N;
        if (!a.uncut && span.off == 0 && kvh == 0 && rg == 0 && threadIdx.x == 0) note_request(a, span);
        const TablePtr table = table_of(a, it.r);
        const int n = (it.t1 - it.t0 + X::TILES - 1) / X::TILES;   // stages
        int pages[2];   // HALVES: of the tile's runs, else of key lane & 31
        const auto look_up = [&](int i) {
            if (!HALVES) {
                const int t = it.t0 + i * X::TILES + ltile, tok = t * kTile + (lane & 31);
                pages[0] = t < it.t1 && tok < it.len ? ((const int32_t *)(uintptr_t)table)[column(a, tok)] : -1;
                return;
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int t = it.t0 + i * X::TILES + ltile, tok = t * kTile + 16 * h;
                pages[h] = t < it.t1 && tok < it.len ? table[column(a, tok)] : -1;
            }
        };
        const auto request = [&](int i) {
            const int tok0 = (it.t0 + i * X::TILES + ltile) * kTile;
            const int buf = i % S;
            if (!HALVES) {
                const int tok = tok0 + (lane & 31);
                const bool there = (unsigned)pages[0] < (unsigned)a.n_pages;
                const uint32_t where = there ? pages[0] * a.page16 + (uint32_t)(tok - column(a, tok) * a.page) * a.token16 : 0;
                const uint32_t seen = (uint32_t)__ballot(there);
                if (!is_value && lane == 0) {
                    s_seen[buf][ltile][0] = seen & 0xffffu;
                    s_seen[buf][ltile][1] = seen >> 16;
                }
#pragma unroll
                for (int l = 0; l < LOADS; ++l) {
                    const int key = first + l * ROWS + lane / CH;
                    const unsigned char *p = pool + (long)(uint32_t)__shfl((int)where, key) * 16 + X::place(lane % CH, key) * 16;
                    __builtin_amdgcn_global_load_lds((GlobalPtr)p, (LdsPtr)&lds[buf * X::STAGE + (block + l) * 64], 16, 0, 0);
                }
                return;
            }
            const unsigned char *at[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int tok = tok0 + 16 * h;
                const bool there = (unsigned)pages[h] < (unsigned)a.n_pages;
                const uint32_t where = there ? pages[h] * a.page16 + (uint32_t)(tok - column(a, tok) * a.page) * a.token16 : 0;
                at[h] = pool + (long)where * 16;
                if (!is_value && lane == 0)
                    s_seen[buf][ltile][h] = !there ? 0u : it.len - tok >= 16 ? 0xffffu : (1u << (it.len - tok)) - 1;
            }
#pragma unroll
            for (int l = 0; l < LOADS; ++l) {
                // (held as 32 bits, so that the address is a scalar base and a lane's offset)
                uint32_t lane_off = off[HALVES ? l : 0];
                asm("" : "+v"(lane_off));
                const unsigned char *p = at[(first + l * ROWS) >> 4] + lane_off;
                __builtin_amdgcn_global_load_lds((GlobalPtr)p, (LdsPtr)&lds[buf * X::STAGE + (block + l) * 64], 16, 0, 0);
            }
        };
        if (n > 0) look_up(0);
        w.init(a.c);
        int node[2];
#pragma unroll
        for (int i = 0; i < S - 1; ++i)
            if (i < n) {
                request(i);
                if (i + 1 < n) look_up(i + 1);
            }
        load_rows(w, a, it.r, kvh, row0, node, g, rr);
        sign_rows(w, a);
        int buf = 0;
        for (int i = 0; i < n; ++i) {
            if (n - 1 - i >= S - 2) wait_loads_barrier<(S - 2) * LOADS>();
            else wait_loads_barrier<0>();
            if (i + S - 1 < n) {
                request(i + S - 1);
                if (i + S < n) look_up(i + S);
            }
            uint32_t seen[TP], any = 0;
#pragma unroll
            for (int tp = 0; tp < TP; ++tp) {
                const int tile = kw + tp * KW;
                seen[tp] = __builtin_amdgcn_readfirstlane(s_seen[buf][tile][0] | s_seen[buf][tile][1] << 16);
                any |= seen[tp];
            }
            const u32x4 *stage = lds + buf * X::STAGE + kw * 64 * CH;
            buf = buf + 1 == S ? 0 : buf + 1;
            if (!any || idle) continue;
            f32x4 s[TP][2][2];
#pragma unroll
            for (int tp = 0; tp < TP; ++tp) {
                u32x4 k[2][G::NK];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int j = 0; j < G::NK; ++j) k[h][j] = stage[tp * KW * 64 * CH + 16 * h * CH + ko[j]];
                w.scores(s[tp], k);
                if (seen[tp] != ~0u) w.hide(s[tp], seen[tp], g);
            }
            w.weigh(s);
#pragma unroll
            for (int tp = 0; tp < TP; ++tp) {
                u32x4 v[8][G::NV];
                const unsigned char *vt = reinterpret_cast<const unsigned char *>(stage + tp * KW * 64 * CH + 32 * CH);
#pragma unroll
                for (int e = 0; e < 8; ++e)
#pragma unroll
                    for (int j = 0; j < G::NV; ++j) {
                        const unsigned char *p = vt + (e >> 2) * 16 * CH * 16 + vo[e & 3] + 256 * j;
                        if constexpr (CH == 8) {
                            const u32x2v z = *reinterpret_cast<const u32x2v *>(p);
                            v[e][j] = u32x4{z[0], z[1], 0, 0};
                        } else {
                            v[e][j] = *reinterpret_cast<const u32x4 *>(p);
                        }
                    }
                if (seen[tp] != ~0u) w.hide(v, seen[tp], g);
                w.values(s[tp], v);
            }
        }
        if (it.nodes && kw == KW - 1 && !idle) attend_nodes(w, a, it.r, kvh, count, node, g, rr);
        __syncthreads();   // the stages are read: their memory is free
        if constexpr (KW > 1) {
            f32x4(*s_o)[G::NT][64] = reinterpret_cast<f32x4(*)[G::NT][64]>(lds);
            float(*s_ml)[2][64] = reinterpret_cast<float(*)[2][64]>(lds + (KW / 2) * RW * G::NT * 64);
            join_waves(w, s_o, s_ml, kw, rw, KW, RW, lane);
        }
        if (kw == 0) write_rows<Out>(w, a, it, kvh, count, row0, node, g, rr);
    }
}

template <int D, int RW, bool HALVES, typename Out> hipError_t launch(int grid, const AttnArgs &a, hipStream_t s)
{
    typedef Staged<D, RW> X;
    static std::once_flag once;
    static hipError_t err;
    const auto kernel = bdgdn_tree_attn_staged_kernel<D, RW, HALVES, Out>;
    std::call_once(once, [&] {
        err = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, X::LDS);
    });
    if (err != hipSuccess) return err;
    kernel<<<grid, 64 * X::W, X::LDS, s>>>(a);
    return hipGetLastError();
}

template <int D, typename Out> hipError_t launch_rw(int grid, const AttnArgs &a, hipStream_t s)
{
    if (a.page % 16 == 0) return a.RW == 2 ? launch<D, 2, true, Out>(grid, a, s) : launch<D, 4, true, Out>(grid, a, s);
    return a.RW == 2 ? launch<D, 2, false, Out>(grid, a, s) : launch<D, 4, false, Out>(grid, a, s);
}

}  // namespace

hipError_t launch_tree_attn_staged(bool f32_out, int d, int grid, const AttnArgs &a, hipStream_t s)
{
#define BDGDN_STAGED(D) (f32_out ? launch_rw<D, float>(grid, a, s) : launch_rw<D, __bf16>(grid, a, s))
    return d == 64 ? BDGDN_STAGED(64) : d == 128 ? BDGDN_STAGED(128) : BDGDN_STAGED(256);
#undef BDGDN_STAGED
}

}  // namespace bdgdn
