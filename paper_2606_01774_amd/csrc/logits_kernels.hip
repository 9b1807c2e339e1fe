// logits_kernels.hip -- penalties for repeated tokens, biases and grammar masks on the logits of a
// round's nodes, and the histories that the penalties go by (include/bdgdn.h, bdgdn_logits,
// bdgdn_history_add).
//
// A workgroup takes a tile of the vocabulary through several nodes of one request: the history's words
// and the biases of a lane's tokens stay in registers, each row of logits is read and written once.
// What a tile holds beside its history, a request's biases and the nodes' own tokens, is found
// once a tile: an LDS word for every token names its bias and says whether a node carries it.
//
// Bound by memory: 64 requests of 8 nodes over 131072 bf16 logits with history, 300 biases and a grammar
// 57 us, 310 MB at 5.4 TB/s; one node each 16 us without biases and grammar, 67 MB at 4.1 (a workgroup has one row then
// and loads nothing ahead: its waves wait for 56 % of their time); one request of 8 nodes over 32001 4.8 us.
// bdgdn_history_add: 64 x 8 tokens 2.8 us, a launch; 64 x 2000 7.1.
#include "anywhere.hpp"
#include "layer.hpp"

namespace bdgdn {

namespace {

constexpr int kThreads = 256;
constexpr int kPer = 8;                       // tokens of a lane
constexpr int kTile = kThreads * kPer;
constexpr int32_t kPrompt = 1 << 30;
constexpr uint32_t kNode = 0x80000000u;       // a node of the block carries the token

// A lane's logits of one row, and its bits of the grammar's words, as they lie in memory.
template <typename X> struct Row {
    u32x4 w[sizeof(X) / 2];
    uint32_t bits;
    __device__ __forceinline__ void load(const X *x, const uint8_t *allow, int left)
    {
        if (left <= 0) return;
        if (left >= kPer) {
#pragma unroll
            for (int i = 0; i < (int)sizeof(X) / 2; ++i) w[i] = reinterpret_cast<const typename AnyPlace<X>::type *>(x)[i];
        } else {
            X v[kPer];
#pragma unroll
            for (int i = 0; i < kPer; ++i) v[i] = i < left ? x[i] : to_e<X>(0.f);
            __builtin_memcpy(w, v, sizeof(w));
        }
        bits = allow ? *allow : 0xffu;
    }
    __device__ __forceinline__ void get(float (&l)[kPer]) const
    {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if constexpr (sizeof(X) == 2) l[i] = __uint_as_float(i & 1 ? w[0][i >> 1] & 0xffff0000u : w[0][i >> 1] << 16);
            else l[i] = __uint_as_float(w[i >> 2][i & 3]);
        }
    }
};

template <typename X, typename Y> __global__ void __launch_bounds__(kThreads) bdgdn_logits_kernel(LogitsArgs a)
{
    __shared__ uint32_t s_mark[kTile];        // entry of bias + 1, kNode
    __shared__ int32_t s_token[64], s_node[64];
    __shared__ int s_nodes, s_marks;
    const int tid = threadIdx.x, r = blockIdx.y, v0 = blockIdx.x * kTile, v = v0 + tid * kPer;
    const int n0 = blockIdx.z * a.group, nodes = a.count ? min(a.count[r], a.N) : a.N, n1 = min(n0 + a.group, nodes);
    if (n0 >= n1) return;
    const int left = min(a.V - v, kPer);      // this lane's tokens (none or fewer at the row's end)
    const float rho_given = a.repetition ? a.repetition[r] : 1.f;
    const float rho = rho_given > 0.f ? rho_given : 1.f, inv = 1.f / rho;
    const float presence = a.presence ? a.presence[r] : 0.f, frequency = a.frequency ? a.frequency[r] : 0.f;
    const bool penal = rho != 1.f || presence != 0.f || frequency != 0.f;
    const int slot = a.slot ? a.slot[r] : r;
    const bool with_history = penal && a.history && (unsigned)slot < (unsigned)a.n_slots;
    const bool with_nodes = penal && a.token;

    // (what comes from memory is on its way while the tile's marks are set)
    const X *x = static_cast<const X *>(a.x) + r * a.x_req + v;
    const uint8_t *allow = a.allow ? reinterpret_cast<const uint8_t *>(a.allow + r * a.a_req) + (v >> 3) : nullptr;
    auto grammar = [&](int n) { return allow ? allow + 4 * n * a.a_row : nullptr; };
    Row<X> next;
    next.load(x + n0 * a.x_row, grammar(n0), left);
    int32_t word[kPer] = {};
    if (with_history && left > 0) {
        const int32_t *from = a.history + slot * a.h_row + v;
        if (left >= kPer) {
            const u32x4 lo = reinterpret_cast<const u32x4_e4 *>(from)[0], hi = reinterpret_cast<const u32x4_e4 *>(from)[1];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                word[i] = (int32_t)lo[i];
                word[4 + i] = (int32_t)hi[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < kPer; ++i) word[i] = i < left ? from[i] : 0;
        }
    }
    uint32_t mark[kPer] = {};
    float bias[kPer] = {};
    if (with_nodes || a.n_bias) {
        if (tid == 0) s_nodes = s_marks = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) s_mark[i * kThreads + tid] = 0;
        lds_barrier();
        for (int j = tid; j < a.n_bias; j += kThreads) {
            const unsigned t = (unsigned)a.bias_token[(long)r * a.n_bias + j] - (unsigned)v0;
            if (t < (unsigned)kTile) {
                atomicMax(&s_mark[t], (uint32_t)j + 1);
                s_marks = 1;
            }
        }
        lds_barrier();
        if (with_nodes && tid < nodes) {
            const int t = a.token[(long)r * a.N + tid];
            if ((unsigned)t - (unsigned)v0 < (unsigned)kTile && (unsigned)t < (unsigned)a.V) {
                const int at = atomicAdd(&s_nodes, 1);
                s_token[at] = t;
                s_node[at] = tid;
                atomicOr(&s_mark[t - v0], kNode);
                s_marks = 1;
            }
        }
        lds_barrier();
        if (s_marks) {
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                mark[i] = s_mark[tid * kPer + i];
                const uint32_t j = mark[i] & ~kNode;
                if (j && i < left) bias[i] = a.bias[(long)r * a.n_bias + j - 1];
            }
        }
    }
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) any |= mark[i] & kNode;
    if (left <= 0) return;

    Y *y = static_cast<Y *>(a.y) + r * a.y_req + v;
    for (int n = n0; n < n1; ++n) {
        float l[kPer];
        next.get(l);
        const uint32_t bits = next.bits;
        if (n + 1 < n1) next.load(x + (n + 1) * a.x_row, grammar(n + 1), left);
        const uint64_t path = a.mask ? a.mask[(long)r * a.N + n] : (2ull << n) - 1;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            int c = word[i] & (kPrompt - 1);
            if (any && (mark[i] & kNode))
                for (int j = 0; j < s_nodes; ++j) c += s_token[j] == v + i && ((path >> s_node[j]) & 1);
            float t = l[i];
            if (penal) {
                const bool seen = c > 0 || (word[i] & kPrompt);
                if (seen) t *= t > 0.f ? inv : rho;
                if (c > 0) t -= fmaf(frequency, (float)c, presence);
            }
            t += bias[i];
            l[i] = (bits >> i) & 1 ? t : -INFINITY;
        }
        if (left >= kPer) store8(y + n * a.y_row, l);
        else
            for (int i = 0; i < left; ++i) (y + n * a.y_row)[i] = to_e<Y>(l[i]);
    }
}

__global__ void __launch_bounds__(kThreads) bdgdn_history_add_kernel(int R, int N, int V, int n_slots, long row, int32_t *history,
                                                                     const int32_t *slot, const int32_t *token,
                                                                     const int32_t *path, const int32_t *count, int prompt)
{
    const long all = (long)R * N;
    for (long x = (long)blockIdx.x * kThreads + threadIdx.x; x < all; x += (long)gridDim.x * kThreads) {
        const int r = (int)(x / N), j = (int)(x - (long)r * N);
        if (count && j >= count[r]) continue;
        const int s = slot ? slot[r] : r, n = path ? path[x] : j;
        if ((unsigned)s >= (unsigned)n_slots || (unsigned)n >= (unsigned)N) continue;
        const int t = token[(long)r * N + n];
        if ((unsigned)t >= (unsigned)V) continue;
        int32_t *word = history + s * row + t;
        if (prompt) atomicOr(word, kPrompt);
        else atomicAdd(word, 1);
    }
}

}  // namespace

hipError_t launch_logits(bool bf16, bool f32_out, LogitsArgs &a, hipStream_t s)
{
    const int tiles = (a.V + kTile - 1) / kTile;
    // all nodes to a workgroup, fewer where that leaves compute units idle
    a.group = a.N;
    while (a.group > 1 && (long)tiles * a.R * ((a.N + a.group - 1) / a.group) < 1024) a.group = (a.group + 1) / 2;
    const dim3 grid(tiles, a.R, (a.N + a.group - 1) / a.group);
    if (!bf16) bdgdn_logits_kernel<float, float><<<grid, kThreads, 0, s>>>(a);
    else if (f32_out) bdgdn_logits_kernel<__bf16, float><<<grid, kThreads, 0, s>>>(a);
    else bdgdn_logits_kernel<__bf16, __bf16><<<grid, kThreads, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_history_add(int R, int N, int V, int n_slots, long row, int32_t *history, const int32_t *slot,
                              const int32_t *token, const int32_t *path, const int32_t *count, int prompt, hipStream_t s)
{
    const long blocks = ((long)R * N + kThreads - 1) / kThreads;
    bdgdn_history_add_kernel<<<(unsigned)(blocks < 4096 ? blocks : 4096), kThreads, 0, s>>>(R, N, V, n_slots, row, history, slot,
                                                                                           token, path, count, prompt);
    return hipGetLastError();
}

}  // namespace bdgdn
