// verify_kernels.hip -- verification of drafted tokens against the target's logits from given
// random numbers, in four launches, or two for vocabularies of up to 32768.
//
//   stats  (row, part of the vocabulary): reads every row of logits that a walk may need once
//          and leaves the part's maximum and sum of exponentials, or (greedy requests) the
//          index of its maximum.  This is where the bytes are: 64 requests of 8 nodes over
//          131072 bf16 logits, 16 of them greedy (their draft rows are not read), 39 us, 222 MB at
//          5.7 TB/s; bound by memory.
//   walk   (request): the rows' laws and every child's odds at once, then the walk itself in
//          LDS.  7.5 us for the same requests, 9 for trees of 24 over 100003 fp32 logits with certain
//          drafts: latency.  Only a refusal with a sibling left reads a row again, for the
//          residual's mass, and that is one workgroup's work: with sampled drafts each such refusal takes 17 us
//          over 131072 bf16 logits (5 over 32001), one after the other.  64 requests with 2, 4, 7
//          drafts side by side: calls of 82, 114, 161 us where one takes 69.
//   race   (request, part): argmax of law(t) / noise(t) over a part of one row; 13.8 us for the
//          same 64 (50 MB read, 3.6 TB/s: half of it latency).  Short rows are raced over by the walk's
//          workgroup.
//   pick   (request): the best of the parts; 4 us, of which most is a launch's own.
// Statistics, laws, residuals and scores are fp32, from logits of either type; the only rounding
// to fewer bits is the caller's.
// For long rows one workgroup to a request takes three times as long (36 us for
// a row of 131072 with its draft and noise, 64 requests), and joining the parts by the last of
// a request's workgroups twice (each has to write back its caches first).
#include "common.hpp"
#include "round.hpp"

namespace bdgdn {

namespace {

constexpr int kStatThreads = 256;
constexpr int kWalkThreads = 1024;
constexpr int kRaceThreads = 256;
constexpr int kMaxNodes = 64;

// Rows of logits begin anywhere: vectors of 16 bytes that are aligned to an element only.
typedef u32x4 u32x4_e2 __attribute__((aligned(2)));
typedef u32x4 u32x4_e4 __attribute__((aligned(4)));

template <typename E> struct Vec;
template <> struct Vec<__bf16> {
    static constexpr int n = 8;
    static __device__ __forceinline__ void load(float (&x)[8], const __bf16 *p)
    {
        const u32x4 w = *reinterpret_cast<const u32x4_e2 *>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
};
template <> struct Vec<float> {
    static constexpr int n = 4;
    static __device__ __forceinline__ void load(float (&x)[4], const float *p)
    {
        const u32x4 w = *reinterpret_cast<const u32x4_e4 *>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(w[i]);
    }
};

// A part's statistics: maximum, sum of exp2((x - max) k); greedy requests: maximum, NaN if
// there is one among the logits and 1 if not, index of the maximum.
struct Stat {
    float max, sum;
    int arg;
};

__device__ __forceinline__ Stat join(Stat a, Stat b, float k, bool greedy)
{
    Stat r;
    const bool second = b.max > a.max || (b.max == a.max && b.arg < a.arg);
    r.max = second ? b.max : a.max;
    r.arg = second ? b.arg : a.arg;
    const float m = r.max == -INFINITY ? 0.f : r.max;
    r.sum = greedy ? a.sum * b.sum : a.sum * fexp2((a.max - m) * k) + b.sum * fexp2((b.max - m) * k);
    return r;
}

// log2(e) / T, or 1 for a greedy request; kept where no product with a difference of logits is
// 0 x inf.
__device__ __forceinline__ float temper(const VerifyArgs &a, int r, bool &greedy)
{
    const float T = a.temperature ? a.temperature[r] : 1.f;
    greedy = !(T > 0.f);
    return greedy ? 1.f : fminf(fmaxf(kLog2e / T, 1.2e-38f), 1e38f);
}

// Nodes of request r.
__device__ __forceinline__ int nodes_of(const VerifyArgs &a, int r)
{
    return a.count ? min(a.count[r], a.N) : a.N;
}

// Running statistics of the elements that a thread reads.
template <bool GREEDY> struct Running {
    Stat s;
    __device__ __forceinline__ Running() : s{-INFINITY, GREEDY ? 1.f : 0.f, 0x7fffffff} {}
    template <int N> __device__ __forceinline__ void add(const float (&x)[N], int v, float k)
    {
        if (GREEDY) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if (x[i] > s.max) {
                    s.max = x[i];
                    s.arg = v + i;
                }
                if (x[i] != x[i]) s.sum = x[i];
            }
        } else {
            float m = s.max;
#pragma unroll
            for (int i = 0; i < N; ++i) m = fmaxf(m, x[i]);
            const float base = m == -INFINITY ? 0.f : m;
            s.sum *= fexp2((s.max - base) * k);
            s.max = m;
#pragma unroll
            for (int i = 0; i < N; ++i) s.sum += fexp2((x[i] - base) * k);
        }
    }
};

template <typename E, bool GREEDY>
__device__ __forceinline__ Stat part_stats(const E *x, int v0, int v1, float k)
{
    constexpr int N = Vec<E>::n, U = 4;   // four loads in flight
    Running<GREEDY> run;
    int v = v0 + threadIdx.x * N;
    for (; v + (U - 1) * kStatThreads * N + N <= v1; v += U * kStatThreads * N) {
        float y[U][N];
#pragma unroll
        for (int u = 0; u < U; ++u) Vec<E>::load(y[u], x + v + u * kStatThreads * N);
        if (GREEDY) {
#pragma unroll
            for (int u = 0; u < U; ++u) run.add(y[u], v + u * kStatThreads * N, k);
        } else {
            float z[U * N];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < N; ++i) z[u * N + i] = y[u][i];
            run.add(z, v, k);
        }
    }
    for (; v < v1; v += kStatThreads * N) {
        float y[N];
        if (v + N <= v1) {
            Vec<E>::load(y, x + v);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) y[i] = v + i < v1 ? to_f(x[v + i]) : -INFINITY;
        }
        run.add(y, v, k);
    }
    return run.s;
}

template <typename E> __global__ void __launch_bounds__(kStatThreads) bdgdn_verify_stats_kernel(VerifyArgs a)
{
    __shared__ Stat lds[kStatThreads / 64];
    const int row = blockIdx.x / a.splits, split = blockIdx.x - row * a.splits, rows = a.R * a.N;
    const bool is_draft = row >= rows;
    const int rn = is_draft ? row - rows : row, r = rn / a.N, n = rn - r * a.N;
    const int count = nodes_of(a, r);
    if (n >= count) return;
    bool greedy;
    const float k = temper(a, r, greedy);
    if (is_draft) {   // only the rows of nodes with children, and of requests that look at them
        if (greedy) return;
        bool child = false;
        if (a.parent) {
            const int c = threadIdx.x & 63;
            child = __any(c > n && c < count && a.parent[(long)r * a.N + min(c, a.N - 1)] == n);
        } else {
            child = n + 1 < count;
        }
        if (!child) return;
    }
    const E *x = is_draft ? static_cast<const E *>(a.draft) + r * a.d_req + n * a.d_row
                          : static_cast<const E *>(a.target) + r * a.t_req + n * a.t_row;
    const int v0 = split * a.part, v1 = min(v0 + a.part, a.V);
    Stat st = greedy ? part_stats<E, true>(x, v0, v1, k) : part_stats<E, false>(x, v0, v1, k);
#pragma unroll
    for (int o = 32; o; o >>= 1) {
        const Stat b = {__shfl_xor(st.max, o), __shfl_xor(st.sum, o), __shfl_xor(st.arg, o)};
        st = join(st, b, k, greedy);
    }
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = st;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kStatThreads / 64; ++w) st = join(st, lds[w], k, greedy);
        float *p = a.stats + ((long)row * a.splits + split) * 4;
        *reinterpret_cast<f32x4 *>(p) = f32x4{st.max, st.sum, __int_as_float(st.arg), 0.f};
    }
}

// A row's law: p(x) = exp2((x - max) k) inv, or all on `arg` where k is 0; inv 0 for no law.
struct Law {
    float max, inv, k;
    int arg;
    __device__ __forceinline__ bool ok() const { return inv > 0.f; }
    __device__ __forceinline__ float of(float x) const { return fexp2((x - max) * k) * inv; }
    __device__ __forceinline__ float at(float x, int v) const { return k == 0.f ? (v == arg ? inv : 0.f) : of(x); }
};

// Joined by one wave, a part to a lane.
__device__ __forceinline__ Law law_of(const VerifyArgs &a, long row, float k, bool greedy, int lane)
{
    Stat st = {-INFINITY, greedy ? 1.f : 0.f, 0x7fffffff};
    if (lane < a.splits) {
        const f32x4 p = *reinterpret_cast<const f32x4 *>(a.stats + (row * a.splits + lane) * 4);
        st = Stat{p[0], p[1], __float_as_int(p[2])};
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) {
        const Stat b = {__shfl_xor(st.max, o), __shfl_xor(st.sum, o), __shfl_xor(st.arg, o)};
        st = join(st, b, k, greedy);
    }
    const bool ok = st.sum > 0.f && st.sum < INFINITY && fabsf(st.max) < INFINITY;
    return Law{st.max, !ok ? 0.f : greedy ? 1.f : 1.f / st.sum, greedy ? 0.f : k, st.arg};
}

// The law that is left of a row (of a request that is not greedy) from its logits.
template <typename E> struct Residual {
    const E *t, *d;
    Law p, q;
    float c;
    const int *gone;   // refused tokens that are out of the law
    int n_gone;
    __device__ __forceinline__ bool out(int v) const
    {
        bool found = false;
        for (int i = 0; i < n_gone; ++i) found |= gone[i] == v;
        return found;
    }
    // x: the target's logits, then what is left of the law but for what `out` says; y: the
    // draft's logits where c > 0
    // (without a fused multiply-add, so that equal laws leave exactly nothing)
    template <int N> __device__ __forceinline__ void of(float (&x)[N], const float (&y)[N]) const
    {
#pragma clang fp contract(off)
        if (c > 0.f) {
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = fmaxf(p.of(x[i]) - c * q.of(y[i]), 0.f);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = p.of(x[i]);
        }
    }
    __device__ __forceinline__ float one(int v) const
    {
        float x[1] = {to_f(t[v])}, y[1] = {0.f};
        if (c > 0.f) y[0] = to_f(d[v]);
        of(x, y);
        return x[0];
    }
};

struct Best {
    float score;
    int at;
    __device__ __forceinline__ void take(float x, int v)
    {
        if (x > score || (x == score && (unsigned)v < (unsigned)at)) {
            score = x;
            at = v;
        }
    }
};

// What the walk leaves for the race.
struct Walked {
    Law p, q;
    float c;           // law = (p - c q)+; c 0: q is not looked at
    int node, n_gone;  // the node whose row is raced for, or -1; refused tokens out of the law
    int next;          // of a request without a race
    int gone[kMaxNodes];
};

template <int THREADS> __device__ __forceinline__ Best best_of_block(Best b, Best *lds)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) b.take(__shfl_xor(b.score, o), __shfl_xor(b.at, o));
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = b;
    __syncthreads();
    b = lds[0];
    for (int w = 1; w < THREADS / 64; ++w) b.take(lds[w].score, lds[w].at);
    __syncthreads();
    return b;
}

// argmax over [v0, v1) of law / noise, -1 where nothing is above zero.  Every thread of the
// workgroup gets it.  The quotient is formed only where a product says that it may pass the
// best one of the wave (x >= best e, less what the rounding of either can hide).
template <int THREADS, typename E> __device__ __forceinline__ Best race(const Residual<E> &res, const float *noise, int v0, int v1, Best *lds)
{
    constexpr int N = Vec<E>::n;
    Best b = {0.f, -1};
    float bar = 0.f;
    const auto consider = [&](const float x, const float e, int at) {
        const float y = x / e;
        if (y > b.score && !res.out(at)) b = Best{y, at};
    };
    const int whole = v0 + (v1 - v0) / N * N;
#pragma unroll 2
    for (int v = v0; v < whole; v += THREADS * N) {
        const int at = v + threadIdx.x * N;
        const bool in = at < whole;
        float x[N], y[N], e[N];
        bool pass = false;
        if (in) {
            Vec<E>::load(x, res.t + at);
            if (res.c > 0.f) Vec<E>::load(y, res.d + at);
#pragma unroll
            for (int i = 0; i < N; i += 4) Vec<float>::load(reinterpret_cast<float(&)[4]>(e[i]), noise + at + i);
            res.of(x, y);
#pragma unroll
            for (int i = 0; i < N; ++i) pass |= x[i] >= bar * e[i];
        }
        if (!__any(pass)) continue;
        if (pass) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (x[i] >= bar * e[i]) consider(x[i], e[i], at + i);
        }
        float top = b.score;
#pragma unroll
        for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
        bar = top * 0.999999f;
    }
    if (whole + (int)threadIdx.x < v1) {
        const int at = whole + threadIdx.x;
        consider(res.one(at), noise[at], at);
    }
    return best_of_block<THREADS>(b, lds);
}

// RACE: the walk's workgroup also draws the next token.
template <typename E, bool RACE> __global__ void __launch_bounds__(kWalkThreads) bdgdn_verify_walk_kernel(VerifyArgs a)
{
    __shared__ Law s_law[2][kMaxNodes];
    __shared__ float s_p[kMaxNodes], s_q[kMaxNodes], s_u[kMaxNodes];
    __shared__ int s_parent[kMaxNodes], s_token[kMaxNodes];
    __shared__ float s_sum[kWalkThreads / 64];
    __shared__ int s_gone[kMaxNodes];
    const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int count = nodes_of(a, r);
    Walked *out = static_cast<Walked *>(a.walked) + r;
    int32_t *path = a.path + (long)r * a.N;
    if (count < 1) {
        for (int n = tid; n < a.N; n += kWalkThreads) path[n] = -1;
        if (tid == 0) {
            a.n_accept[r] = 0;
            if (a.n_path) a.n_path[r] = 0;
            if (RACE) a.next[r] = -1;
            else out->node = out->next = -1;
        }
        return;
    }
    bool greedy;
    const float k = temper(a, r, greedy);
    const bool certain = greedy || !a.draft;
    const E *target = static_cast<const E *>(a.target) + r * a.t_req;
    const E *draft = certain ? nullptr : static_cast<const E *>(a.draft) + r * a.d_req;
    if (tid < count) {
        const int p = tid == 0 ? -1 : a.parent ? a.parent[(long)r * a.N + tid] : tid - 1;
        const int t = tid == 0 ? -1 : a.token[(long)r * a.N + tid];
        s_parent[tid] = p < tid ? p : -1;
        s_token[tid] = (unsigned)t < (unsigned)a.V ? t : -1;
        s_u[tid] = tid == 0 ? 0.f : a.u[(long)r * a.N + tid];
    }
    __syncthreads();
    // every node's law and, where children were drawn from it, its draft's
    for (int i = wave; i < 2 * count; i += kWalkThreads / 64) {
        const int n = i >> 1;
        if (i & 1) {
            if (certain || !__any(lane > n && lane < count && s_parent[min(lane, count - 1)] == n)) continue;
        }
        const Law l = law_of(a, (long)(i & 1 ? a.R * a.N : 0) + (long)r * a.N + n, k, greedy, lane);
        if (lane == 0) s_law[i & 1][n] = l;
    }
    __syncthreads();
    if (tid < count && s_parent[tid] >= 0 && s_token[tid] >= 0) {
        const int p = s_parent[tid], t = s_token[tid];
        s_p[tid] = s_law[0][p].ok() ? s_law[0][p].at(to_f(target[p * a.t_row + t]), t) : 0.f;
        s_q[tid] = certain ? 1.f : s_law[1][p].at(to_f(draft[p * a.d_row + t]), t);
    }
    __syncthreads();

    int cur = 0, steps = 0, n_gone = 0;
    float c = 0.f, W = 1.f;
    const int my_parent = lane < count ? s_parent[lane] : -1;
    // (a child's number is higher than its parent's, so the children come in index order)
    unsigned long long children = __ballot(my_parent == cur);
    while (children) {
        const int n = __ffsll(children) - 1;
        children &= children - 1;
        const int tok = s_token[n];
        if (tok < 0 || !s_law[0][cur].ok() || (!certain && !s_law[1][cur].ok())) continue;
        bool out_already = false;
        for (int i = 0; i < n_gone; ++i) out_already |= s_gone[i] == tok;
        const float left = certain ? (out_already ? 0.f : s_p[n]) : fmaxf(s_p[n] - c * s_q[n], 0.f);
        if (s_u[n] * W * s_q[n] < left) {
            cur = n;
            ++steps;
            if (tid == 0) path[steps] = n;
            c = 0.f;
            W = 1.f;
            n_gone = 0;
            children = __ballot(my_parent == cur);
            continue;
        }
        if (certain) {
            if (out_already) continue;
            __syncthreads();
            if (tid == 0) s_gone[n_gone] = tok;
            ++n_gone;
            __syncthreads();
        } else {
            c += W;
        }
        if (!children) continue;
        // the residual's mass.  What is left of certain proposals follows by subtraction as
        // long as that keeps all but four bits.
        if (certain && W - left > 0.0625f) {
            W -= left;
            continue;
        }
        const Residual<E> res = {target + cur * a.t_row, certain ? nullptr : draft + cur * a.d_row, s_law[0][cur],
                                 certain ? Law{} : s_law[1][cur], c, s_gone, n_gone};
        constexpr int N = Vec<E>::n;
        float sum = 0.f;
        const int whole = a.V / N * N;
#pragma unroll 2
        for (int v = tid * N; v < whole; v += kWalkThreads * N) {
            float x[N], y[N];
            Vec<E>::load(x, res.t + v);
            if (c > 0.f) Vec<E>::load(y, res.d + v);
            res.of(x, y);
#pragma unroll
            for (int i = 0; i < N; ++i) sum += certain && res.out(v + i) ? 0.f : x[i];
        }
        if (whole + tid < a.V && !(certain && res.out(whole + tid))) sum += res.one(whole + tid);
        for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
        if (lane == 0) s_sum[wave] = sum;
        __syncthreads();
        W = 0.f;
        for (int i = 0; i < kWalkThreads / 64; ++i) W += s_sum[i];
        __syncthreads();
    }
    for (int n = tid; n < a.N; n += kWalkThreads)
        if (n > steps) path[n] = -1;
    if (tid == 0) {
        path[0] = 0;
        a.n_accept[r] = steps;
        if (a.n_path) a.n_path[r] = steps + 1;
    }
    // (an integer comparison of the law's bits: from one of floats hipcc 7.2 has made a select
    // on a condition that it had not set)
    const bool lawful = __builtin_amdgcn_readfirstlane(__float_as_int(s_law[0][cur].inv)) > 0;
    if (RACE) {
        if (!lawful || greedy) {   // (a greedy law is all on one token, and that was not refused)
            if (tid == 0) a.next[r] = lawful ? s_law[0][cur].arg : -1;
            return;
        }
        __shared__ Best s_best[kWalkThreads / 64];
        Residual<E> res = {target + cur * a.t_row, c > 0.f ? draft + cur * a.d_row : nullptr, s_law[0][cur],
                           c > 0.f ? s_law[1][cur] : Law{}, c, s_gone, n_gone};
        const float *noise = a.noise + r * a.noise_stride;
        Best b = race<kWalkThreads>(res, noise, 0, a.V, s_best);
        if (b.at < 0) {   // nothing is left of the law: p itself
            res.c = 0.f;
            res.n_gone = 0;
            b = race<kWalkThreads>(res, noise, 0, a.V, s_best);
        }
        if (tid == 0) a.next[r] = b.at;
        return;
    }
    if (tid < n_gone) out->gone[tid] = s_gone[tid];
    if (tid == 0) {
        out->p = s_law[0][cur];
        if (c > 0.f) out->q = s_law[1][cur];
        out->c = c;
        out->node = lawful && !greedy ? cur : -1;
        out->n_gone = n_gone;
        // a greedy law is all on one token, and that was not refused
        out->next = lawful ? s_law[0][cur].arg : -1;
    }
}

template <typename E> __device__ __forceinline__ Residual<E> left_of(const VerifyArgs &a, const Walked &w, int r)
{
    return Residual<E>{static_cast<const E *>(a.target) + r * a.t_req + w.node * a.t_row,
                       w.c > 0.f ? static_cast<const E *>(a.draft) + r * a.d_req + w.node * a.d_row : nullptr, w.p, w.q, w.c,
                       w.gone, w.n_gone};
}

template <typename E> __global__ void __launch_bounds__(kRaceThreads) bdgdn_verify_race_kernel(VerifyArgs a)
{
    __shared__ Best lds[kRaceThreads / 64];
    const int r = blockIdx.y;
    const Walked &w = static_cast<const Walked *>(a.walked)[r];
    if (w.node < 0) return;
    const int v0 = blockIdx.x * a.race_part, v1 = min(v0 + a.race_part, a.V);
    const Best b = race<kRaceThreads>(left_of<E>(a, w, r), a.noise + r * a.noise_stride, v0, v1, lds);
    if (threadIdx.x == 0) static_cast<Best *>(a.best)[(long)r * a.race_splits + blockIdx.x] = b;
}

template <typename E> __global__ void __launch_bounds__(kRaceThreads) bdgdn_verify_pick_kernel(VerifyArgs a)
{
    __shared__ Best lds[kRaceThreads / 64];
    const int r = blockIdx.x;
    const Walked &w = static_cast<const Walked *>(a.walked)[r];
    if (w.node < 0) {
        if (threadIdx.x == 0) a.next[r] = w.next;
        return;
    }
    Best b = {0.f, -1};
    for (int i = threadIdx.x; i < a.race_splits; i += kRaceThreads) {
        const Best x = static_cast<const Best *>(a.best)[(long)r * a.race_splits + i];
        b.take(x.score, x.at);
    }
    b = best_of_block<kRaceThreads>(b, lds);
    if (b.at < 0) {   // nothing is left of the law: p itself
        Residual<E> res = left_of<E>(a, w, r);
        res.c = 0.f;
        res.n_gone = 0;
        b = race<kRaceThreads>(res, a.noise + r * a.noise_stride, 0, a.V, lds);
    }
    if (threadIdx.x == 0) a.next[r] = b.at;
}

template <typename E> void launch(const VerifyArgs &a, hipStream_t s)
{
    bdgdn_verify_stats_kernel<E><<<(a.draft ? 2 : 1) * a.R * a.N * a.splits, kStatThreads, 0, s>>>(a);
    if (a.race_splits == 0) {
        bdgdn_verify_walk_kernel<E, true><<<a.R, kWalkThreads, 0, s>>>(a);
        return;
    }
    bdgdn_verify_walk_kernel<E, false><<<a.R, kWalkThreads, 0, s>>>(a);
    bdgdn_verify_race_kernel<E><<<dim3(a.race_splits, a.R), kRaceThreads, 0, s>>>(a);
    bdgdn_verify_pick_kernel<E><<<a.R, kRaceThreads, 0, s>>>(a);
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace

// Parts of a row: enough workgroups for the chip (2048 hold all its threads); of a row's statistics
// at most 64, one to a lane of the wave that joins them.
VerifyPlan verify_plan(int R, int N, int V)
{
    // As many parts as give 2048 workgroups, of 4096 logits or 1024 raced ones at least: less than an
    // unrolled step of a workgroup's loads (8192 bf16 logits) and, raced in bf16, half a step, since few
    // rows are all latency.  12 rows of 100003 fp32 logits: the race 6.3 us in parts of 1024, 8.6 in parts of 4096.
    // Replayed calls for one row of 40003: fp32 16.7 us, 17.4 with raced parts of 2048, bf16 15.4 and
    // 15.7; with statistics in parts of 8192 bf16 16.5 (over 131072 14.8 for 15.2).
    const auto cut = [V](long rows, long limit, int least, int &parts, int &part) {
        const long most = (V + least - 1) / least;
        long n = (2048 + rows - 1) / rows;
        n = n > most ? most : n;
        n = n > limit ? limit : n;
        part = (int)(((V + n - 1) / n + 7) / 8 * 8);
        parts = (V + part - 1) / part;
    };
    VerifyPlan p;
    cut(2L * R * N, 64, 4096, p.splits, p.part);
    cut(R, 2048, 1024, p.race_splits, p.race_part);
    // Up to 32768 logits the walk's workgroup races over all of them: two launches fewer (one
    // request over 1000: 22 -> 17 us a call, over 32001 23 -> 19; 64 requests over 32001 33.5 ->
    // 31, of fp32 40 -> 38; at 65536, 16 requests, it would be 30 instead of 25).
    if (V <= 32768) p.race_splits = 0;
    p.walked_at = align256(2 * (size_t)R * N * p.splits * 16);
    p.best_at = p.walked_at + align256((size_t)R * sizeof(Walked));
    p.bytes = p.best_at + align256((size_t)R * p.race_splits * sizeof(Best));
    return p;
}

hipError_t launch_verify(bool bf16, VerifyArgs &a, const VerifyPlan &p, void *workspace, hipStream_t s)
{
    char *ws = static_cast<char *>(workspace);
    a.stats = reinterpret_cast<float *>(ws);
    a.walked = ws + p.walked_at;
    a.best = ws + p.best_at;
    a.splits = p.splits; a.part = p.part;
    a.race_splits = p.race_splits; a.race_part = p.race_part;
    if (bf16) launch<__bf16>(a, s);
    else launch<float>(a, s);
    return hipGetLastError();
}

}  // namespace bdgdn
