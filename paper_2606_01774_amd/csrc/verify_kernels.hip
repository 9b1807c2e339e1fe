// verify_kernels.hip -- verification of drafted tokens against the target's logits from given
// random numbers.  A first kernel reads every row of logits that a walk may need once and
// leaves its maximum and its sum of exponentials by parts of the vocabulary; a second one, a
// workgroup per request, walks the tree and draws the next token by the exponential race.
#include "common.hpp"
#include "round.hpp"

namespace bdgdn {

namespace {

constexpr int kStatThreads = 256;
constexpr int kWalkThreads = 1024;

// A part's statistics: maximum, sum of exp2((x - max) k), index of the maximum.
struct Stat {
    float max, sum;
    int arg;
};

__device__ __forceinline__ float load_logit(const __bf16 *p) { return (float)*p; }
__device__ __forceinline__ float load_logit(const float *p) { return *p; }

__device__ __forceinline__ Stat join(Stat a, Stat b, float k)
{
    Stat r;
    const bool second = b.max > a.max || (b.max == a.max && b.arg < a.arg);
    r.max = second ? b.max : a.max;
    r.arg = second ? b.arg : a.arg;
    const float m = r.max == -INFINITY ? 0.f : r.max;
    r.sum = a.sum * fexp2((a.max - m) * k) + b.sum * fexp2((b.max - m) * k);
    return r;
}

// log2(e) / T, or log2(e) for a greedy request (its sum only says whether the row has a law).
__device__ __forceinline__ float temper(const VerifyArgs &a, int r, bool &greedy)
{
    const float T = a.temperature ? a.temperature[r] : 1.f;
    greedy = !(T > 0.f);
    return greedy ? kLog2e : kLog2e / T;
}

template <typename E> __global__ void __launch_bounds__(kStatThreads) bdgdn_verify_stats_kernel(VerifyArgs a)
{
    __shared__ Stat lds[kStatThreads / 64];
    const int row = blockIdx.x, rows = a.R * a.N;
    const bool is_draft = row >= rows;
    const int rn = is_draft ? row - rows : row, r = rn / a.N, n = rn - r * a.N;
    const int count = a.count ? min(a.count[r], a.N) : a.N;
    if (n >= count) return;
    bool greedy;
    const float k = temper(a, r, greedy);
    if (is_draft) {   // only the rows of nodes with children, and of requests that look at them
        if (greedy) return;
        bool child = false;
        if (a.parent) {
            for (int c = n + 1; c < count; ++c) child |= a.parent[r * a.N + c] == n;
        } else {
            child = n + 1 < count;
        }
        if (!child) return;
    }
    const E *x = is_draft ? static_cast<const E *>(a.draft) + r * a.d_req + n * a.d_row
                          : static_cast<const E *>(a.target) + r * a.t_req + n * a.t_row;
    const int per = (a.V + a.splits - 1) / a.splits;
    const int v0 = blockIdx.y * per, v1 = min(v0 + per, a.V);
    Stat st = {-INFINITY, 0.f, 0x7fffffff};
    for (int v = v0 + threadIdx.x; v < v1; v += kStatThreads) {
        const float y = load_logit(x + v);
        if (y > st.max) {
            st.sum = st.sum * fexp2((st.max - y) * k) + 1.f;
            st.max = y;
            st.arg = v;
        } else {   // also a NaN, which stays in the sum, and -inf beside -inf, which adds nothing
            st.sum += y == -INFINITY ? 0.f : fexp2((y - st.max) * k);
        }
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int o = 32; o; o >>= 1) {
        Stat b = {__shfl_xor(st.max, o), __shfl_xor(st.sum, o), __shfl_xor(st.arg, o)};
        st = join(st, b, k);
    }
    if (lane == 0) lds[wave] = st;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kStatThreads / 64; ++w) st = join(st, lds[w], k);
        float *p = a.stats + ((long)row * a.splits + blockIdx.y) * 4;
        p[0] = st.max;
        p[1] = st.sum;
        p[2] = __int_as_float(st.arg);
    }
}

// A row's law: p(x) = exp2((x - max) k) inv, or all on `arg` where k is 0; inv 0 for no law.
struct Law {
    float max, inv, k;
    int arg;
    bool ok;
    __device__ __forceinline__ float at(float x, int v) const
    {
        return k == 0.f ? (v == arg ? inv : 0.f) : fexp2((x - max) * k) * inv;
    }
};

__device__ Law law_of(const VerifyArgs &a, bool is_draft, int r, int n, float k, bool greedy)
{
    const float *p = a.stats + ((long)((is_draft ? a.R * a.N : 0) + r * a.N + n) * a.splits) * 4;
    Stat st = {p[0], p[1], __float_as_int(p[2])};
    for (int s = 1; s < a.splits; ++s) st = join(st, Stat{p[4 * s], p[4 * s + 1], __float_as_int(p[4 * s + 2])}, k);
    Law l;
    l.ok = st.sum > 0.f && st.sum < INFINITY && fabsf(st.max) < INFINITY;
    l.max = st.max;
    l.arg = st.arg;
    l.k = greedy ? 0.f : k;
    l.inv = !l.ok ? 0.f : greedy ? 1.f : 1.f / st.sum;
    return l;
}

template <typename E> struct Walk {
    const VerifyArgs &a;
    const E *t, *d;          // rows of the current node (d null: certain proposals)
    Law p, q;
    float c, W;
    int gone[64], n_gone;    // refused tokens (certain proposals)

    __device__ float residual(int v) const
    {
        const float pv = p.ok ? p.at(load_logit(t + v), v) : 0.f;
        if (d) return q.ok ? fmaxf(pv - c * q.at(load_logit(d + v), v), 0.f) : pv;
        for (int i = 0; i < n_gone; ++i)
            if (gone[i] == v) return 0.f;
        return pv;
    }
};

template <typename E> __global__ void __launch_bounds__(kWalkThreads) bdgdn_verify_walk_kernel(VerifyArgs a)
{
    __shared__ float s_sum[kWalkThreads / 64];
    __shared__ float s_best[2][kWalkThreads / 64];
    __shared__ int s_at[2][kWalkThreads / 64];
    const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int count = a.count ? min(a.count[r], a.N) : a.N;
    int32_t *path = a.path + r * a.N;
    if (count < 1) {
        for (int n = tid; n < a.N; n += kWalkThreads) path[n] = -1;
        if (tid == 0) {
            a.n_accept[r] = 0;
            if (a.n_path) a.n_path[r] = 0;
            a.next[r] = -1;
        }
        return;
    }
    bool greedy;
    const float k = temper(a, r, greedy);
    const bool certain = greedy || !a.draft;
    const E *target = static_cast<const E *>(a.target) + r * a.t_req;
    const E *draft = certain ? nullptr : static_cast<const E *>(a.draft) + r * a.d_req;
    Walk<E> w = {a, target, nullptr, {}, {}, 0.f, 1.f, {}, 0};
    int cur = 0, steps = 0;
    w.p = law_of(a, false, r, 0, k, greedy);
    bool fresh = true;   // no child of cur has been tried
    for (int n = 1; n < count; ++n) {
        if ((a.parent ? a.parent[r * a.N + n] : n - 1) != cur) continue;
        if (fresh && !certain) {
            w.d = draft + cur * a.d_row;
            w.q = law_of(a, true, r, cur, k, false);
        }
        fresh = false;
        const int tok = a.token[r * a.N + n];
        const bool in = (unsigned)tok < (unsigned)a.V && (certain || w.q.ok);
        const float left = in ? w.residual(tok) : 0.f;
        const float odds = !in ? 0.f : certain ? 1.f : w.q.at(load_logit(w.d + tok), tok);
        if (in && w.p.ok && a.u[r * a.N + n] * w.W * odds < left) {
            cur = n;
            ++steps;
            if (tid == 0) path[steps] = n;
            w.t = target + cur * a.t_row;
            w.p = law_of(a, false, r, cur, k, greedy);
            w.d = nullptr;
            w.c = 0.f;
            w.W = 1.f;
            w.n_gone = 0;
            fresh = true;
            continue;
        }
        if (!in) continue;
        if (certain) {
            w.gone[w.n_gone++] = tok;
        } else {
            w.c += w.W;
        }
        float sum = 0.f;
        for (int v = tid; v < a.V; v += kWalkThreads) sum += w.residual(v);
        for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
        if (lane == 0) s_sum[wave] = sum;
        __syncthreads();
        sum = 0.f;
        for (int i = 0; i < kWalkThreads / 64; ++i) sum += s_sum[i];
        __syncthreads();
        w.W = sum;
    }
    // the race, for the residual and (where that is zero everywhere) for p itself
    const float *noise = a.noise + r * a.noise_stride;
    float best[2] = {0.f, 0.f};
    int at[2] = {-1, -1};
    if (w.p.ok) {
        for (int v = tid; v < a.V; v += kWalkThreads) {
            const float e = noise[v], x = w.residual(v) / e, y = w.p.at(load_logit(w.t + v), v) / e;
            if (x > best[0]) { best[0] = x; at[0] = v; }
            if (y > best[1]) { best[1] = y; at[1] = v; }
        }
    }
    for (int i = 0; i < 2; ++i) {
        for (int o = 32; o; o >>= 1) {
            const float x = __shfl_xor(best[i], o);
            const int y = __shfl_xor(at[i], o);
            if (x > best[i] || (x == best[i] && (unsigned)y < (unsigned)at[i])) { best[i] = x; at[i] = y; }
        }
        if (lane == 0) { s_best[i][wave] = best[i]; s_at[i][wave] = at[i]; }
    }
    for (int n = tid; n < a.N; n += kWalkThreads)
        if (n > steps) path[n] = -1;
    __syncthreads();
    if (tid == 0) {
        for (int i = 0; i < 2; ++i)
            for (int j = 1; j < kWalkThreads / 64; ++j)
                if (s_best[i][j] > best[i] || (s_best[i][j] == best[i] && (unsigned)s_at[i][j] < (unsigned)at[i])) {
                    best[i] = s_best[i][j];
                    at[i] = s_at[i][j];
                }
        path[0] = 0;
        a.n_accept[r] = steps;
        if (a.n_path) a.n_path[r] = steps + 1;
        a.next[r] = at[0] >= 0 ? at[0] : at[1];
    }
}

}  // namespace

// Parts of the vocabulary: enough workgroups for the chip, of 4096 logits at least.
int verify_splits(int R, int N, int V)
{
    const long rows = 2L * R * N;
    long s = (2048 + rows - 1) / rows;
    const long most = (V + 4095) / 4096;
    return (int)(s < 1 ? 1 : s > most ? most : s);
}

hipError_t launch_verify(bool bf16, const VerifyArgs &a, hipStream_t s)
{
    const dim3 grid((a.draft ? 2 : 1) * a.R * a.N, a.splits);
    if (bf16) {
        bdgdn_verify_stats_kernel<__bf16><<<grid, kStatThreads, 0, s>>>(a);
        bdgdn_verify_walk_kernel<__bf16><<<a.R, kWalkThreads, 0, s>>>(a);
    } else {
        bdgdn_verify_stats_kernel<float><<<grid, kStatThreads, 0, s>>>(a);
        bdgdn_verify_walk_kernel<float><<<a.R, kWalkThreads, 0, s>>>(a);
    }
    return hipGetLastError();
}

}  // namespace bdgdn
