// norm.hpp -- what the forward and the backward of the norms around a mixer share: a row's elements
// in the registers of its lanes, the gate, sums over a row.
//
// A row belongs to LANES lanes, each with C chunks of 8 neighbouring elements of it, so that a row is
// read once however many sums it needs.  Chunks are 16 or 32 bytes at any element's address.  WHOLE:
// d is a multiple of 8; else the last chunk is read and written an element at a time.
#pragma once

#include "anywhere.hpp"
#include "layer.hpp"

namespace bdgdn {

constexpr int kActSilu = 1;   // (of the gates: 0 takes z itself, others the sigmoid)

// The first element of chunk c of this lane.
template <int LANES> __device__ __forceinline__ int element(int c, int lane) { return (c * LANES + lane) * 8; }

// C chunks of a lane's part of a row of d elements as they lie in memory (zeros beyond its end): loads that
// nothing waits for until get().
template <bool WHOLE, int LANES, int C, typename E> struct Ahead {
    static constexpr int N = sizeof(E) / 2;   // 16-byte parts of a chunk
    u32x4 w[C * N];
    E v[WHOLE ? 1 : 8];                       // the elements of a last chunk that is not whole
    __device__ __forceinline__ void load(const E *row, int d, int lane)
    {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int e = element<LANES>(c, lane);
#pragma unroll
            for (int i = 0; i < N; ++i)
                w[c * N + i] = (WHOLE ? e : e + 7) < d ? reinterpret_cast<const typename AnyPlace<E>::type *>(row + e)[i] : u32x4{0, 0, 0, 0};
        }
        if constexpr (!WHOLE) {
            const int e = last(d, lane);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = e + i < d ? row[e + i] : to_e<E>(0.f);
        }
    }
    // The first element of this lane's chunk that is not whole, d if it has none.
    static __device__ __forceinline__ int last(int d, int lane)
    {
        const int chunk = d >> 3;
        return (d & 7) && chunk % LANES == lane ? chunk * 8 : d;
    }
    __device__ __forceinline__ void get(float (&to)[C][8], int d, int lane) const
    {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if constexpr (N == 1) to[c][i] = __uint_as_float(i & 1 ? w[c][i >> 1] & 0xffff0000u : w[c][i >> 1] << 16);
                else to[c][i] = __uint_as_float(w[c * N + (i >> 2)][i & 3]);
                if (!WHOLE && element<LANES>(c, lane) + 7 >= d) to[c][i] = element<LANES>(c, lane) < d ? to_f(v[i]) : 0.f;
            }
    }
};

// Chunk c of a lane's part of a row of d elements.
template <bool WHOLE, int LANES, typename E> __device__ __forceinline__ void load_chunk(float (&v)[8], const E *row, int c, int d, int lane)
{
    const int e = element<LANES>(c, lane);
    if ((WHOLE ? e : e + 7) < d) {
        load8(v, row + e);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = !WHOLE && e + i < d ? to_f(row[e + i]) : 0.f;
    }
}
template <bool WHOLE, int LANES, typename E>
__device__ __forceinline__ void store_chunk(E *row, const float (&v)[8], int c, int d, int lane)
{
    const int e = element<LANES>(c, lane);
    if (e + 8 <= d) {
        store8(row + e, v);
    } else if (!WHOLE) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (e + i < d) row[e + i] = to_e<E>(v[i]);
    }
}

// All chunks.
template <bool WHOLE, int LANES, int C, typename E> __device__ __forceinline__ void load_row(float (&v)[C][8], const E *row, int d, int lane)
{
#pragma unroll
    for (int c = 0; c < C; ++c) load_chunk<WHOLE, LANES>(v[c], row, c, d, lane);
}
template <bool WHOLE, int LANES, int C, typename E> __device__ __forceinline__ void store_row(E *row, const float (&v)[C][8], int d, int lane)
{
#pragma unroll
    for (int c = 0; c < C; ++c) store_chunk<WHOLE, LANES>(row, v[c], c, d, lane);
}

// 1 / (1 + exp(-z)); a large -z gives exp = inf and the result 0.
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + fexp2(-kLog2e * z)); }
// e = sigmoid(z), and 1 - e in 32 bits of its own: the difference cancels where e is near 1 (at z = 12 1 % of it
// is rounding, from 17 on all), so there it is exp(-z) e.
__device__ __forceinline__ float sigmoid(float z, float &rest)
{
    const float t = fexp2(-kLog2e * z), e = __builtin_amdgcn_rcpf(1.f + t);
    rest = z > 0.f ? t * e : 1.f - e;
    return e;
}

// Sums over the LANES lanes of a row, in every lane of it.  Rows of several waves meet in LDS: two
// buffers take turns, so that a sum needs one barrier (between a buffer's readers and its next
// writers lies the other's).  Every thread of the workgroup calls it.
template <int LANES, int THREADS, int MOST> struct RowSum {
    static constexpr int WAVES = THREADS / 64, ROW = LANES / 64;
    float *lds;   // [2][MOST][WAVES]
    int turn = 0;
    __device__ __forceinline__ explicit RowSum(float *p) : lds(p) {}
    template <int K> __device__ __forceinline__ void operator()(float (&x)[K])
    {
        static_assert(K <= MOST, "room");
#pragma unroll
        for (int o = 1; o < (LANES < 64 ? LANES : 64); o <<= 1)
#pragma unroll
            for (int k = 0; k < K; ++k) x[k] += __shfl_xor(x[k], o);
        if constexpr (LANES > 64) {
            float *buf = lds + turn * MOST * WAVES;
            turn ^= 1;
            const int wave = threadIdx.x >> 6;
            if ((threadIdx.x & 63) == 0)
#pragma unroll
                for (int k = 0; k < K; ++k) buf[k * WAVES + wave] = x[k];
            lds_barrier();
#pragma unroll
            for (int k = 0; k < K; ++k) {
                x[k] = 0.f;
#pragma unroll
                for (int w = 0; w < ROW; ++w) x[k] += buf[k * WAVES + (wave & ~(ROW - 1)) + w];
            }
        }
    }
};

// Which of the workgroup's rows is this lane's (the same for a whole wave where a row has 64 lanes).
template <int LANES> __device__ __forceinline__ unsigned row_of()
{
    const unsigned mine = threadIdx.x / LANES;
    return LANES >= 64 ? __builtin_amdgcn_readfirstlane(mine) : mine;
}

template <typename E> __device__ __forceinline__ E *row_at(const void *p, const RowStride &s, int a, int b)
{
    return static_cast<E *>(const_cast<void *>(p)) + a * s.outer + b * s.inner;
}


}  // namespace bdgdn
