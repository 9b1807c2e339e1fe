// norm.hpp -- what the forward and the backward of the norms around a mixer share: a row's elements
// in the registers of its lanes, the gate, sums over a row.
//
// A row belongs to LANES lanes, each with C chunks of 8 of its elements in registers, so that a
// row is read once however many sums it needs.  WIDE: a chunk is 8 neighbouring elements (16 or
// 32 bytes); else (odd sizes, addresses or strides) elements LANES apart, one load each.
#pragma once

#include "common.hpp"
#include "layer.hpp"

namespace bdgdn {

constexpr int kActSilu = 1, kActSigmoid = 2;

// The element of place i of chunk c of this lane.
template <bool WIDE, int LANES> __device__ __forceinline__ int element(int c, int i, int lane)
{
    return WIDE ? (c * LANES + lane) * 8 + i : (c * 8 + i) * LANES + lane;
}

__device__ __forceinline__ void load8(float (&v)[8], const __bf16 *p)
{
    const u32x4 w = *reinterpret_cast<const u32x4 *>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void load8(float (&v)[8], const float *p)
{
    const f32x4 a = *reinterpret_cast<const f32x4 *>(p), b = *reinterpret_cast<const f32x4 *>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = a[i];
        v[4 + i] = b[i];
    }
}
__device__ __forceinline__ void store8(__bf16 *p, const float (&v)[8])
{
    bf16x8 w;
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = (__bf16)v[i];
    *reinterpret_cast<bf16x8 *>(p) = w;
}
__device__ __forceinline__ void store8(float *p, const float (&v)[8])
{
    *reinterpret_cast<f32x4 *>(p) = f32x4{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<f32x4 *>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
}

// Chunk c of a lane's part of a row of d elements; zeros beyond its end.
template <bool WIDE, int LANES, typename E> __device__ __forceinline__ void load_chunk(float (&v)[8], const E *row, int c, int d, int lane)
{
    if constexpr (WIDE) {
        const int e = element<WIDE, LANES>(c, 0, lane);
        if (e < d) load8(v, row + e);
        else
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = 0.f;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = element<WIDE, LANES>(c, i, lane);
            v[i] = e < d ? to_f(row[e]) : 0.f;
        }
    }
}
template <bool WIDE, int LANES, typename E>
__device__ __forceinline__ void store_chunk(E *row, const float (&v)[8], int c, int d, int lane)
{
    if constexpr (WIDE) {
        const int e = element<WIDE, LANES>(c, 0, lane);
        if (e < d) store8(row + e, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = element<WIDE, LANES>(c, i, lane);
            if (e < d) row[e] = to_e<E>(v[i]);
        }
    }
}

// C chunks of a lane's part of a row as they lie in memory: loads that nothing waits for until get().
template <bool WIDE, int LANES, int C, typename E> struct Ahead {
    static constexpr int N = sizeof(E) / 2;   // 16-byte parts of a chunk
    u32x4 w[WIDE ? C * N : 1];
    E v[WIDE ? 1 : C * 8];
    __device__ __forceinline__ void load(const E *row, int d, int lane)
    {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if constexpr (WIDE) {
                const int e = element<WIDE, LANES>(c, 0, lane);
#pragma unroll
                for (int i = 0; i < N; ++i) w[c * N + i] = e < d ? reinterpret_cast<const u32x4 *>(row + e)[i] : u32x4{0, 0, 0, 0};
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int e = element<WIDE, LANES>(c, i, lane);
                    v[c * 8 + i] = e < d ? row[e] : to_e<E>(0.f);
                }
            }
        }
    }
    __device__ __forceinline__ void get(float (&to)[C][8]) const
    {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if constexpr (!WIDE) to[c][i] = to_f(v[c * 8 + i]);
                else if constexpr (N == 1) to[c][i] = __uint_as_float(i & 1 ? w[c][i >> 1] & 0xffff0000u : w[c][i >> 1] << 16);
                else to[c][i] = __uint_as_float(w[c * N + (i >> 2)][i & 3]);
            }
    }
};

// All chunks.
template <bool WIDE, int LANES, int C, typename E> __device__ __forceinline__ void load_row(float (&v)[C][8], const E *row, int d, int lane)
{
#pragma unroll
    for (int c = 0; c < C; ++c) load_chunk<WIDE, LANES>(v[c], row, c, d, lane);
}
template <bool WIDE, int LANES, int C, typename E> __device__ __forceinline__ void store_row(E *row, const float (&v)[C][8], int d, int lane)
{
#pragma unroll
    for (int c = 0; c < C; ++c) store_chunk<WIDE, LANES>(row, v[c], c, d, lane);
}

// 1 / (1 + exp(-z)); a large -z gives exp = inf and the result 0.
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + fexp2(-kLog2e * z)); }

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
