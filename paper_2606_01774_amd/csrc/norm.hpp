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

// A lane's part of a row of d elements; `past` beyond its end.
template <bool WIDE, int LANES, int C, typename E>
__device__ __forceinline__ void load_row(float (&v)[C][8], const E *row, int d, int lane, float past = 0.f)
{
#pragma unroll
    for (int c = 0; c < C; ++c) {
        if constexpr (WIDE) {
            const int e = element<WIDE, LANES>(c, 0, lane);
            if (e < d) load8(v[c], row + e);
            else
#pragma unroll
                for (int i = 0; i < 8; ++i) v[c][i] = past;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int e = element<WIDE, LANES>(c, i, lane);
                v[c][i] = e < d ? to_f(row[e]) : past;
            }
        }
    }
}
template <bool WIDE, int LANES, int C, typename E>
__device__ __forceinline__ void store_row(E *row, const float (&v)[C][8], int d, int lane)
{
#pragma unroll
    for (int c = 0; c < C; ++c) {
        if constexpr (WIDE) {
            const int e = element<WIDE, LANES>(c, 0, lane);
            if (e < d) store8(row + e, v[c]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int e = element<WIDE, LANES>(c, i, lane);
                if (e < d) row[e] = to_e<E>(v[c][i]);
            }
        }
    }
}

// 1 / (1 + exp(-z)); a large -z gives exp = inf and the result 0.
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + fexp2(-kLog2e * z)); }

// The sum of K values over the LANES lanes of a row, in every lane of it.  Rows of several waves
// meet in lds ([K][waves of the workgroup]); every thread of the workgroup calls it.
template <int LANES, int THREADS, int K> __device__ __forceinline__ void row_sum(float (&x)[K], float *lds)
{
#pragma unroll
    for (int o = 1; o < (LANES < 64 ? LANES : 64); o <<= 1)
#pragma unroll
        for (int k = 0; k < K; ++k) x[k] += __shfl_xor(x[k], o);
    if constexpr (LANES > 64) {
        constexpr int W = LANES / 64, ALL = THREADS / 64;
        const int wave = threadIdx.x >> 6;
        __syncthreads();   // the last sum has been read
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < K; ++k) lds[k * ALL + wave] = x[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            x[k] = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) x[k] += lds[k * ALL + (wave & ~(W - 1)) + w];
        }
    }
}

template <typename E> __device__ __forceinline__ E *row_at(const void *p, const RowStride &s, int a, int b)
{
    return static_cast<E *>(const_cast<void *>(p)) + a * s.outer + b * s.inner;
}


}  // namespace bdgdn
