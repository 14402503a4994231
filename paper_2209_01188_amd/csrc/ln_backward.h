// Derivative of a LayerNorm y = g x_hat + b, x_hat = (x - mean) / sqrt(var + eps), of one row by one workgroup:
//   dx = inv (dy g - mean(dy g) - x_hat mean(dy g x_hat)),  inv = 1 / sqrt(var + eps)
// All row sums in fp64, the variance about the mean.
#pragma once
#include "common.h"

// Columns (threadIdx.x + i NT) 8 .. + 8 of the row belong to this thread; acc holds dy and receives dx.
template <int NT, int PER>
__device__ __forceinline__ void ln_backward(float (&acc)[PER][8], const __half *__restrict__ x, const __half *__restrict__ g, int H,
                                            float eps, double (*sm)[2]) {
    float xv[PER][8];
    double s1 = 0.0, sa = 0.0;
#pragma unroll
    for (int i = 0; i < PER; i++) {
        const int k = (threadIdx.x + i * NT) * 8;
        if (k < H) {
            const v8h f = *(const v8h_any *)(x + k), gg = *(const v8h_any *)(g + k);
#pragma unroll
            for (int e = 0; e < 8; e++) {
                xv[i][e] = (float)f[e];
                acc[i][e] *= (float)gg[e];
                s1 += (double)xv[i][e];
                sa += (double)acc[i][e];
            }
        }
    }
    const auto both = [&](double &a, double &b) {
        a = wave_sum(a);
        b = wave_sum(b);
        if ((threadIdx.x & 63) == 0) {
            sm[threadIdx.x >> 6][0] = a;
            sm[threadIdx.x >> 6][1] = b;
        }
        __syncthreads();
        a = b = 0.0;
#pragma unroll
        for (int w = 0; w < NT / 64; w++) {
            a += sm[w][0];
            b += sm[w][1];
        }
        __syncthreads();
    };
    both(s1, sa);
    const double rH = 1.0 / (double)H, mean = s1 * rH, ma = sa * rH;
    double s2 = 0.0, sb = 0.0;
#pragma unroll
    for (int i = 0; i < PER; i++) {
        const int k = (threadIdx.x + i * NT) * 8;
        if (k < H) {
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const double xc = (double)xv[i][e] - mean;
                s2 = fma(xc, xc, s2);
                sb = fma((double)acc[i][e], xc, sb);
            }
        }
    }
    both(s2, sb);
    const double inv = 1.0 / sqrt(s2 * rH + (double)eps), along = inv * inv * sb * rH;
#pragma unroll
    for (int i = 0; i < PER; i++) {
        const int k = (threadIdx.x + i * NT) * 8;
        if (k < H) {
#pragma unroll
            for (int e = 0; e < 8; e++) acc[i][e] = (float)(inv * ((double)acc[i][e] - ma - ((double)xv[i][e] - mean) * along));
        }
    }
}
typedef float v4f_row __attribute__((ext_vector_type(4), aligned(4)));     // callers' rows carry no alignment promise
template <int NT, int PER>
__device__ __forceinline__ void ln_store(const float (&acc)[PER][8], float *__restrict__ row, int H) {
#pragma unroll
    for (int i = 0; i < PER; i++) {
        const int k = (threadIdx.x + i * NT) * 8;
        if (k < H) {
#pragma unroll
            for (int h = 0; h < 2; h++)
                *(v4f_row *)(row + k + 4 * h) = v4f{acc[i][4 * h], acc[i][4 * h + 1], acc[i][4 * h + 2], acc[i][4 * h + 3]};
        }
    }
}
template <int NT, int PER>
__device__ __forceinline__ void ln_store(const float (&acc)[PER][8], __half *__restrict__ row, int H) {
#pragma unroll
    for (int i = 0; i < PER; i++) {
        const int k = (threadIdx.x + i * NT) * 8;
        if (k < H) {
            v8h o;
#pragma unroll
            for (int e = 0; e < 8; e++) o[e] = (_Float16)acc[i][e];
            *(v8h_any *)(row + k) = o;
        }
    }
}
