// Derivative of a LayerNorm y = g x_hat + b, x_hat = (x - mean) / sqrt(var + eps), of one row by one workgroup:
//   dx = inv (dy g - mean(dy g) - x_hat mean(dy g x_hat)),  inv = 1 / sqrt(var + eps)
// (Its barriers order LDS only.)
// All row sums in fp64, the variance about the mean.
#pragma once
#include "common.h"

// Columns (threadIdx.x + i NT) 8 .. + 8 of the row belong to this thread; acc holds dy and receives dx.  The row and the gain are
// asked for beforehand (zeros beyond H), so that they arrive while dy is summed up.
template <int PER>
struct LnRow {
    v8h x[PER], g[PER];
};
template <int NT, int PER>
__device__ __forceinline__ void ln_load(LnRow<PER> &r, const __half *__restrict__ x, const __half *__restrict__ g, int H) {
#pragma unroll
    for (int i = 0; i < PER; i++) {
        const int k = (threadIdx.x + i * NT) * 8;
        r.x[i] = r.g[i] = v8h{0, 0, 0, 0, 0, 0, 0, 0};
        if (k < H) {
            r.x[i] = *(const v8h_any *)(x + k);
            r.g[i] = *(const v8h_any *)(g + k);
        }
    }
}
template <int NT, int PER>
__device__ __forceinline__ void ln_backward(float (&acc)[PER][8], const LnRow<PER> &row, int H, float eps, double (*sm)[2]) {
    double s1 = 0.0, sa = 0.0;
#pragma unroll
    for (int i = 0; i < PER; i++) {
#pragma unroll
        for (int e = 0; e < 8; e++) {
            acc[i][e] *= (float)row.g[i][e];
            s1 += (double)(float)row.x[i][e];
            sa += (double)acc[i][e];
        }
    }
    const auto both = [&](double &a, double &b) {
        a = wave_sum(a);
        b = wave_sum(b);
        if ((threadIdx.x & 63) == 0) {
            sm[threadIdx.x >> 6][0] = a;
            sm[threadIdx.x >> 6][1] = b;
        }
        lds_barrier();
        const int lane = threadIdx.x & 63;                          // (all waves' sums in one lane would be 4 registers each)
        a = wave_sum(lane < NT / 64 ? sm[lane][0] : 0.0);
        b = wave_sum(lane < NT / 64 ? sm[lane][1] : 0.0);
        lds_barrier();
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
                const double xc = (double)(float)row.x[i][e] - mean;
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
            for (int e = 0; e < 8; e++) acc[i][e] = (float)(inv * ((double)acc[i][e] - ma - ((double)(float)row.x[i][e] - mean) * along));
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
// acc += rows 0 .. n - 1 in order, row(r) the address of row r; AHEAD of them on their way at once
template <int NT, int PER, typename T, int AHEAD = sizeof(T) == 2 ? 8 : 4, typename F>
__device__ __forceinline__ void add_rows(float (&acc)[PER][8], int n, int H, F row) {
    typedef T v8 __attribute__((ext_vector_type(8), aligned(2)));
    for (int r0 = 0; r0 < n; r0 += AHEAD) {
        const T *from[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; u++) from[u] = row(min(r0 + u, n - 1));
#pragma unroll
        for (int i = 0; i < PER; i++) {
            const int k = (threadIdx.x + i * NT) * 8;
            if (k >= H) continue;
            v8 f[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; u++) f[u] = *(const v8 *)(from[u] + k);
#pragma unroll
            for (int u = 0; u < AHEAD; u++)
                if (r0 + u < n) {
#pragma unroll
                    for (int e = 0; e < 8; e++) acc[i][e] += (float)f[u][e];
                }
        }
    }
}
