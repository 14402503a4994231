// Derivative of a LayerNorm y = g x_hat + b, x_hat = (x - mean) / sqrt(var + eps), of one row by one workgroup:
//   dx = inv (dy g - mean(dy g) - x_hat mean(dy g x_hat)),  inv = 1 / sqrt(var + eps)
// The four row sums in fp64 and in one go, with x about the row's first value: a row of equal values has variance 0 exactly, and
// what cancels in sum (x - x0)^2 - H (mean - x0)^2 cancels in fp64.
#pragma once
#include "common.h"

// Columns (threadIdx.x + i NT) 8 .. + 8 of the row belong to this thread; acc holds dy and receives dx.  The row and the gain are
// asked for beforehand (zeros beyond H), so that they arrive while dy is summed up.
template <int PER>
struct LnRow {
    v8h x[PER], g[PER];
    float x0;
};
template <int NT, int PER>
__device__ __forceinline__ void ln_load(LnRow<PER> &r, const __half *__restrict__ x, const __half *__restrict__ g, int H) {
    r.x0 = __half2float(x[0]);
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
// sm: NT / 64 of them.  One barrier, which orders LDS only.
template <int NT, int PER>
__device__ __forceinline__ void ln_backward(float (&acc)[PER][8], const LnRow<PER> &row, int H, float eps, double (*sm)[4]) {
    double s1 = 0.0, s2 = 0.0, sa = 0.0, sb = 0.0;
#pragma unroll
    for (int i = 0; i < PER; i++) {
        if ((int)(threadIdx.x + i * NT) * 8 < H) {
#pragma unroll
            for (int e = 0; e < 8; e++) {
                acc[i][e] *= (float)row.g[i][e];
                const double xc = (double)(float)row.x[i][e] - (double)row.x0;
                s1 += xc;
                s2 = fma(xc, xc, s2);
                sa += (double)acc[i][e];
                sb = fma((double)acc[i][e], xc, sb);
            }
        }
    }
    s1 = wave_sum(s1);
    s2 = wave_sum(s2);
    sa = wave_sum(sa);
    sb = wave_sum(sb);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (lane == 0) {
        sm[wave][0] = s1;
        sm[wave][1] = s2;
        sm[wave][2] = sa;
        sm[wave][3] = sb;
    }
    lds_barrier();
    const bool in = lane < NT / 64;                                             // (all waves' sums in one lane would be 8 registers each)
    s1 = wave_sum(in ? sm[lane][0] : 0.0);
    s2 = wave_sum(in ? sm[lane][1] : 0.0);
    sa = wave_sum(in ? sm[lane][2] : 0.0);
    sb = wave_sum(in ? sm[lane][3] : 0.0);
    const double rH = 1.0 / (double)H, mc = s1 * rH, ma = sa * rH;              // mean - x0, mean of dy g
    const double inv = 1.0 / sqrt(fmax(fma(-mc, mc, s2 * rH), 0.0) + (double)eps), along = inv * inv * (sb * rH - mc * ma), mean = (double)row.x0 + mc;
#pragma unroll
    for (int i = 0; i < PER; i++)
#pragma unroll
        for (int e = 0; e < 8; e++) acc[i][e] = (float)(inv * ((double)acc[i][e] - ma - ((double)(float)row.x[i][e] - mean) * along));
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

// acc += columns k0 + 8 NT i .. + 8 (below H) of rows r0 .. r0 + N - 1 in order, row(r) the address of row r, all N on their way at once
template <int NT, int PER, typename T, int N, typename F>
__device__ __forceinline__ void add_some_rows(float (&acc)[PER][8], int r0, int k0, int H, F row) {
    typedef T v8 __attribute__((ext_vector_type(8), aligned(sizeof(T))));
    const T *from[N];
#pragma unroll
    for (int u = 0; u < N; u++) from[u] = row(r0 + u);
#pragma unroll
    for (int i = 0; i < PER; i++) {
        const int k = k0 + i * NT * 8;
        if (k >= H) continue;
        v8 f[N];
#pragma unroll
        for (int u = 0; u < N; u++) f[u] = *(const v8 *)(from[u] + k);
#pragma unroll
        for (int u = 0; u < N; u++)
#pragma unroll
            for (int e = 0; e < 8; e++) acc[i][e] += (float)f[u][e];
    }
}
// rows 0 .. n - 1, AHEAD (a power of two) at a time
template <int NT, int PER, typename T, int AHEAD, typename F>
__device__ __forceinline__ void add_rows(float (&acc)[PER][8], int n, int k0, int H, F row) {
    int r = 0;
    for (; r + AHEAD <= n; r += AHEAD) add_some_rows<NT, PER, T, AHEAD>(acc, r, k0, H, row);
    if constexpr (AHEAD > 1) {
        if (r < n) add_rows<NT, PER, T, AHEAD / 2>(acc, n - r, k0, H, [&](int q) { return row(r + q); });
    }
}
