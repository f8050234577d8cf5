// Operators that work row by row or element by element: the RMS norm and its gradients, 8-bit checkpoints, the gradient at what an
// activation is taken of, sums over rows.  All are bound by memory.
#ifndef RINR_NN_ROWS_HIP_H
#define RINR_NN_ROWS_HIP_H

#include "rinr_nn_common.hip.h"

namespace rinr_nn {

// ---- sums over the threads of one row ------------------------------------------------------------------------------------------------

// TPR threads share a row: 64 (a wavefront) or a whole workgroup of more.  `scratch`: 2 floats for each wavefront.
template <int TPR> __device__ __forceinline__ void row_sums(float &a, float &b, float *scratch) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        a += __shfl_xor(a, d);
        b += __shfl_xor(b, d);
    }
    if (TPR > 64) {
        const int w = threadIdx.x >> 6;
        __syncthreads();                                                         // what the row before left has been read
        if ((threadIdx.x & 63) == 0) {
            scratch[2 * w] = a;
            scratch[2 * w + 1] = b;
        }
        __syncthreads();
        a = b = 0.0f;
#pragma unroll
        for (int i = 0; i < TPR / 64; ++i) {
            a += scratch[2 * i];
            b += scratch[2 * i + 1];
        }
    }
}

// ---- RMS norm ------------------------------------------------------------------------------------------------------------------------

struct NormArgs {
    int64_t rows;
    int cols;
    float eps;
    const void *x, *residual;
    const float *gain;
    void *y, *h;
    uint8_t *y_scales;
    int64_t ld_x, ld_residual, ld_y, ld_h;
    bool past;                                                                   // results go past the L2s
};

// y = gain h / sqrt(mean h^2 + eps), h = x + residual.  A row stays in registers from the one time it is read; TPR threads share it and
// each holds NV groups of 8 neighbouring columns: a wavefront up to 1024 columns, so that the sum needs no barrier.  Bound by memory: 32768 x 1024 in bf16
// with residual 40 us (6.7 TB/s, part of it from the cache; 131072 rows 5.9), with 8-bit output 36.
template <class T, int TPR, int NV, bool PACKED> __global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void norm_kernel(const NormArgs a) {
    constexpr int THREADS = TPR < 256 ? 256 : TPR, SLOTS = THREADS / TPR;
    __shared__ float scratch[2 * THREADS / 64];
    const int t = threadIdx.x % TPR;
    const int64_t row = block_of() * SLOTS + threadIdx.x / TPR;
    if (row >= a.rows) return;                                                   // of a whole wavefront, or a whole workgroup
    float h[NV][8], ss = 0.0f, none = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int col = (v * TPR + t) * 8, have = a.cols - col;
        load_n<T, 8>((const T *)a.x + row * a.ld_x + col, have, h[v]);
        if (a.residual) {
            float r[8];
            load_n<T, 8>((const T *)a.residual + row * a.ld_residual + col, have, r);
#pragma unroll
            for (int i = 0; i < 8; ++i) h[v][i] += r[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) ss += h[v][i] * h[v][i];
    }
    row_sums<TPR>(ss, none, scratch);
    const float s = 1.0f / sqrtf(ss / (float)a.cols + a.eps);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int col = (v * TPR + t) * 8, have = a.cols - col;
        if (a.h) store_n<T, 8>((T *)a.h + row * a.ld_h + col, have, h[v], a.past);
        float g[8], y[8];
        load_n<float, 8>(a.gain + col, have, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = h[v][i] * s * g[i];
        if (PACKED) store_packed((int8_t *)a.y, a.y_scales, row, a.ld_y, col, a.cols, y, a.past);
        else store_n<T, 8>((T *)a.y + row * a.ld_y + col, have, y, a.past);
    }
}

struct NormGradArgs {
    int64_t rows;
    int cols;
    float eps;
    const void *dy, *h, *dres;
    const float *gain;
    void *dh;
    float *part;                                                                 // [gridDim.x][cols], or NULL where no gradient of the gain is asked for
    int64_t ld_dy, ld_h, ld_dres, ld_dh;
    bool past;
};

// dh = s (g - u mean(g u)) + dres with u = h s, g = dy gain.  A workgroup takes every gridDim.x-th group of rows and keeps its columns' sums of
// dy u in registers until the end.  Bound by memory: 32768 x 1024 in bf16 with the residual's gradient 44 us (6.1 TB/s), and 4.7 for the sums of 1024 workgroups.
template <class T, int TPR, int NV> __global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void norm_grad_kernel(const NormGradArgs a) {
    constexpr int THREADS = TPR < 256 ? 256 : TPR, SLOTS = THREADS / TPR;
    __shared__ float scratch[2 * THREADS / 64];
    __shared__ float shares[SLOTS > 1 ? (SLOTS - 1) * TPR * NV * 8 : 1];
    const int t = threadIdx.x % TPR, slot = threadIdx.x / TPR;
    float dgain[NV][8] = {};
    for (int64_t row = (int64_t)blockIdx.x * SLOTS + slot; row < a.rows; row += (int64_t)gridDim.x * SLOTS) {
        float h[NV][8], dy[NV][8], ss = 0.0f, gh = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int col = (v * TPR + t) * 8, have = a.cols - col;
            float g[8];
            load_n<T, 8>((const T *)a.h + row * a.ld_h + col, have, h[v]);
            load_n<T, 8>((const T *)a.dy + row * a.ld_dy + col, have, dy[v]);
            load_n<float, 8>(a.gain + col, have, g);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                ss += h[v][i] * h[v][i];
                gh += dy[v][i] * g[i] * h[v][i];
            }
        }
        row_sums<TPR>(ss, gh, scratch);
        const float s = 1.0f / sqrtf(ss / (float)a.cols + a.eps);
        const float along = gh / (float)a.cols * s * s;                          // mean(g u) s
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int col = (v * TPR + t) * 8, have = a.cols - col;
            float g[8], d[8];
            load_n<float, 8>(a.gain + col, have, g);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                dgain[v][i] += dy[v][i] * (h[v][i] * s);
                d[i] = s * (dy[v][i] * g[i] - h[v][i] * along);
            }
            if (a.dres) {
                float r[8];
                load_n<T, 8>((const T *)a.dres + row * a.ld_dres + col, have, r);
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] += r[i];
            }
            store_n<T, 8>((T *)a.dh + row * a.ld_dh + col, have, d, a.past);
        }
    }
    if (!a.part) return;
    if (SLOTS > 1 && slot > 0) {
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) shares[(((slot - 1) * NV + v) * 8 + i) * TPR + t] = dgain[v][i];
    }
    if (SLOTS > 1) __syncthreads();
    if (slot == 0) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int col = (v * TPR + t) * 8;
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int o = 1; o < SLOTS; ++o) dgain[v][i] += shares[(((o - 1) * NV + v) * 8 + i) * TPR + t];
            store_n<float, 8>(a.part + (int64_t)blockIdx.x * a.cols + col, a.cols - col, dgain[v]);
        }
    }
}

// out[c] = sum over p of part[p][c], in the order of p within each of 32 threads and then theirs: 32 columns a workgroup.  8 loads of a thread are under
// way together: with one after the other, 1024 parts of 1024 columns took 20 us.
__global__ __launch_bounds__(1024) void sum_parts_kernel(const float *part, int64_t n_parts, int64_t cols, float *out) {
    __shared__ float shares[32][33];
    const int c = threadIdx.x & 31, k = threadIdx.x >> 5;
    const int64_t col = (int64_t)blockIdx.x * 32 + c;
    float s = 0.0f;
    if (col < cols)
        for (int64_t p = k; p < n_parts; p += 256) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = p + 32 * i < n_parts ? part[(p + 32 * i) * cols + col] : 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) s += v[i];
        }
    shares[k][c] = s;
    __syncthreads();
    if (k == 0 && col < cols) {
#pragma unroll
        for (int i = 1; i < 32; ++i) s += shares[i][c];
        out[col] = s;
    }
}

// ---- 8-bit checkpoints ----------------------------------------------------------------------------------------------------------------

// Four lanes take a block of 32 columns, 8 each; groups of 8 columns are numbered row by row over whole blocks.  Bound by memory: 134 M values of bf16 71 us
// (5.7 TB/s), back 58 (7.0), back through GELU 90 (its 19 vector instructions a value).
template <class T> __global__ __launch_bounds__(256) void pack_kernel(int64_t rows, int cols, const T *x, int64_t ld_x, int8_t *codes, int64_t ld, uint8_t *scales, bool past) {
    const int64_t per_row = (cols + kBlock8 - 1) / kBlock8 * 4;
    const int64_t at = block_of() * 256 + threadIdx.x;
    const int64_t row = at / per_row;
    const int col = (int)(at - row * per_row) * 8;
    float v[8] = {};
    if (row < rows) load_n<T, 8>(x + row * ld_x + col, cols - col, v);
    if (row < rows) store_packed(codes, scales, row, ld, col, cols, v, past);          // a block's four lanes have the same row
}

// An activation's values as T; with LOW what T leaves of them, as T, `rows` rows further down (a product of both blocks takes them to twice T's bits)
template <class T, bool LOW> __device__ __forceinline__ void store_act(T *x, int64_t row, int64_t rows, int64_t ld_x, int col, int64_t have, const float (&v)[8], bool past) {
    store_n<T, 8>(x + row * ld_x + col, have, v, past);
    if (LOW) {
        float low[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float left = v[i] - (float)from_float<T>(v[i]);
            low[i] = __builtin_fabsf(left) < __builtin_inff() ? left : 0.0f;     // of an infinity or a NaN nothing is left
        }
        store_n<T, 8>(x + (rows + row) * ld_x + col, have, low, past);
    }
}

template <class T, bool LOW> __global__ __launch_bounds__(256) void unpack_kernel(int64_t rows, int cols, const int8_t *codes, int64_t ld, const uint8_t *scales, const Act act, T *x,
                                                                       int64_t ld_x, bool past) {
    const int64_t per_row = (cols + 7) / 8;
    const int64_t at = block_of() * 256 + threadIdx.x;
    const int64_t row = at / per_row;
    if (row >= rows) return;
    const int col = (int)(at - row * per_row) * 8;
    Kept<T> kept;
    float v[8];
    kept.load(codes, scales, ld, true, row, col, cols - col);
    kept.get(true, v);
    act_all<T>(v, act);
    store_act<T, LOW>(x, row, rows, ld_x, col, cols - col, v, past);
}

template <class T, bool LOW> __global__ __launch_bounds__(256) void act_kernel(int64_t rows, int cols, const T *z, int64_t ld_z, const Act act, T *x, int64_t ld_x, bool past) {
    const int64_t per_row = (cols + 7) / 8;
    const int64_t at = block_of() * 256 + threadIdx.x;
    const int64_t row = at / per_row;
    if (row >= rows) return;
    const int col = (int)(at - row * per_row) * 8;
    float v[8];
    load_n<T, 8>(z + row * ld_z + col, cols - col, v);
    act_all<T>(v, act);
    store_act<T, LOW>(x, row, rows, ld_x, col, cols - col, v, past);
}

// Zeros: `bytes` (a multiple of 2) at blockIdx.x * stride
__global__ __launch_bounds__(256) void clear_kernel(char *p, int64_t stride, int64_t bytes) {
    uint16_t *row = (uint16_t *)(p + blockIdx.x * stride);
    for (int64_t i = threadIdx.x; i < bytes / 2; i += 256) row[i] = 0;
}

// ---- the gradient at what an activation was taken of ------------------------------------------------------------------------------------

struct SlopeArgs {
    int64_t rows, cols, rows_each;                                               // rows of one workgroup
    const void *dy, *z;
    const uint8_t *z_scales;
    void *dz;                                                                    // NULL: sums only
    float *part;                                                                 // [gridDim.y][cols], or NULL
    int64_t ld_dy, ld_z, ld_dz, cols_dz;                                         // dz has zeros from `cols` to cols_dz
    bool packed, past, twice;                                                    // twice: dz once more, `rows` rows further down
    Act act;
};

// dz = dy act'(z), and the columns' sums over this workgroup's rows: 256 columns, 8 rows at a time.  Bound by memory: sums of 32768 x 1024 in bf16 15 us (4.5 TB/s).
template <class T> __global__ __launch_bounds__(256) void slope_kernel(const SlopeArgs a) {
    __shared__ float shares[7][256];
    const int t = threadIdx.x & 31, k = threadIdx.x >> 5;
    const int64_t col = (int64_t)blockIdx.x * 256 + t * 8, have = a.cols - col;
    const int64_t from = (int64_t)blockIdx.y * a.rows_each, to = from + a.rows_each < a.rows ? from + a.rows_each : a.rows;
    float sum[8] = {};
    if (col < a.cols_dz) {
        for (int64_t row = from + k; row < to; row += 8) {
            float d[8];
            load_n<T, 8>((const T *)a.dy + row * a.ld_dy + col, have, d);
            if (a.act.kind != RINR_ACT_NONE) {
                if (have > 0) {
                    Kept<T> kept;
                    float z[8];
                    kept.load(a.z, a.z_scales, a.ld_z, a.packed, row, col, have);
                    kept.get(a.packed, z);
                    slope_all<T>(d, z, a.act);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] = i < have ? d[i] : 0.0f;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += d[i];
            if (a.dz) store_n<T, 8>((T *)a.dz + row * a.ld_dz + col, a.cols_dz - col, d, a.past);
            if (a.twice) store_n<T, 8>((T *)a.dz + (a.rows + row) * a.ld_dz + col, a.cols_dz - col, d, a.past);
        }
    }
    if (!a.part) return;
    if (k > 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) shares[k - 1][i * 32 + t] = sum[i];
    }
    __syncthreads();
    if (k == 0 && have > 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int o = 0; o < 7; ++o) sum[i] += shares[o][i * 32 + t];
        store_n<float, 8>(a.part + (int64_t)blockIdx.y * a.cols + col, have, sum);
    }
}

}  // namespace rinr_nn
#endif
