// Layer norm over rows of `dim` values, forward and backward.
//
//   mean = sum x / dim,  rstd = 1 / sqrt(sum (x - mean)^2 / dim + eps),  z = (x - mean) rstd
//   y  = gain z + bias
//   dx = rstd (t - sum t / dim - z sum (t z) / dim),  t = dy gain
//   dgain = sum over rows of dy z,  dbias = sum over rows of dy
//
// Bound by memory: forward moves x and y once, backward x, dy and dx once.  A row is held in the
// registers of one group of threads, so the variance is taken around the mean (two sums, no
// cancellation) without reading the row twice.  In the backward pass a group keeps going over
// rows and its threads keep the column sums of dgain and dbias in fp32 registers; one row of partial sums
// per CTA goes to the workspace and a second small kernel adds those in a fixed order: no atomics, the
// same bits every time.
#pragma once

#include "train.cuh"

namespace tk {

constexpr int kNormThreads = 256;   // per CTA, unless a row needs a larger group
constexpr int kNormFinishCols = 32, kNormFinishSlices = 8;

template <typename T, int VEC>
struct alignas(sizeof(T) * VEC) Pack {
    T v[VEC];
};

struct NormArgs {
    const void* x;
    const void* dy;      // backward
    void* out;           // y or dx (dx may be null)
    const void* gain;
    const void* bias;    // forward; may be null
    float* mean;         // [rows]; forward: written unless null; backward: read
    float* rstd;
    float* partial;      // backward: [gridDim.x][2][dim] sums of dgain and dbias, or null
    int64_t rows, x_stride, dy_stride, out_stride;
    int dim;
    int param_bf16;
    float eps;
};

// VEC parameters from column c as fp32
template <int VEC>
__device__ __forceinline__ void load_params(const void* p, int c, bool is_bf16, float (&out)[VEC]) {
    if (VEC == 1) {
        out[0] = load_any(p, c, is_bf16);
    } else if (is_bf16) {
        constexpr int W = VEC < 8 ? VEC : 8;
#pragma unroll
        for (int i = 0; i < VEC; i += W) {
            Pack<bf16, W> q = *(const Pack<bf16, W>*)((const bf16*)p + c + i);
#pragma unroll
            for (int j = 0; j < W; ++j) out[i + j] = to_float(q.v[j]);
        }
    } else {
        constexpr int W = VEC < 4 ? VEC : 4;
#pragma unroll
        for (int i = 0; i < VEC; i += W) {
            Pack<float, W> q = *(const Pack<float, W>*)((const float*)p + c + i);
#pragma unroll
            for (int j = 0; j < W; ++j) out[i + j] = q.v[j];
        }
    }
}

// Sums of a and b over a group of G threads, in every thread.  red: one float2 per warp of the CTA and
// buffer; consecutive calls alternate buffers (one barrier then separates reuse of a buffer).
template <int G>
__device__ __forceinline__ float2 group_sum2(float a, float b, float2* red, int& buffer) {
    a = warp_sum(a);
    b = warp_sum(b);
    if (G == 32) return make_float2(a, b);
    const int warp = threadIdx.x >> 5, first = (threadIdx.x / G) * (G / 32);
    float2* r = red + buffer * 32;
    buffer ^= 1;
    if ((threadIdx.x & 31) == 0) r[warp] = make_float2(a, b);
    asm volatile("bar.sync %0, %1;" ::"r"(1 + (int)(threadIdx.x / G)), "n"(G) : "memory");
    float2 s = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < G / 32; ++i) {
        float2 v = r[first + i];
        s.x += v.x;
        s.y += v.y;
    }
    return s;
}

// A group of G threads per row; thread t holds vectors t, t + G, ... (NV of them, VEC values each).
template <typename T, int VEC, int NV, int G>
__global__ void __launch_bounds__(G > kNormThreads ? G : kNormThreads) norm_forward_kernel(const __grid_constant__ NormArgs A) {
    __shared__ float2 red[64];
    const int t = threadIdx.x % G, groups = blockDim.x / G;
    const float inv = 1.0f / (float)A.dim;
    int buffer = 0;
    for (int64_t row = (int64_t)blockIdx.x * groups + threadIdx.x / G; row < A.rows; row += (int64_t)gridDim.x * groups) {
        const T* x = (const T*)A.x + row * A.x_stride;
        T* y = (T*)A.out + row * A.out_stride;
        float v[NV][VEC], sum = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * G + t) * VEC;
            if (c < A.dim) {
                Pack<T, VEC> q = *(const Pack<T, VEC>*)(x + c);
#pragma unroll
                for (int i = 0; i < VEC; ++i) sum += v[j][i] = to_float(q.v[i]);
            }
        }
        const float mean = group_sum2<G>(sum, 0.0f, red, buffer).x * inv;
        float sq = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if ((j * G + t) * VEC < A.dim) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    v[j][i] -= mean;
                    sq += v[j][i] * v[j][i];
                }
            }
        const float rstd = 1.0f / sqrtf(group_sum2<G>(sq, 0.0f, red, buffer).x * inv + A.eps);
        if (t == 0 && A.mean) {
            A.mean[row] = mean;
            A.rstd[row] = rstd;
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * G + t) * VEC;
            if (c < A.dim) {
                float gain[VEC], bias[VEC];
                load_params<VEC>(A.gain, c, A.param_bf16, gain);
                if (A.bias) load_params<VEC>(A.bias, c, A.param_bf16, bias);
                Pack<T, VEC> q;
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    float z = v[j][i] * rstd;
                    q.v[i] = from_float<T>(A.bias ? z * gain[i] + bias[i] : z * gain[i]);
                }
                *(Pack<T, VEC>*)(y + c) = q;
            }
        }
    }
}

template <typename T, int VEC, int NV, int G>
__global__ void __launch_bounds__(G > kNormThreads ? G : kNormThreads) norm_backward_kernel(const __grid_constant__ NormArgs A) {
    __shared__ float2 red[64];
    extern __shared__ float sums[];   // [2][dim] when several groups share the CTA
    const int t = threadIdx.x % G, groups = blockDim.x / G, group = threadIdx.x / G;
    const float inv = 1.0f / (float)A.dim;
    int buffer = 0;
    float dgain[NV][VEC], dbias[NV][VEC];
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < VEC; ++i) dgain[j][i] = dbias[j][i] = 0.0f;
    for (int64_t row = (int64_t)blockIdx.x * groups + group; row < A.rows; row += (int64_t)gridDim.x * groups) {
        const T* x = (const T*)A.x + row * A.x_stride;
        const T* dy = (const T*)A.dy + row * A.dy_stride;
        const float mean = A.mean[row], rstd = A.rstd[row];
        float z[NV][VEC], u[NV][VEC], s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * G + t) * VEC;
            if (c < A.dim) {
                Pack<T, VEC> qx = *(const Pack<T, VEC>*)(x + c);
                Pack<T, VEC> qd = *(const Pack<T, VEC>*)(dy + c);
                float gain[VEC];
                load_params<VEC>(A.gain, c, A.param_bf16, gain);
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    float d = to_float(qd.v[i]);
                    z[j][i] = (to_float(qx.v[i]) - mean) * rstd;
                    dgain[j][i] += d * z[j][i];
                    dbias[j][i] += d;
                    u[j][i] = d * gain[i];
                    s1 += u[j][i];
                    s2 += u[j][i] * z[j][i];
                }
            }
        }
        if (A.out) {
            const float2 s = group_sum2<G>(s1, s2, red, buffer);
            const float a = s.x * inv, b = s.y * inv;
            T* dx = (T*)A.out + row * A.out_stride;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int c = (j * G + t) * VEC;
                if (c < A.dim) {
                    Pack<T, VEC> q;
#pragma unroll
                    for (int i = 0; i < VEC; ++i) q.v[i] = from_float<T>((u[j][i] - a - z[j][i] * b) * rstd);
                    *(Pack<T, VEC>*)(dx + c) = q;
                }
            }
        }
    }
    if (!A.partial) return;
    float* mine = A.partial + (int64_t)blockIdx.x * 2 * A.dim;
    for (int turn = 0; turn < groups; ++turn) {
        if (turn == group) {
            float* to = turn == groups - 1 ? mine : sums;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int c = (j * G + t) * VEC;
                if (c < A.dim) {
#pragma unroll
                    for (int i = 0; i < VEC; ++i) {
                        float a = dgain[j][i], b = dbias[j][i];
                        if (turn > 0) {
                            a += sums[c + i];
                            b += sums[A.dim + c + i];
                        }
                        to[c + i] = a;
                        to[A.dim + c + i] = b;
                    }
                }
            }
        }
        if (turn < groups - 1) __syncthreads();
    }
}

// Rows too long for the registers of a CTA: one CTA per row, which reads the row again for each sum.
template <typename T>
__global__ void __launch_bounds__(1024) norm_wide_kernel(const __grid_constant__ NormArgs A, int backward) {
    __shared__ float2 red[64];
    const float inv = 1.0f / (float)A.dim;
    int buffer = 0;
    for (int64_t row = blockIdx.x; row < A.rows; row += gridDim.x) {
        const T* x = (const T*)A.x + row * A.x_stride;
        T* out = (T*)A.out + row * A.out_stride;
        if (!backward) {
            float sum = 0.0f, sq = 0.0f;
            for (int c = threadIdx.x; c < A.dim; c += 1024) sum += to_float(x[c]);
            const float mean = group_sum2<1024>(sum, 0.0f, red, buffer).x * inv;
            for (int c = threadIdx.x; c < A.dim; c += 1024) {
                float d = to_float(x[c]) - mean;
                sq += d * d;
            }
            const float rstd = 1.0f / sqrtf(group_sum2<1024>(sq, 0.0f, red, buffer).x * inv + A.eps);
            if (threadIdx.x == 0 && A.mean) {
                A.mean[row] = mean;
                A.rstd[row] = rstd;
            }
            for (int c = threadIdx.x; c < A.dim; c += 1024) {
                float z = (to_float(x[c]) - mean) * rstd * load_any(A.gain, c, A.param_bf16);
                out[c] = from_float<T>(A.bias ? z + load_any(A.bias, c, A.param_bf16) : z);
            }
        } else {
            const T* dy = (const T*)A.dy + row * A.dy_stride;
            const float mean = A.mean[row], rstd = A.rstd[row];
            float s1 = 0.0f, s2 = 0.0f;
            for (int c = threadIdx.x; c < A.dim; c += 1024) {
                float u = to_float(dy[c]) * load_any(A.gain, c, A.param_bf16);
                s1 += u;
                s2 += u * (to_float(x[c]) - mean) * rstd;
            }
            const float2 s = group_sum2<1024>(s1, s2, red, buffer);
            const float a = s.x * inv, b = s.y * inv;
            for (int c = threadIdx.x; c < A.dim; c += 1024) {
                float u = to_float(dy[c]) * load_any(A.gain, c, A.param_bf16);
                out[c] = from_float<T>((u - a - (to_float(x[c]) - mean) * rstd * b) * rstd);
            }
        }
    }
}

// Column sums over the rows y, y + gridDim.y, ... for rows too long for registers: one thread per column.
template <typename T>
__global__ void __launch_bounds__(kNormThreads) norm_columns_kernel(const __grid_constant__ NormArgs A) {
    const int c = blockIdx.x * kNormThreads + threadIdx.x;
    if (c >= A.dim) return;
    float a = 0.0f, b = 0.0f;
    for (int64_t row = blockIdx.y; row < A.rows; row += gridDim.y) {
        float d = to_float(((const T*)A.dy)[row * A.dy_stride + c]);
        a += d * (to_float(((const T*)A.x)[row * A.x_stride + c]) - A.mean[row]) * A.rstd[row];
        b += d;
    }
    A.partial[((int64_t)blockIdx.y * 2) * A.dim + c] = a;
    A.partial[((int64_t)blockIdx.y * 2 + 1) * A.dim + c] = b;
}

// dgain and dbias from `parts` rows of partial sums, added in the order of the rows of each slice and then
// of the slices.
__global__ void __launch_bounds__(kNormFinishCols* kNormFinishSlices)
    norm_finish_kernel(const float* partial, int parts, int dim, void* dgain, void* dbias, int grad_bf16) {
    __shared__ float part[kNormFinishSlices][kNormFinishCols];
    const int lane = threadIdx.x % kNormFinishCols, slice = threadIdx.x / kNormFinishCols;
    const int64_t c = (int64_t)blockIdx.x * kNormFinishCols + lane;
    float s = 0.0f;
    if (c < 2 * (int64_t)dim)
        for (int i = slice; i < parts; i += kNormFinishSlices) s += partial[(int64_t)i * 2 * dim + c];
    part[slice][lane] = s;
    __syncthreads();
    if (slice == 0 && c < 2 * (int64_t)dim) {
        s = 0.0f;
#pragma unroll
        for (int i = 0; i < kNormFinishSlices; ++i) s += part[i][lane];
        if (c < dim) {
            if (dgain) store_any(dgain, c, s, grad_bf16);
        } else if (dbias) {
            store_any(dbias, c - dim, s, grad_bf16);
        }
    }
}

}  // namespace tk
