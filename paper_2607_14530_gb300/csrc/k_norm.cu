// RMS norm of the sum of a token's N streams (N = 1: the norm of a hidden vector):
//   s[c] = sum_i X[t][i][c],  r = 1 / sqrt(mean_c s[c]^2 + eps),  y[c] = w[c] s[c] r
// and its backward, with n = s r:
//   ds[c] = r (w[c] dy[c] - n[c] mean_c(w dy n)),  dX[t][i] = ds for every i,  dw[c] = sum_t dy[c] n[c]
// Both are bound by memory: the state is read once and kept in registers between the sum of squares and
// the store.  The backward reads s in fp32 as the forward left it (N = 1: X itself, which is s): 4 bytes a
// channel where the state has 2 N.  In bf16 it would put 2^-9 into every term of dw, which is fp32.
#include "xhc_internal.cuh"

namespace xhc {

namespace {

constexpr int NORM_NT = 256;   // most threads of a block (one token at a time)

// The sums of a block's threads of v (every thread gets it): warps by shuffles, then warp by warp in order.
// sh: 2 x 32 floats, used in turn, so that one barrier is enough.
__device__ __forceinline__ float block_sum(float v, float* sh, int turn) {
    v = warp_sum(v);
    if (blockDim.x <= 32) return v;
    float* s = sh + 32 * (turn & 1);
    const int warp = threadIdx.x >> 5, nw = blockDim.x >> 5;
    if ((threadIdx.x & 31) == 0) s[warp] = v;
    __syncthreads();
    float t = 0.f;
    for (int q = 0; q < nw; ++q) t += s[q];
    return t;
}

// s of one chunk of 8 channels: the N streams added in order, in fp32
__device__ __forceinline__ void stream_chunk(const uint16_t* x, int N, int C, float* s) {
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = 0.f;
    int i = 0;
    for (; i + 8 <= N; i += 8) {
        uint4 v[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = ld_stream(x + (int64_t)(i + q) * C);
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            float f[8];
            unpack8(v[q], f);
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e] += f[e];
        }
    }
    for (; i < N; ++i) {
        float f[8];
        unpack8(ld_stream(x + (int64_t)i * C), f);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] += f[e];
    }
}

// CH: chunks of 8 channels a thread holds at most
template <int CH>
__global__ void __launch_bounds__(NORM_NT) k_norm_fwd(int T, int N, int C, float eps, const uint16_t* X, const float* w,
                                                      uint16_t* y, float* sum, float* rstd) {
    pdl_entry();
    __shared__ float sh[64];
    const int nch = C / 8;
    int turn = 0;
    for (int64_t t = blockIdx.x; t < T; t += gridDim.x, ++turn) {
        float s[CH][8], q2 = 0.f;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int c = (threadIdx.x + j * blockDim.x) * 8;
            if (c >= C) continue;
            stream_chunk(X + t * N * C + c, N, C, s[j]);
#pragma unroll
            for (int e = 0; e < 8; ++e) q2 = fmaf(s[j][e], s[j][e], q2);
        }
        const float r = 1.0f / sqrtf(block_sum(q2, sh, turn) / (float)C + eps);
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int q = threadIdx.x + j * blockDim.x;
            if (q >= nch) continue;
            const float4 w0 = *reinterpret_cast<const float4*>(w + 8 * q), w1 = *reinterpret_cast<const float4*>(w + 8 * q + 4);
            const float wv[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
            float o[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = s[j][e] * r * wv[e];
            *reinterpret_cast<uint4*>(y + t * C + 8 * q) = pack8(o);
            if (sum) {
                *reinterpret_cast<float4*>(sum + t * C + 8 * q) = make_float4(s[j][0], s[j][1], s[j][2], s[j][3]);
                *reinterpret_cast<float4*>(sum + t * C + 8 * q + 4) = make_float4(s[j][4], s[j][5], s[j][6], s[j][7]);
            }
        }
        if (rstd && threadIdx.x == 0) rstd[t] = r;
    }
}

// A block walks tokens blockIdx.x, + gridDim.x, ... and leaves its part of dw in part[blockIdx.x][C].
template <int CH>
__global__ void __launch_bounds__(NORM_NT) k_norm_bwd(int T, int N, int C, const uint16_t* X, const float* sum,
                                                      const float* rstd, const float* w, const uint16_t* dy,
                                                      uint16_t* dX, float* part) {
    pdl_entry();
    __shared__ float sh[64];
    const int nch = C / 8;
    float dw[CH][8];
#pragma unroll
    for (int j = 0; j < CH; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[j][e] = 0.f;
    int turn = 0;
    for (int64_t t = blockIdx.x; t < T; t += gridDim.x, ++turn) {
        float n[CH][8], d[CH][8], dot = 0.f;
        const float r = rstd[t];
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int q = threadIdx.x + j * blockDim.x;
            if (q >= nch) continue;
            unpack8(ld_stream(dy + t * C + 8 * q), d[j]);
            if (sum) {
                const float4 a = *reinterpret_cast<const float4*>(sum + t * C + 8 * q);
                const float4 b = *reinterpret_cast<const float4*>(sum + t * C + 8 * q + 4);
                n[j][0] = a.x; n[j][1] = a.y; n[j][2] = a.z; n[j][3] = a.w;
                n[j][4] = b.x; n[j][5] = b.y; n[j][6] = b.z; n[j][7] = b.w;
            } else {
                unpack8(ld_stream(X + t * C + 8 * q), n[j]);
            }
            const float4 w0 = *reinterpret_cast<const float4*>(w + 8 * q), w1 = *reinterpret_cast<const float4*>(w + 8 * q + 4);
            const float wv[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                n[j][e] *= r;
                dw[j][e] = fmaf(d[j][e], n[j][e], dw[j][e]);
                d[j][e] *= wv[e];
                dot = fmaf(d[j][e], n[j][e], dot);
            }
        }
        const float m = block_sum(dot, sh, turn) / (float)C;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int q = threadIdx.x + j * blockDim.x;
            if (q >= nch) continue;
            float o[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = r * (d[j][e] - n[j][e] * m);
            const uint4 v = pack8(o);
            uint16_t* to = dX + t * N * C + 8 * q;
            for (int i = 0; i < N; ++i) *reinterpret_cast<uint4*>(to + (int64_t)i * C) = v;
        }
    }
#pragma unroll
    for (int j = 0; j < CH; ++j) {
        const int q = threadIdx.x + j * blockDim.x;
        if (q >= nch) continue;
        float* p = part + (int64_t)blockIdx.x * C + 8 * q;
        *reinterpret_cast<float4*>(p) = make_float4(dw[j][0], dw[j][1], dw[j][2], dw[j][3]);
        *reinterpret_cast<float4*>(p + 4) = make_float4(dw[j][4], dw[j][5], dw[j][6], dw[j][7]);
    }
}

// dw[c] (+)= sum over the blocks' parts, in order: 32 channels a block, 8 threads a channel over
// interleaved parts
__global__ void __launch_bounds__(256) k_norm_dw(int P, int C, const float* part, float* dw, int accumulate) {
    pdl_entry();
    __shared__ float sh[8][33];
    const int x = threadIdx.x & 31, ty = threadIdx.x >> 5, c = blockIdx.x * 32 + x;
    float s = 0.f;
    if (c < C)
        for (int p = ty; p < P; p += 8) s += part[(int64_t)p * C + c];
    sh[ty][x] = s;
    __syncthreads();
    if (ty == 0 && c < C) {
        float t = 0.f;
#pragma unroll
        for (int q = 0; q < 8; ++q) t += sh[q][x];
        dw[c] = accumulate ? dw[c] + t : t;
    }
}

// Threads of a token's block: two chunks of 8 channels each until 256 threads, then more chunks
int norm_threads(int C) {
    const int nch = C / 8;
    int nt = 32;
    while (nt < NORM_NT && nt * 2 < nch) nt *= 2;
    return nt;
}

}  // namespace

// Blocks of the backward (and parts of dw): what the GPU holds at once, but 8 tokens a block at least
// where that leaves a block for every SM, so that the parts (4 bytes a channel each) stay a small share
// of the traffic.
int norm_bwd_blocks(int64_t T, int C) {
    const int sms = device_sms(), nt = norm_threads(C);
    const int64_t most = (int64_t)sms * (nt >= 256 ? 4 : nt >= 128 ? 8 : 16);
    const int64_t few = T / 8 > sms ? T / 8 : sms;
    int64_t b = most < few ? most : few;
    if (b > T) b = T;
    return (int)b;
}

#define NORM_CH(K, ...)                                                          \
    do {                                                                         \
        const int ch_ = (C / 8 + nt - 1) / nt;                                   \
        if (ch_ <= 1) XHC_LAUNCH(st, grid, nt, 0, (K<1>), __VA_ARGS__);          \
        else if (ch_ <= 2) XHC_LAUNCH(st, grid, nt, 0, (K<2>), __VA_ARGS__);     \
        else if (ch_ <= 4) XHC_LAUNCH(st, grid, nt, 0, (K<4>), __VA_ARGS__);     \
        else XHC_LAUNCH(st, grid, nt, 0, (K<8>), __VA_ARGS__);                   \
    } while (0)

cudaError_t launch_norm_fwd(int T, int N, int C, float eps, const uint16_t* X, const float* w, uint16_t* y,
                            float* sum, float* rstd, cudaStream_t st) {
    const int nt = norm_threads(C);
    const int64_t most = (int64_t)device_sms() * 64;
    const int grid = (int)(T < most ? T : most);
    NORM_CH(k_norm_fwd, T, N, C, eps, X, w, y, sum, rstd);
    return cudaGetLastError();
}

cudaError_t launch_norm_bwd(int T, int N, int C, const uint16_t* X, const float* sum, const float* rstd, const float* w,
                            const uint16_t* dy, uint16_t* dX, float* part, cudaStream_t st) {
    const int nt = norm_threads(C);
    const int grid = norm_bwd_blocks(T, C);
    NORM_CH(k_norm_bwd, T, N, C, X, sum, rstd, w, dy, dX, part);
    return cudaGetLastError();
}

cudaError_t launch_norm_dw(int P, int C, const float* part, float* dw, int accumulate, cudaStream_t st) {
    XHC_LAUNCH(st, (C + 31) / 32, 256, 0, (k_norm_dw), P, C, part, dw, accumulate);
    return cudaGetLastError();
}

}  // namespace xhc
