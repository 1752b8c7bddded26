// RMS norm of the sum of a token's N streams (N = 1: the norm of a hidden vector):
//   s[c] = sum_i X[t][i][c],  r = 1 / sqrt(mean_c s[c]^2 + eps),  y[c] = w[c] s[c] r
// and its backward, with n = s r:
//   ds[c] = r (w[c] dy[c] - n[c] mean_c(w dy n)),  dX[t][i] = ds for every i,  dw[c] = sum_t dy[c] n[c]
// Both are bound by memory: the state is read once and kept in registers between the sum of squares and
// the store.  A group of up to 512 threads holds a token, 8 channels (16 bytes of bf16) a thread and chunk.  Where a token
// is one or two rows (N = 1, and every backward) its loads are too few to fill the memory's latency, so each
// thread copies its chunks of the next tokens into shared memory ahead (cp.async: no registers, and no other thread
// reads them): T = 32768, N = 1, C = 4096 takes 95 us forward (5.7 TB/s) and 141 backward (5.7); with the next token in
// registers it took 116 and 147.  T = 2048, N = 16, C = 4096 with s kept: 52 us forward (6.1 TB/s), 55 backward.  The backward
// reads s in fp32 as the forward left it (N = 1: X itself, which is s): 4 bytes a channel where the state has
// 2 N.  In bf16 it would put 2^-9 into every term of dw, which is fp32.
#include "xhc_internal.cuh"

namespace xhc {

namespace {

constexpr int NORM_NT = 512;   // most threads of a block

// The sum of v over the nt threads of group `id` of a block (every thread gets it): warps by shuffles, then the
// warps' sums alike.  sh: 2 x 16 floats of the group, used in turn, so that one barrier is enough.
__device__ __forceinline__ float group_sum(float v, float* sh, int turn, int nt, int id, int tid) {
    v = warp_sum(v);
    if (nt <= 32) return v;
    float* s = sh + 16 * (turn & 1);
    if ((tid & 31) == 0) s[tid >> 5] = v;
    asm volatile("bar.sync %0, %1;" ::"r"(id + 1), "r"(nt) : "memory");
    const int lane = tid & 31;
    float t = lane < nt >> 5 ? s[lane] : 0.f;   // at most 16 warps
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
    return __shfl_sync(0xffffffffu, t, 0);
}

// s of one chunk of 8 channels: the N streams added in order, in fp32, U loads in flight
template <int U>
__device__ __forceinline__ void stream_chunk(const uint16_t* x, int N, int C, float* s) {
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = 0.f;
    int i = 0;
    for (; i + U <= N; i += U) {
        uint4 v[U];
#pragma unroll
        for (int q = 0; q < U; ++q) v[q] = ld_stream(x + (int64_t)(i + q) * C);
#pragma unroll
        for (int q = 0; q < U; ++q) {
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

// 16 bytes into shared memory, in the thread's own time; a group is what was begun since the last commit
__device__ __forceinline__ void copy16(void* to, const void* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int n>
__device__ __forceinline__ void copy_wait() {   // all but the last n groups are there
    asm volatile("cp.async.wait_group %0;" ::"n"(n) : "memory");
}

__device__ __forceinline__ void load8(const float* p, float* v) {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void store8(float* p, const float* v) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}

// A block holds a token at a time.  CH: chunks of 8 channels a thread holds at most; U: streams in flight
template <int CH, int U>
__global__ void __launch_bounds__(NORM_NT) k_norm_fwd(int T, int N, int C, float eps, const uint16_t* X, const float* w,
                                                      uint16_t* y, float* sum, float* rstd) {
    pdl_entry();
    __shared__ float sh[32];
    const int nch = C / 8, nt = blockDim.x;
    int turn = 0;
    for (int64_t t = blockIdx.x; t < T; t += gridDim.x, ++turn) {
        float s[CH][8], q2 = 0.f;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int q = threadIdx.x + j * nt;
            if (q >= nch) continue;
            stream_chunk<U>(X + t * N * C + 8 * q, N, C, s[j]);
#pragma unroll
            for (int e = 0; e < 8; ++e) q2 = fmaf(s[j][e], s[j][e], q2);
        }
        const float r = rsqrtf(fmaf(group_sum(q2, sh, turn, nt, 0, threadIdx.x), 1.0f / (float)C, eps));
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int q = threadIdx.x + j * nt;
            if (q >= nch) continue;
            float wv[8], o[8];
            load8(w + 8 * q, wv);
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = s[j][e] * r * wv[e];
            *reinterpret_cast<uint4*>(y + t * C + 8 * q) = pack8(o);
            if (sum) store8(sum + t * C + 8 * q, s[j]);
        }
        if (rstd && threadIdx.x == 0) rstd[t] = r;
    }
}

// The same for N = 1, with NORM_AHEAD tokens in flight
constexpr int NORM_AHEAD = 3;
template <int CH>
__global__ void __launch_bounds__(NORM_NT, CH == 1 ? 4 : 1) k_norm_fwd1(int T, int C, float eps, const uint16_t* X, const float* w,
                                                                      uint16_t* y, float* rstd) {
    pdl_entry();
    extern __shared__ uint4 ring[];   // [NORM_AHEAD][CH][nt]
    __shared__ float sh[32];
    const int nch = C / 8, nt = blockDim.x;
    const int64_t step = (int64_t)gridDim.x * C;
    const float inv = 1.0f / (float)C;
    const int64_t at = (int64_t)blockIdx.x * C + threadIdx.x * 8;
    const uint16_t* from = X + at;   // of the next token to copy
    int ahead = blockIdx.x;
    auto fetch = [&](uint4* to) {
        if (ahead < T) {
#pragma unroll
            for (int j = 0; j < CH; ++j)
                if (threadIdx.x + j * nt < nch) copy16(to + j * nt, from + j * nt * 8);
        }
        copy_commit();
        from += step;
        ahead += gridDim.x;
    };
    uint4* mine = ring + threadIdx.x;
#pragma unroll
    for (int k = 0; k < NORM_AHEAD; ++k) fetch(mine + k * CH * nt);
    y += at;
    int turn = 0, k = 0;
    for (int t = blockIdx.x; t < T; t += gridDim.x, ++turn, y += step) {
        float s[CH][8], q2 = 0.f;
        copy_wait<NORM_AHEAD - 1>();
        uint4* slot = mine + k * CH * nt;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            if (threadIdx.x + j * nt >= nch) continue;
            unpack8(slot[j * nt], s[j]);
#pragma unroll
            for (int e = 0; e < 8; ++e) q2 = fmaf(s[j][e], s[j][e], q2);
        }
        fetch(slot);
        if (++k == NORM_AHEAD) k = 0;
        const float r = rsqrtf(fmaf(group_sum(q2, sh, turn, nt, 0, threadIdx.x), inv, eps));
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int q = threadIdx.x + j * nt;
            if (q >= nch) continue;
            float wv[8], o[8];
            load8(w + 8 * q, wv);
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = s[j][e] * r * wv[e];
            *reinterpret_cast<uint4*>(y + j * nt * 8) = pack8(o);
        }
        if (rstd && threadIdx.x == 0) rstd[t] = r;
    }
}

// blockDim.y groups of blockDim.x threads, a token each at a time: group g of block b walks tokens
// b G + g, + gridDim.x G, ...  The block's part of dw goes to part[b][C], its groups added in order.
// A thread copies the chunks of norm_back tokens ahead: dy and X (ONE: N = 1), or dy and the two halves of s.
constexpr int norm_back(int chunks, bool one) { return chunks <= 2 ? 3 : one ? 3 : 2; }   // 197 KB of a block at most
template <int CH, bool ONE>
__global__ void __launch_bounds__(NORM_NT, CH == 1 ? 2 : 1) k_norm_bwd(int T, int N, int C, const uint16_t* X, const float* sum,
                                                                     const float* rstd, const float* w, const uint16_t* dy,
                                                                     uint16_t* dX, float* part) {
    pdl_entry();
    constexpr int OPS = ONE ? 2 : 3, BACK = norm_back(CH, ONE);
    extern __shared__ uint4 ring[];   // [BACK][CH][OPS][G nt], then per group 32 floats, then the block's dw [C]
    const int nch = C / 8, nt = blockDim.x, g = threadIdx.y, tid = threadIdx.x, all = nt * blockDim.y, me = g * nt + tid;
    float* sm = reinterpret_cast<float*>(ring + BACK * CH * OPS * all);
    float* sh = sm + 32 * g;
    float dw[CH][8];
#pragma unroll
    for (int j = 0; j < CH; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[j][e] = 0.f;
    const int groups = gridDim.x * blockDim.y, t0 = blockIdx.x * blockDim.y + g;   // tokens t0, t0 + groups, ...
    const int64_t step = (int64_t)groups * C;
    const float inv = 1.0f / (float)C;
    int64_t from = (int64_t)t0 * C + tid * 8;   // of the next token to copy
    int ahead = t0;
    auto fetch = [&](uint4* to) {
        if (ahead < T) {
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                if (tid + j * nt >= nch) continue;
                const int64_t o = from + j * nt * 8;
                copy16(to + j * OPS * all, dy + o);
                if (ONE) {
                    copy16(to + (j * OPS + 1) * all, X + o);
                } else {
                    copy16(to + (j * OPS + 1) * all, sum + o);
                    copy16(to + (j * OPS + 2) * all, sum + o + 4);
                }
            }
        }
        copy_commit();
        from += step;
        ahead += groups;
    };
#pragma unroll
    for (int k = 0; k < BACK; ++k) fetch(ring + k * CH * OPS * all + me);
    float nr = t0 < T ? rstd[t0] : 0.f;
    int turn = 0, k = 0;
    dX += ((int64_t)t0 * N * C + tid * 8);
    for (int t = t0; t < T; t += groups, ++turn, dX += step * N) {
        float n[CH][8], d[CH][8], dot = 0.f;
        const float r = nr;
        if (t + groups < T) nr = rstd[t + groups];
        copy_wait<BACK - 1>();
        uint4* slot = ring + k * CH * OPS * all + me;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int q = tid + j * nt;
            if (q >= nch) continue;
            const uint4* at = slot + j * OPS * all;
            unpack8(at[0], d[j]);
            if (ONE) {
                unpack8(at[all], n[j]);
            } else {
                const uint4 a = at[all], b = at[2 * all];
                const uint32_t u[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
                for (int e = 0; e < 8; ++e) n[j][e] = __uint_as_float(u[e]);
            }
            float wv[8];
            load8(w + 8 * q, wv);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                n[j][e] *= r;
                dw[j][e] = fmaf(d[j][e], n[j][e], dw[j][e]);
                d[j][e] *= wv[e];
                dot = fmaf(d[j][e], n[j][e], dot);
            }
        }
        fetch(slot);
        if (++k == BACK) k = 0;
        const float m = group_sum(dot, sh, turn, nt, g, tid) * inv;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            if (tid + j * nt >= nch) continue;
            float o[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = r * (d[j][e] - n[j][e] * m);
            const uint4 v = pack8(o);
            uint16_t* to = dX + j * nt * 8;
            if (ONE) {
                *reinterpret_cast<uint4*>(to) = v;
            } else {
                for (int i = 0; i < N; ++i, to += C) *reinterpret_cast<uint4*>(to) = v;
            }
        }
    }
    float* acc = sm + 32 * blockDim.y;
    for (int q = 0; q < (int)blockDim.y; ++q) {
        const bool last = q + 1 == (int)blockDim.y;
        if (g == q) {
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                const int c = (tid + j * nt) * 8;
                if (c >= C) continue;
                if (q > 0) {
                    float a[8];
                    load8(acc + c, a);
#pragma unroll
                    for (int e = 0; e < 8; ++e) dw[j][e] += a[e];
                }
                store8(last ? part + (int64_t)blockIdx.x * C + c : acc + c, dw[j]);
            }
        }
        if (!last) __syncthreads();
    }
}

// dw[c] (+)= sum over the blocks' parts: 32 channels a block, 16 threads a channel over interleaved parts (8 loads in
// flight), then these in order
constexpr int DW_TY = 16;
__global__ void __launch_bounds__(32 * DW_TY) k_norm_dw(int P, int C, const float* part, float* dw, int accumulate) {
    pdl_entry();
    __shared__ float sh[DW_TY][33];
    const int x = threadIdx.x & 31, ty = threadIdx.x >> 5, c = blockIdx.x * 32 + x;
    float s = 0.f;
    if (c < C) {
#pragma unroll 8
        for (int p = ty; p < P; p += DW_TY) s += part[(int64_t)p * C + c];
    }
    sh[ty][x] = s;
    __syncthreads();
    if (ty == 0 && c < C) {
        float t = 0.f;
#pragma unroll
        for (int q = 0; q < DW_TY; ++q) t += sh[q][x];
        dw[c] = accumulate ? dw[c] + t : t;
    }
}

// Threads of a token in whole warps: a chunk of 8 channels each up to 512 threads, else 2 or 4.  (More chunks share the
// sum over the threads among them, but leave too few warps: with 4 at T = 32768, N = 1, C = 4096 138 us forward for 103.)
int norm_chunks(int C) { return C / 8 <= NORM_NT ? 1 : C / 8 <= 2 * NORM_NT ? 2 : 4; }
int norm_threads(int C) { return (C / 8 + norm_chunks(C) * 32 - 1) / (norm_chunks(C) * 32) * 32; }

}  // namespace

// The backward's blocks: groups of threads fill them to 512 threads, and blocks an SM to 1024 (512, where a thread holds
// more than a chunk), so that the parts of dw stay a few bytes a channel for every SM.
static int norm_bwd_groups(int C) { return NORM_NT / norm_threads(C); }
int norm_bwd_blocks(int64_t T, int C) {
    const int64_t g = norm_bwd_groups(C), b = (T + g - 1) / g;
    const int64_t most = (int64_t)device_sms() * (norm_chunks(C) == 1 ? 1024 / (int)(g * norm_threads(C)) : 1);
    return (int)(b < most ? b : most);
}

#define NORM_CH(chunks, LAUNCH)                              \
    do {                                                     \
        const int ch_ = chunks;                              \
        if (ch_ <= 1) { LAUNCH(1); }                         \
        else if (ch_ <= 2) { LAUNCH(2); }                    \
        else { LAUNCH(4); }                                  \
    } while (0)

// Few tokens: all of a token's streams in flight at once (24 tokens of 16 x 4096: 4.0 us captured; 8 streams at a
// time and two chunks a thread took 2.3 us more).
cudaError_t launch_norm_fwd(int T, int N, int C, float eps, const uint16_t* X, const float* w, uint16_t* y,
                            float* sum, float* rstd, cudaStream_t st) {
    const int nt = norm_threads(C);
    if (N == 1) {
        const size_t smem = (size_t)NORM_AHEAD * norm_chunks(C) * nt * 16;
        const int per = norm_chunks(C) == 1 ? 2048 / nt : 1;   // blocks an SM
        const int64_t most = (int64_t)device_sms() * (per < 32 ? per : 32);
        const int grid = (int)(T < most ? T : most);
#define NORM_FWD1(CH)                                                                             \
    const cudaError_t e_ = smem_optin((const void*)k_norm_fwd1<CH>, smem);                        \
    if (e_ != cudaSuccess) return e_;                                                             \
    XHC_LAUNCH(st, grid, nt, smem, (k_norm_fwd1<CH>), T, C, eps, X, w, y, rstd)
        NORM_CH(norm_chunks(C), NORM_FWD1);
        return cudaGetLastError();
    }
    const int64_t most = (int64_t)device_sms() * 64;
    const int grid = (int)(T < most ? T : most);
    const bool wide = T <= 2 * device_sms() && N >= 16;
#define NORM_FWD(CH)                                                                                               \
    if (wide) XHC_LAUNCH(st, grid, nt, 0, (k_norm_fwd<CH, 16>), T, N, C, eps, X, w, y, sum, rstd);                  \
    else XHC_LAUNCH(st, grid, nt, 0, (k_norm_fwd<CH, 8>), T, N, C, eps, X, w, y, sum, rstd)
    NORM_CH(norm_chunks(C), NORM_FWD);
    return cudaGetLastError();
}

cudaError_t launch_norm_bwd(int T, int N, int C, const uint16_t* X, const float* sum, const float* rstd, const float* w,
                            const uint16_t* dy, uint16_t* dX, float* part, cudaStream_t st) {
    const int ch = norm_chunks(C), nt = norm_threads(C), grid = norm_bwd_blocks(T, C);
    const dim3 block(nt, norm_bwd_groups(C));
    const size_t smem = (size_t)norm_back(ch, N == 1) * ch * (N == 1 ? 2 : 3) * nt * block.y * 16 +
                        (32 * block.y + (block.y > 1 ? C : 0)) * sizeof(float);
#define NORM_BWD_OF(CH, ONE)                                                                      \
    const cudaError_t e_ = smem_optin((const void*)k_norm_bwd<CH, ONE>, smem);                    \
    if (e_ != cudaSuccess) return e_;                                                             \
    XHC_LAUNCH(st, grid, block, smem, (k_norm_bwd<CH, ONE>), T, N, C, X, sum, rstd, w, dy, dX, part)
#define NORM_BWD(CH)                    \
    if (N == 1) { NORM_BWD_OF(CH, true); } \
    else { NORM_BWD_OF(CH, false); }
    NORM_CH(ch, NORM_BWD);
    return cudaGetLastError();
}

cudaError_t launch_norm_dw(int P, int C, const float* part, float* dw, int accumulate, cudaStream_t st) {
    XHC_LAUNCH(st, (C + 31) / 32, 32 * DW_TY, 0, (k_norm_dw), P, C, part, dw, accumulate);
    return cudaGetLastError();
}

}  // namespace xhc
