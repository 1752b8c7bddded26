// The gated feed-forward block on the 5th-generation tensor cores:
//   forward   h = q u, q = act(g), g = x W_gate^T, u = x W_up^T;  y = h W_down^T
//   backward  dh = dy W_down;  dg = dh p, p = u act'(g);  du = dh q
//             dx = dg W_gate + du W_up;  dW_gate = dg^T x, dW_up = du^T x, dW_down = dy^T h
// One persistent kernel template runs all of these products.  A tile of 128 CG x 128 CG outputs belongs to
// a CTA (CG = 1) or to a pair of CTAs on two SMs (CG = 2: each stages half of A's rows and half of B's, the
// MMA reads both halves, so an operand byte in shared memory feeds twice the products).  Operands arrive by
// TMA in the memory's own order: K-major where a row holds the summed index, MN-major where it holds
// the output's (the weights in the input gradients, both operands of the weight gradients), so nothing is
// transposed.  Warp 0 loads, warp 1 issues the MMAs, warps 2..5 read the finished accumulator from TMEM
// and store; two accumulators let the stores of a tile run under the products of the next.
// Rounding: h, p, q, dg and du are stored as bf16 (once, from fp32): they are operands of the next product,
// whose matrix instruction takes 16-bit operands; p and q rather than g and u, so that the
// activation's derivative is formed from the fp32 g and the backward needs no activation at all.
#include <math.h>

#include "k_tc.cuh"

namespace xhc {

namespace {

constexpr int GM_NT = 192;
constexpr int GM_BK = 64;                       // k-elements of a stage: one 128-byte swizzle row of bf16
constexpr int GM_HALF = 128 * GM_BK * 2;        // one operand's bytes of a stage and CTA
constexpr int GM_STAGE = 2 * GM_HALF;
constexpr int GM_STAGES = 6;
constexpr int GM_SMEM = GM_STAGES * GM_STAGE + (2 * GM_STAGES + 5) * 8 + 16 + 1024;
constexpr int GM_GROUP = 8;                     // tile rows walked together: their B tiles are shared in L2

enum { EPI_GATE, EPI_OUT, EPI_DH };

struct GemmMaps {
    CUtensorMap a[3], b[3];
};

struct GemmArgs {
    int nprob;              // problems (EPI_OUT: up to 3, each with its own operands; else 1)
    int M[3], N[3];         // output rows and columns
    int tm[3], tn[3];       // tiles
    int first[4];           // first tile of each problem
    int kb1, kb;            // k-blocks of the first operand pair and of both (EPI_OUT of one problem)
    int act;
    uint64_t wait_ns;
    int* err;
    void* out[3];           // EPI_GATE: h; EPI_OUT: the products; EPI_DH: dg, du
    uint4* p;               // EPI_GATE (null: not kept), EPI_DH: p and q, see pq_at
    uint4* q;
    int f32, accumulate;    // EPI_OUT: fp32 outputs, added to what is there
};

// p and q lie in blocks of 32 rows and 8 columns, a row's 16 bytes after the other: the 32 lanes of an
// epilogue warp hold 32 rows of the same columns, and so write and read 512 contiguous bytes.
__host__ __device__ __forceinline__ int64_t pq_at(int64_t row, int col, int F) {
    return ((row >> 5) * (F / 8) + col / 8) * 32 + (row & 31);
}

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// the address of the same variable in CTA `rank` of the cluster
__device__ __forceinline__ uint32_t map_rank(uint32_t a, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
    return r;
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t a) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(a) : "memory");
}

template <int CG>
__device__ __forceinline__ void gm_load(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    if (CG == 1) {
        tma_load_2d(dst, map, x, y, bar);
    } else {
        // own shared memory, the barrier of the pair's first CTA
        asm volatile(
            "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
            " [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"((uint64_t)map), "r"(x), "r"(y), "r"(bar)
            : "memory");
    }
}
template <int CG>
__device__ __forceinline__ void gm_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accum) {
    if (CG == 1) {
        mma_bf16(d, a, b, idesc, accum);
    } else {
        asm volatile(
            "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
            " tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d), "l"(a), "l"(b), "r"(idesc),
            "r"(accum)
            : "memory");
    }
}
// the barrier at this offset, in both CTAs of a pair, is arrived at when the MMAs issued so far are done
template <int CG>
__device__ __forceinline__ void gm_commit(uint32_t bar) {
    if (CG == 1) {
        mma_commit(bar);
    } else {
        asm volatile(
            "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
            "h"((uint16_t)3)
            : "memory");
    }
}

// act(g) and its derivative
__device__ __forceinline__ void mlp_act(int act, float g, float& q, float& dq) {
    if (act == XHC_ACT_SILU) {
        const float e = 1.0f / (1.0f + expf(-g));
        q = g * e;
        dq = e * (1.0f + g * (1.0f - e));
    } else if (act == XHC_ACT_GELU) {
        const float c = normcdff(g);
        q = g * c;
        dq = c + g * 0.3989422804f * expf(-0.5f * g * g);
    } else {
        q = g > 0.f ? g : g != g ? g : 0.f;
        dq = g > 0.f ? 1.f : 0.f;
    }
}

struct GmTile {
    int p, m, n;   // problem, tile row, tile column
};
__device__ __forceinline__ GmTile gm_tile(const GemmArgs& a, int t) {
    GmTile r;
    r.p = 0;
    while (r.p + 1 < a.nprob && t >= a.first[r.p + 1]) ++r.p;
    t -= a.first[r.p];
    const int per = GM_GROUP * a.tn[r.p], g = t / per, rows = min(GM_GROUP, a.tm[r.p] - g * GM_GROUP);
    t -= g * per;
    r.n = t / rows;
    r.m = g * GM_GROUP + t - r.n * rows;
    return r;
}

template <int CG, bool AMN, bool BMN, int EPI>
__global__ void __launch_bounds__(GM_NT, 1) k_mlp_gemm(const __grid_constant__ GemmMaps maps, GemmArgs a) {
    constexpr int BM = 128 * CG, BN = 128 * CG;          // the tile
    constexpr int TN = EPI == EPI_GATE ? BN / 2 : BN;    // output columns: gate and up share an accumulator
    constexpr uint32_t COLS = 2 * BN;                    // TMEM columns: two accumulators
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + GM_STAGES * GM_STAGE);
    const uint32_t full = smem_u32(bars), empty = full + 8 * GM_STAGES, accfull = empty + 8 * GM_STAGES,
                   accempty = accfull + 16, drain = accempty + 16;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * GM_STAGES + 5);
    __shared__ int s_abort;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = CG == 2 ? cluster_rank() : 0u;
    const int c0 = blockIdx.x / CG, nc = gridDim.x / CG, tiles = a.first[a.nprob];

    if (threadIdx.x == 0) {
        s_abort = 0;
        for (int s = 0; s < GM_STAGES; ++s) {
            mbar_init(full + 8 * s, 1);
            mbar_init(empty + 8 * s, 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(accfull + 8 * s, 1);
            mbar_init(accempty + 8 * s, 4 * CG);
        }
        mbar_init(drain, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        if (CG == 1) {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(COLS) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(COLS) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        }
    }
    tc_fence_before();
    __syncthreads();
    if (CG == 2) cluster_sync();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    pdl_entry();

    auto give_up = [&](int code) {
        atomicExch(a.err, code);
        *(volatile int*)&s_abort = 1;
    };
    auto aborted = [&]() { return *(volatile int*)&s_abort != 0; };

    if (warp == 0) {
        // ---------------- TMA producer ----------------
        if (lane == 0) {
            const uint32_t lead = CG == 2 ? map_rank(full, 0) : full;
            int s = 0, issued = 0;
            uint32_t ph = 0;
            for (int t = c0; t < tiles && !aborted(); t += nc) {
                const GmTile tl = gm_tile(a, t);
                const int m0 = tl.m * BM + (int)rank * 128, n0 = tl.n * TN;
                for (int kb = 0; kb < a.kb; ++kb) {
                    if (issued >= GM_STAGES && !mbar_wait(empty + 8 * s, ph ^ 1, a.wait_ns)) {
                        give_up(11);
                        break;
                    }
                    if (aborted()) break;
                    if (rank == 0) mbar_expect_tx(full + 8 * s, CG * GM_STAGE);
                    const int set = EPI == EPI_OUT ? (a.nprob > 1 ? tl.p : kb >= a.kb1 ? 1 : 0) : 0;
                    const int k0 = (set && a.nprob == 1 ? kb - a.kb1 : kb) * GM_BK;
                    const uint32_t sa = smem_u32(smem + s * GM_STAGE), sb = sa + GM_HALF, bar = lead + 8 * s;
                    if (AMN) {
                        gm_load<CG>(sa, &maps.a[set], m0, k0, bar);
                        gm_load<CG>(sa + GM_HALF / 2, &maps.a[set], m0 + 64, k0, bar);
                    } else {
                        gm_load<CG>(sa, &maps.a[set], k0, m0, bar);
                    }
                    if (EPI == EPI_GATE) {
                        // gate rows, then up rows: the halves of the accumulator's columns
                        if (CG == 2) {
                            gm_load<CG>(sb, &maps.b[rank], k0, n0, bar);
                        } else {
                            gm_load<CG>(sb, &maps.b[0], k0, n0, bar);
                            gm_load<CG>(sb + GM_HALF / 2, &maps.b[1], k0, n0, bar);
                        }
                    } else if (BMN) {
                        gm_load<CG>(sb, &maps.b[set], n0 + (int)rank * 128, k0, bar);
                        gm_load<CG>(sb + GM_HALF / 2, &maps.b[set], n0 + (int)rank * 128 + 64, k0, bar);
                    } else {
                        gm_load<CG>(sb, &maps.b[set], k0, n0 + (int)rank * 128, bar);
                    }
                    ++issued;
                    if (++s == GM_STAGES) { s = 0; ph ^= 1u; }
                }
            }
            if (!aborted()) {
                // the MMAs' releases of the last stages reach both CTAs of a pair before either ends
                for (int q = 0; q < GM_STAGES; ++q) {
                    if (issued + q >= GM_STAGES && !mbar_wait(empty + 8 * s, ph ^ 1, a.wait_ns)) {
                        give_up(15);
                        break;
                    }
                    if (++s == GM_STAGES) { s = 0; ph ^= 1u; }
                }
            } else if (rank == 0) {
                // a wait ran out: the copies in flight land before this memory is given back
                for (int q = 0; q < GM_STAGES && q < issued; ++q) {
                    if (--s < 0) { s = GM_STAGES - 1; ph ^= 1u; }
                    mbar_wait(full + 8 * s, ph, a.wait_ns);
                }
            }
        }
    } else if (warp == 1) {
        // ---------------- MMA issuer ----------------
        if (lane == 0 && rank == 0) {
            const uint32_t idesc = idesc_bf16(BM, BN, AMN) | ((BMN ? 1u : 0u) << 16);
            int s = 0, i = 0;
            uint32_t ph = 0;
            for (int t = c0; t < tiles && !aborted(); t += nc, ++i) {
                const int buf = i & 1;
                if (i >= 2 && !mbar_wait(accempty + 8 * buf, (uint32_t)((i >> 1) & 1) ^ 1u, a.wait_ns)) {
                    give_up(12);
                    break;
                }
                tc_fence_after();
                for (int kb = 0; kb < a.kb; ++kb) {
                    if (!mbar_wait(full + 8 * s, ph, a.wait_ns)) {
                        give_up(13);
                        break;
                    }
                    tc_fence_after();
                    const uint32_t sa = smem_u32(smem + s * GM_STAGE), sb = sa + GM_HALF;
#pragma unroll
                    for (int kk = 0; kk < GM_BK / 16; ++kk) {
                        // K-major: 32 bytes on in the swizzled row; MN-major: 16 rows of 128 bytes on
                        const uint64_t da = AMN ? sw128_desc_mn(sa + kk * 2048, GM_HALF / 2) : sw128_desc(sa + kk * 32);
                        const uint64_t db = BMN ? sw128_desc_mn(sb + kk * 2048, GM_HALF / 2) : sw128_desc(sb + kk * 32);
                        gm_mma<CG>(tmem + (uint32_t)(buf * BN), da, db, idesc, (kb | kk) ? 1u : 0u);
                    }
                    gm_commit<CG>(empty + 8 * s);
                    if (++s == GM_STAGES) { s = 0; ph ^= 1u; }
                }
                if (aborted()) break;
                gm_commit<CG>(accfull + 8 * buf);
            }
            if (aborted()) {   // the MMAs issued so far end before TMEM is given back
                gm_commit<CG>(drain);
                mbar_wait(drain, 0, a.wait_ns);
            }
        }
    } else {
        // ---------------- epilogue (warps 2..5) ----------------
        const int quarter = warp & 3;
        const uint32_t free_bar = CG == 2 ? map_rank(accempty, 0) : accempty;
        int i = 0;
        for (int t = c0; t < tiles && !__any_sync(0xffffffffu, aborted()); t += nc, ++i) {
            const GmTile tl = gm_tile(a, t);
            const int buf = i & 1;
            if (!__all_sync(0xffffffffu, mbar_wait(accfull + 8 * buf, (uint32_t)((i >> 1) & 1), a.wait_ns))) {
                if (lane == 0) give_up(14);
                break;
            }
            tc_fence_after();
            const int M = a.M[tl.p], N = a.N[tl.p];
            const int row = tl.m * BM + (int)rank * 128 + quarter * 32 + lane, n0 = tl.n * TN;
            const uint32_t acc = tmem + (uint32_t)(buf * BN) + ((uint32_t)(quarter * 32) << 16);
            for (int c = 0; c < TN && n0 + c < N; c += 16) {
                float v[16];
                tmem_ld16(acc + c, v);
                if (EPI == EPI_GATE) {
                    float u[16], p[16];
                    tmem_ld16(acc + TN + c, u);
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        float dq;
                        mlp_act(a.act, v[e], v[e], dq);
                        p[e] = u[e] * dq;
                        u[e] *= v[e];
                    }
                    if (row < M) {
#pragma unroll
                        for (int o = 0; o < 16; o += 8)
                            if (n0 + c + o < N) {
                                *reinterpret_cast<uint4*>((uint16_t*)a.out[0] + (int64_t)row * N + n0 + c + o) = pack8(u + o);
                                if (a.p) {
                                    a.p[pq_at(row, n0 + c + o, N)] = pack8(p + o);
                                    a.q[pq_at(row, n0 + c + o, N)] = pack8(v + o);
                                }
                            }
                    }
                } else if (EPI == EPI_DH) {
                    if (row < M) {
#pragma unroll
                        for (int o = 0; o < 16; o += 8)
                            if (n0 + c + o < N) {
                                float p[8], q[8];
                                unpack8(a.p[pq_at(row, n0 + c + o, N)], p);
                                unpack8(a.q[pq_at(row, n0 + c + o, N)], q);
#pragma unroll
                                for (int e = 0; e < 8; ++e) {
                                    p[e] *= v[o + e];
                                    q[e] *= v[o + e];
                                }
                                const int64_t at = (int64_t)row * N + n0 + c + o;
                                *reinterpret_cast<uint4*>((uint16_t*)a.out[0] + at) = pack8(p);
                                *reinterpret_cast<uint4*>((uint16_t*)a.out[1] + at) = pack8(q);
                            }
                    }
                } else if (row < M) {
#pragma unroll
                    for (int o = 0; o < 16; o += 8)
                        if (n0 + c + o < N) {
                            const int64_t at = (int64_t)row * N + n0 + c + o;
                            if (!a.f32) {
                                *reinterpret_cast<uint4*>((uint16_t*)a.out[tl.p] + at) = pack8(v + o);
                            } else {
                                float4* to = reinterpret_cast<float4*>((float*)a.out[tl.p] + at);
                                float4 x = make_float4(v[o], v[o + 1], v[o + 2], v[o + 3]), z = make_float4(v[o + 4], v[o + 5], v[o + 6], v[o + 7]);
                                if (a.accumulate) {
                                    const float4 x0 = to[0], z0 = to[1];
                                    x.x += x0.x; x.y += x0.y; x.z += x0.z; x.w += x0.w;
                                    z.x += z0.x; z.y += z0.y; z.z += z0.z; z.w += z0.w;
                                }
                                to[0] = x;
                                to[1] = z;
                            }
                        }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (CG == 2) mbar_arrive_cluster(free_bar + 8 * buf);
                else mbar_arrive(free_bar + 8 * buf);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (CG == 2) cluster_sync();   // the pair's MMAs, arrivals and copies are done in both CTAs
    if (warp == 1) {
        tc_fence_after();
        if (CG == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(COLS) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(COLS) : "memory");
    }
}

// ---- host ----

// A launch of CG-CTA clusters: as many as the GPU holds at once, at most one per tile.  (An SM without a
// partner in its cluster of SMs takes no pair: the driver says how many fit.)
template <int CG, bool AMN, bool BMN, int EPI>
cudaError_t gm_launch(const GemmMaps& maps, const GemmArgs& a, cudaStream_t st) {
    auto* k = k_mlp_gemm<CG, AMN, BMN, EPI>;
    cudaError_t e = smem_optin((const void*)k, GM_SMEM);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(GM_NT);
    cfg.dynamicSmemBytes = GM_SMEM;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = CG;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    int most = device_sms();
    if (CG == 2) {
        cfg.gridDim = dim3(device_sms() / 2 * 2);
        if ((e = cudaOccupancyMaxActiveClusters(&most, k, &cfg)) != cudaSuccess) return e;
        if (most < 1) return cudaErrorInvalidConfiguration;
    }
    const int tiles = a.first[a.nprob];
    cfg.gridDim = dim3(CG * (tiles < most ? tiles : most));
    cfg.numAttrs = pdl_on() ? 2 : 1;
    e = cudaLaunchKernelEx(&cfg, k, maps, a);
    note_launch();
    return e == cudaSuccess ? cudaGetLastError() : e;
}

// Pairs or single CTAs: the time of a product's last wave counts.  A single CTA's tile has a quarter of a
// pair's products on half the SMs and reads twice the shared memory for them.
bool gm_pairs(int64_t tiles2, int64_t tiles1) {
    const int sms = device_sms();
    const int64_t w2 = (tiles2 + sms / 2 - 1) / (sms / 2), w1 = (tiles1 + sms - 1) / sms;
    return 10 * 2 * w2 <= 13 * w1;
}

void gm_tiles(GemmArgs& a, int cg, bool gate) {
    a.first[0] = 0;
    for (int p = 0; p < a.nprob; ++p) {
        const int bm = 128 * cg, tn = gate ? bm / 2 : bm;
        a.tm[p] = (a.M[p] + bm - 1) / bm;
        a.tn[p] = (a.N[p] + tn - 1) / tn;
        a.first[p + 1] = a.first[p] + a.tm[p] * a.tn[p];
    }
}

template <bool AMN, bool BMN, int EPI>
cudaError_t gm_run(const GemmMaps& maps, GemmArgs& a, int cg, cudaStream_t st) {
    gm_tiles(a, cg, EPI == EPI_GATE);
    if (cg == 2) return gm_launch<2, AMN, BMN, EPI>(maps, a, st);
    return gm_launch<1, AMN, BMN, EPI>(maps, a, st);
}

int gm_choose(GemmArgs& a, bool gate) {
    gm_tiles(a, 2, gate);
    const int t2 = a.first[a.nprob];
    gm_tiles(a, 1, gate);
    return gm_pairs(t2, a.first[a.nprob]) ? 2 : 1;
}

GemmArgs gm_args(int M, int N, int K, int* err) {
    GemmArgs a = {};
    a.nprob = 1;
    a.M[0] = M;
    a.N[0] = N;
    a.kb1 = a.kb = (K + GM_BK - 1) / GM_BK;
    a.err = err;
    a.wait_ns = debug_wait_ns();
    return a;
}

// operand stored [rows][inner] with the summed index inside: boxes of 64 k-elements and `box` rows
bool map_k(CUtensorMap* m, const void* p, int rows, int inner, int box) {
    return make_map_box(m, p, (uint64_t)inner, (uint64_t)rows, GM_BK, (uint32_t)box);
}
// operand stored [k][outputs]: boxes of 64 outputs and 64 k-elements
bool map_mn(CUtensorMap* m, const void* p, int k, int outs) {
    return make_map_box(m, p, (uint64_t)outs, (uint64_t)k, 64, GM_BK);
}

}  // namespace

size_t mlp_pq_bytes(int64_t T, int F) { return (size_t)((T + 31) / 32 * 32) * F * 2; }

cudaError_t launch_mlp_gate(int T, int C, int F, int act, const uint16_t* x, const uint16_t* Wg, const uint16_t* Wu,
                            uint16_t* h, void* p, void* q, int* err, cudaStream_t st) {
    GemmArgs a = gm_args(T, F, C, err);
    a.act = act;
    a.out[0] = h;
    a.p = (uint4*)p;
    a.q = (uint4*)q;
    const int cg = gm_choose(a, true);
    GemmMaps m;
    if (!map_k(&m.a[0], x, T, C, 128) || !map_k(&m.b[0], Wg, F, C, 64 * cg) || !map_k(&m.b[1], Wu, F, C, 64 * cg))
        return cudaErrorInvalidValue;
    m.a[1] = m.a[2] = m.a[0];
    m.b[2] = m.b[0];
    return gm_run<false, false, EPI_GATE>(m, a, cg, st);
}

cudaError_t launch_mlp_down(int T, int C, int F, const uint16_t* h, const uint16_t* Wd, uint16_t* y, int* err,
                            cudaStream_t st) {
    GemmArgs a = gm_args(T, C, F, err);
    a.out[0] = y;
    const int cg = gm_choose(a, false);
    GemmMaps m;
    if (!map_k(&m.a[0], h, T, F, 128) || !map_k(&m.b[0], Wd, C, F, 128)) return cudaErrorInvalidValue;
    m.a[1] = m.a[2] = m.a[0];
    m.b[1] = m.b[2] = m.b[0];
    return gm_run<false, false, EPI_OUT>(m, a, cg, st);
}

cudaError_t launch_mlp_dh(int T, int C, int F, const uint16_t* dy, const uint16_t* Wd, const void* p, const void* q,
                          uint16_t* dg, uint16_t* du, int* err, cudaStream_t st) {
    GemmArgs a = gm_args(T, F, C, err);
    a.p = (uint4*)const_cast<void*>(p);
    a.q = (uint4*)const_cast<void*>(q);
    a.out[0] = dg;
    a.out[1] = du;
    const int cg = gm_choose(a, false);
    GemmMaps m;
    if (!map_k(&m.a[0], dy, T, C, 128) || !map_mn(&m.b[0], Wd, C, F)) return cudaErrorInvalidValue;
    m.a[1] = m.a[2] = m.a[0];
    m.b[1] = m.b[2] = m.b[0];
    return gm_run<false, true, EPI_DH>(m, a, cg, st);
}

cudaError_t launch_mlp_dx(int T, int C, int F, const uint16_t* dg, const uint16_t* du, const uint16_t* Wg,
                          const uint16_t* Wu, uint16_t* dx, int* err, cudaStream_t st) {
    GemmArgs a = gm_args(T, C, F, err);
    a.kb = 2 * a.kb1;
    a.out[0] = dx;
    const int cg = gm_choose(a, false);
    GemmMaps m;
    if (!map_k(&m.a[0], dg, T, F, 128) || !map_k(&m.a[1], du, T, F, 128) || !map_mn(&m.b[0], Wg, F, C) ||
        !map_mn(&m.b[1], Wu, F, C))
        return cudaErrorInvalidValue;
    m.a[2] = m.a[0];
    m.b[2] = m.b[0];
    return gm_run<false, true, EPI_OUT>(m, a, cg, st);
}

cudaError_t launch_mlp_dw(int T, int C, int F, const uint16_t* x, const uint16_t* dy, const uint16_t* h,
                          const uint16_t* dg, const uint16_t* du, void* dWg, void* dWu, void* dWd, int f32,
                          int accumulate, int* err, cudaStream_t st) {
    GemmArgs a = gm_args(F, C, T, err);
    a.nprob = 3;
    a.M[1] = F;
    a.N[1] = C;
    a.M[2] = C;
    a.N[2] = F;
    a.out[0] = dWg;
    a.out[1] = dWu;
    a.out[2] = dWd;
    a.f32 = f32;
    a.accumulate = accumulate;
    const int cg = gm_choose(a, false);
    GemmMaps m;
    if (!map_mn(&m.a[0], dg, T, F) || !map_mn(&m.a[1], du, T, F) || !map_mn(&m.a[2], dy, T, C) ||
        !map_mn(&m.b[0], x, T, C) || !map_mn(&m.b[2], h, T, F))
        return cudaErrorInvalidValue;
    m.b[1] = m.b[0];
    return gm_run<true, true, EPI_OUT>(m, a, cg, st);
}

}  // namespace xhc
