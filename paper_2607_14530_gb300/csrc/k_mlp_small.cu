// The feed-forward block's forward for few tokens (a decode step), in one launch:
//   h = act(x W_gate^T) * (x W_up^T), then y = h W_down^T
// It is bound by reading the weights once, 6 C F bytes.  The weights are the MMA's A operand (M = 128), the tokens its
// N of 16 to 128: outputs transposed.  A tile is 64 outputs: of the first product 64 rows of W_gate above 64 of W_up;
// of the second the same 64 rows of W_down at two neighbouring k-steps, each multiplied with both steps'
// tokens, of which one half of the rows is used.  (Tiles of 128 outputs: 16 of them at C = 2048 left most SMs
// without work in the second product, 26 us a call for 24 tokens of F = 5632, now 22.)
// A cluster of four CTAs takes a tile, a quarter of its k-range each, through rings of 192 to 200 KB that keep
// the memory busy.  The four partial sums meet in shared memory: the lanes that hold rows 16 j .. 16 j + 15 send
// them to CTA j (st.async, which counts on j's barrier), and CTA j adds the four in order and finishes these
// rows.  (Equal shares of the stream for every SM with the parts left in L2 and waited for by
// counters took 59 us at C = 4096, F = 11008: every exchange is four trips through L2.)
// The cut depends on C and F alone: a token's bits do not depend on the other tokens or on their number.
// The second product needs all of h: the CTAs (one an SM, launched cooperatively, so all are there) meet at a
// counter.  Loads of W_down do not need h and fill the ring before that wait, so the stream of weights
// hardly stops between the products.
#include <atomic>

#include "k_mlp.cuh"

namespace xhc {

namespace {

constexpr int SM_NT = 192;                   // warp 0 TMA, warp 1 MMA, warps 2..5 epilogue
constexpr int SM_S = 4;                      // CTAs of a cluster
constexpr int SM_BOX = 64 * 64 * 2;          // a box of 64 weight rows and 64 k-elements; two a stage
constexpr int SM_ARRIVE = 0, SM_LEAVE = 1;   // counters

template <int NT>
struct SmShape {
    static constexpr int B = NT * 64 * 2, STAGE = 2 * SM_BOX + 2 * B;
    static constexpr int STAGES = NT == 16 ? 10 : NT == 32 ? 8 : NT == 64 ? 6 : 4;
    static constexpr int RT = NT < 32 ? NT : 32;            // tokens exchanged at a time
    static constexpr int PART = 2 * RT * 16;                // floats of a CTA's part: [half][token][row]
    static constexpr int RECV = SM_S * PART * 4;
    static constexpr int SMEM = STAGES * STAGE + 2 * RECV + (2 * STAGES + 7) * 8 + 16 + 1024;
    static constexpr uint32_t COLS = 4 * NT;                // two accumulators of two times NT columns
};

// One of the two products: `tiles` weight tiles of `kb` stages; cluster c takes tiles c, c + clusters, ..., its CTA r
// stages [kb r / 4, kb (r + 1) / 4) of each.
struct SmPhase {
    int kb, tiles;
};
struct SmMaps {
    CUtensorMap gate, up, down, x, h;
};
struct SmArgs {
    int T, C, F;
    int down_blocks;       // W_down and h in boxes of two k-steps (64 divides F)
    SmPhase ph[2];
    int* cnt;              // counters, zero between launches
    uint16_t *h, *y;
    unsigned char* pq;     // p, then q (null: not kept)
    int64_t q_off;
    uint64_t wait_ns;
    int* err;
};

__device__ __forceinline__ int ld_acquire(const int* p) {
    int v;
    asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
// after a barrier: what all its threads wrote before is seen by whoever sees the sum
__device__ __forceinline__ void add_release(int* p) {
    asm volatile("red.release.gpu.global.add.s32 [%0], 1;" ::"l"(p) : "memory");
}
// into the shared memory of a CTA of the cluster, counted in bytes on its barrier
__device__ __forceinline__ void send(uint32_t to, float a, uint32_t bar) {
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.b32 [%0], %1, [%2];" ::"r"(to), "r"(__float_as_uint(a)), "r"(bar) : "memory");
}
template <int NT, int ACT>
__global__ void __launch_bounds__(SM_NT, 1) k_mlp_small(const __grid_constant__ SmMaps maps, const __grid_constant__ SmArgs a) {
    using S = SmShape<NT>;
    constexpr int STAGES = S::STAGES, RT = S::RT;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    unsigned char* recv_mem = smem + STAGES * S::STAGE;
    uint64_t* bars = reinterpret_cast<uint64_t*>(recv_mem + 2 * S::RECV);
    const uint32_t full = smem_u32(bars), empty = full + 8 * STAGES, accfull = empty + 8 * STAGES, accempty = accfull + 16,
                   recv = accempty + 16, drain = recv + 16;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * STAGES + 7);
    __shared__ int s_abort, s_last;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)cluster_rank(), cl = blockIdx.x / SM_S, ncl = gridDim.x / SM_S;
    if (threadIdx.x == 0) {
        s_abort = 0;
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(full + 8 * s, 1);
            mbar_init(empty + 8 * s, 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(accfull + 8 * s, 1);
            mbar_init(accempty + 8 * s, 4);
            mbar_init(recv + 8 * s, 1);
        }
        mbar_init(drain, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(S::COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (warp == 2 && lane < 5) {
        const CUtensorMap* m = lane == 0 ? &maps.gate : lane == 1 ? &maps.up : lane == 2 ? &maps.x : lane == 3 ? &maps.down : &maps.h;
        asm volatile("prefetch.tensormap [%0];" ::"l"((uint64_t)m) : "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    pdl_entry();

    auto give_up = [&](int code) {
        atomicExch(a.err, code);
        *(volatile int*)&s_abort = 1;
    };
    auto aborted = [&]() { return __any_sync(0xffffffffu, *(volatile int*)&s_abort != 0) != 0; };   // of a whole warp
    // this CTA's stages of a tile
    auto first_of = [&](const SmPhase& q, int r) { return q.kb * r / SM_S; };

    if (warp == 0) {
        // ---------------- TMA producer ----------------
        int s = 0, issued = 0;
        uint32_t ph = 0;
        const uint32_t ring = smem_u32(smem);
        auto wait_h = [&]() {   // h is whole when every CTA has finished the first product
            uint64_t t0 = 0;
            for (uint32_t it = 0; !__all_sync(0xffffffffu, ld_acquire(a.cnt + SM_ARRIVE) >= (int)gridDim.x); ++it) {
                if ((it & 255u) != 255u) continue;   // reading the timer takes longer than a poll
                uint64_t now;
                asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(now));
                if (t0 == 0) t0 = now;
                if (__any_sync(0xffffffffu, now - t0 > a.wait_ns) || aborted()) {
                    give_up(22);
                    break;
                }
            }
            asm volatile("fence.proxy.async;" ::: "memory");
        };
        // a free stage, told what it will receive
        auto take = [&](int bytes) {
            if (issued >= STAGES && !warp_wait(empty + 8 * s, ph ^ 1, a.wait_ns)) {
                give_up(21);
                return false;
            }
            if (elect_one()) mbar_expect_tx(full + 8 * s, bytes);
            __syncwarp();
            return true;
        };
        auto next = [&]() {
            __syncwarp();
            ++issued;
            if (++s == STAGES) { s = 0; ph ^= 1u; }
        };
        {
            const SmPhase& q = a.ph[0];
            const int k0 = first_of(q, rank) * 64, k1 = first_of(q, rank + 1) * 64;
            for (int m = cl; m < q.tiles && k0 < k1 && !aborted(); m += ncl)
                for (int k = k0; k < k1 && take(2 * SM_BOX + S::B); k += 64) {
                    if (elect_one()) {
                        const uint32_t st = ring + (uint32_t)s * S::STAGE, bar = full + 8 * s;
                        tma_load_2d(st, &maps.gate, k, m * 64, bar);
                        tma_load_2d(st + SM_BOX, &maps.up, k, m * 64, bar);
                        tma_load_2d(st + 2 * SM_BOX, &maps.x, k, 0, bar);
                    }
                    next();
                }
        }
        if (!aborted()) {
            const SmPhase& q = a.ph[1];
            const int k0 = first_of(q, rank) * 128, k1 = first_of(q, rank + 1) * 128;
            // W_down's boxes, and the tokens' once h is there: until then the ring fills with the weights alone
            auto weights = [&](int m, int k) {
                const uint32_t st = ring + (uint32_t)s * S::STAGE, bar = full + 8 * s;
                if (!elect_one()) return;
                if (a.down_blocks) {
                    tma_load_3d(st, &maps.down, 0, m * 64, k / 64, bar);
                } else {
                    tma_load_2d(st, &maps.down, k, m * 64, bar);
                    tma_load_2d(st + SM_BOX, &maps.down, k + 64, m * 64, bar);
                }
            };
            auto tokens = [&](int at, int k) {
                const uint32_t st = ring + (uint32_t)at * S::STAGE + 2 * SM_BOX, bar = full + 8 * at;
                if (!elect_one()) return;
                if (a.down_blocks) {
                    tma_load_3d(st, &maps.h, 0, 0, k / 64, bar);
                } else {
                    tma_load_2d(st, &maps.h, k, 0, bar);
                    tma_load_2d(st + S::B, &maps.h, k + 64, 0, bar);
                }
            };
            const int s0 = s;
            int ahead = 0, m = cl, k = k0;
            for (; m < q.tiles && k0 < k1 && ahead < STAGES; ++ahead) {
                if (!take(2 * SM_BOX + 2 * S::B)) break;
                weights(m, k);
                next();
                if ((k += 128) == k1) { k = k0; m += ncl; }
            }
            if (ahead > 0) {
                if (!aborted()) wait_h();
                // (given up: loaded all the same, so that every stage begun is complete)
                for (int j = 0, at = s0, kt = k0; j < ahead; ++j) {
                    tokens(at, kt);
                    __syncwarp();
                    if (++at == STAGES) at = 0;
                    if ((kt += 128) == k1) kt = k0;
                }
            }
            for (; m < q.tiles && k0 < k1 && !aborted(); m += ncl, k = k0)
                for (; k < k1 && take(2 * SM_BOX + 2 * S::B); k += 128) {
                    weights(m, k);
                    __syncwarp();
                    tokens(s, k);
                    next();
                }
        }
        if (aborted()) {
            // a wait ran out: the copies in flight land before this memory is given back
            for (int q = 0; q < STAGES && q < issued; ++q) {
                if (--s < 0) { s = STAGES - 1; ph ^= 1u; }
                warp_wait(full + 8 * s, ph, a.wait_ns);
            }
        }
    } else if (warp == 1) {
        // ---------------- MMA issuer ----------------
        const uint32_t idesc = idesc_bf16(128, NT);
        int s = 0, seg = 0;
        uint32_t ph = 0;
        for (int f = 0; f < 2 && !aborted(); ++f) {
            const SmPhase& q = a.ph[f];
            const int n = first_of(q, rank + 1) - first_of(q, rank);
            for (int m = cl; m < q.tiles && n > 0 && !aborted(); m += ncl, ++seg) {
                const uint32_t d = tmem + (uint32_t)((seg & 1) * 2 * NT);
                if (seg >= 2 && !warp_wait(accempty + 8 * (seg & 1), (uint32_t)((seg >> 1) & 1) ^ 1u, a.wait_ns)) {
                    give_up(23);
                    break;
                }
                tc_fence_after();
                for (int kb = 0; kb < n; ++kb) {
                    if (!warp_wait(full + 8 * s, ph, a.wait_ns)) {
                        give_up(24);
                        break;
                    }
                    tc_fence_after();
                    const uint32_t sa = smem_u32(smem + s * S::STAGE), sb = sa + 2 * SM_BOX;
                    if (elect_one()) {
#pragma unroll
                        for (int kk = 0; kk < 4; ++kk) {
                            const uint32_t on = kb == 0 && kk == 0 ? 0u : 1u;
                            mma_bf16(d, sw128_desc(sa + kk * 32), sw128_desc(sb + kk * 32), idesc, on);
                            if (f) mma_bf16(d + NT, sw128_desc(sa + kk * 32), sw128_desc(sb + S::B + kk * 32), idesc, on);
                        }
                        mma_commit(empty + 8 * s);
                        if (kb + 1 == n) mma_commit(accfull + 8 * (seg & 1));
                    }
                    __syncwarp();
                    if (++s == STAGES) { s = 0; ph ^= 1u; }
                }
            }
        }
        // all MMAs are done before the ring and TMEM are given back
        if (elect_one()) mma_commit(drain);
        __syncwarp();
        if (!warp_wait(drain, 0, a.wait_ns)) give_up(25);
    } else {
        // ---------------- epilogue (warps 2..5) ----------------
        const int quarter = warp & 3;
        // this lane's row of a half (gate or up; the first or the second k-step) goes to CTA row / 16, into this CTA's part
        const int side = quarter >> 1, r64 = (quarter & 1) * 32 + lane;
        const uint32_t to = map_rank(smem_u32(recv_mem), (uint32_t)(r64 >> 4)) + (uint32_t)(rank * S::PART + side * RT * 16 + (r64 & 15)) * 4;
        const uint32_t to_bar = map_rank(recv, (uint32_t)(r64 >> 4));
        int seg = 0, round = 0;
        bool ok = true;
        // all four warps go on or none
        auto agree = [&](bool mine) {
            int all;
            asm volatile("{\n .reg .pred p, q;\n setp.ne.s32 p, %1, 0;\n bar.red.and.pred q, 2, 128, p;\n selp.s32 %0, 1, 0, q;\n}\n"
                         : "=r"(all) : "r"(mine && *(volatile int*)&s_abort == 0 ? 1 : 0) : "memory");
            return all != 0;
        };
        for (int f = 0; f < 2 && ok; ++f) {
            const SmPhase& q = a.ph[f];
            const bool part = first_of(q, rank) < first_of(q, rank + 1);   // this CTA has a part of every tile
            int parts = 0;
            for (int r = 0; r < SM_S; ++r) parts += first_of(q, r) < first_of(q, r + 1) ? 1 : 0;
            for (int m = cl; m < q.tiles && ok; m += ncl) {
                const uint32_t d = tmem + (uint32_t)((seg & 1) * 2 * NT + (f ? side * NT : 0)) + ((uint32_t)(quarter * 32) << 16);
                const bool done = !part || warp_wait(accfull + 8 * (seg & 1), (uint32_t)((seg >> 1) & 1), a.wait_ns);
                if (!done) give_up(26);
                if (!(ok = agree(done))) break;
                tc_fence_after();
                const int row = m * 64 + rank * 16 + (lane & 15);   // that this CTA finishes
                for (int t0 = 0; t0 < a.T && ok; t0 += RT, ++round) {
                    const int b = round & 1, nt = min(RT, a.T - t0);
                    if (part) {
                        const uint32_t dst = to + (uint32_t)(b * S::RECV), bar = to_bar + 8 * b;
#pragma unroll 1
                        for (int i = 0; i < nt; i += 16) {
                            float v[16];
                            tmem_ld16(d + t0 + i, v);
#pragma unroll
                            for (int e = 0; e < 16; ++e)
                                if (i + e < nt) send(dst + (uint32_t)(i + e) * 64, v[e], bar);
                        }
                        if (t0 + RT >= a.T) {   // the accumulator is read
                            tc_fence_before();
                            __syncwarp();
                            if (lane == 0) mbar_arrive(accempty + 8 * (seg & 1));
                        }
                    }
                    if (threadIdx.x == 64) mbar_expect_tx(recv + 8 * b, (uint32_t)(parts * nt * 2 * 16 * 4));
                    const bool got = warp_wait(recv + 8 * b, (uint32_t)((round >> 1) & 1), a.wait_ns);
                    if (!got) give_up(27);
                    const float* in = reinterpret_cast<const float*>(recv_mem + b * S::RECV);
                    for (int i = 2 * quarter + (lane >> 4); i < nt && got; i += 8) {
                        float v = 0.f, u = 0.f;
#pragma unroll
                        for (int r = 0; r < SM_S; ++r) {
                            if (first_of(q, r) == first_of(q, r + 1)) continue;
                            const float* at = in + r * S::PART + i * 16 + (lane & 15);
                            v += at[0];
                            u += at[RT * 16];
                        }
                        const int t = t0 + i;
                        if (f == 0 && row < a.F) {
                            float p, w, h;
                            mlp_factors<ACT, 1>(&v, &u, &p, &w, &h);
                            a.h[(int64_t)t * a.F + row] = f2bf(h);
                            if (a.pq) {
                                pq_put(a.pq, t, row, a.F, p);
                                pq_put(a.pq + a.q_off, t, row, a.F, w);
                            }
                        } else if (f == 1 && row < a.C) {
                            a.y[(int64_t)t * a.C + row] = f2bf(v + u);
                        }
                    }
                    // The buffer is read before any of these warps sends on.  With two buffers nothing more is
                    // needed: whoever sends round n + 2 has received n + 1, which every CTA sent after it read n.
                    ok = agree(got);
                }
                if (part) ++seg;
            }
            if (f == 0) {
                // this CTA's part of h is written (given up: counted all the same, the others need not wait long)
                asm volatile("fence.proxy.async;" ::: "memory");   // it will be read by TMA
                asm volatile("bar.sync 1, 128;" ::: "memory");
                if (threadIdx.x == 64) add_release(a.cnt + SM_ARRIVE);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();   // nothing is sent to a CTA that has ended
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::COLS) : "memory");
    }
    // the last CTA to leave clears the counters for the next launch
    if (threadIdx.x == 0 && atomicAdd(a.cnt + SM_LEAVE, 1) == (int)gridDim.x - 1) {
        a.cnt[SM_ARRIVE] = 0;
        a.cnt[SM_LEAVE] = 0;
    }
}

template <int NT, int ACT>
cudaError_t sm_launch(const SmMaps& maps, const SmArgs& a, cudaStream_t st) {
    static std::atomic<int> fit[64];   // clusters that a device holds at once, asked for once
    auto* k = k_mlp_small<NT, ACT>;
    cudaError_t e = smem_optin((const void*)k, SmShape<NT>::SMEM);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(device_sms() / SM_S * SM_S);
    cfg.blockDim = dim3(SM_NT);
    cfg.dynamicSmemBytes = SmShape<NT>::SMEM;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = SM_S;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeCooperative;   // the CTAs wait for one another
    at[1].val.cooperative = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    int dev = 0, n = 0;
    if ((e = cudaGetDevice(&dev)) != cudaSuccess) return e;
    const bool keep = dev >= 0 && dev < 64;
    if (!keep || (n = fit[dev].load(std::memory_order_relaxed)) < 1) {
        if ((e = cudaOccupancyMaxActiveClusters(&n, k, &cfg)) != cudaSuccess) return e;
        if (n < 1) return cudaErrorInvalidConfiguration;
        if (keep) fit[dev].store(n, std::memory_order_relaxed);
    }
    const int tiles = a.ph[0].tiles > a.ph[1].tiles ? a.ph[0].tiles : a.ph[1].tiles;
    cfg.gridDim = dim3(SM_S * (n < tiles ? n : tiles));
    cfg.numAttrs = 2;
    e = cudaLaunchKernelEx(&cfg, k, maps, a);
    note_launch();
    return e == cudaSuccess ? cudaGetLastError() : e;
}
template <int NT>
cudaError_t sm_launch_act(int act, const SmMaps& maps, const SmArgs& a, cudaStream_t st) {
    if (act == XHC_ACT_SILU) return sm_launch<NT, XHC_ACT_SILU>(maps, a, st);
    if (act == XHC_ACT_GELU) return sm_launch<NT, XHC_ACT_GELU>(maps, a, st);
    return sm_launch<NT, XHC_ACT_RELU>(maps, a, st);
}

}  // namespace

// Up to 64 tokens, 128 where the weights are 48 MB or more: us a call here / with the tiles of k_mlp.cu, captured,
// C = 4096, F = 11008: 51 / 117 at 1 token, 58 / 86 at 64, 72 / 88 at 128; C = 2048, F = 5632: 21 / 40 at 1, 31 / 38 at 65, 40 / 39
// at 128; C = 1024, F = 2816: 13 / 27 at 1, 20 / 21 at 64, 22 / 21 at 65; C = 264, F = 712: 8.5 / 12.3 at 1, 13 / 13 at 64.
bool mlp_small(int64_t T, int C, int F) { return T <= ((int64_t)C * F >= (int64_t)1 << 23 ? 128 : 64); }

cudaError_t launch_mlp_small(int T, int C, int F, int act, const uint16_t* x, const uint16_t* Wg, const uint16_t* Wu,
                             const uint16_t* Wd, uint16_t* h, void* pq, uint16_t* y, int* cnt, int* err, cudaStream_t st) {
    SmArgs a = {};
    a.T = T;
    a.C = C;
    a.F = F;
    a.ph[0] = {(C + 63) / 64, (F + 63) / 64};
    a.ph[1] = {(F + 127) / 128, (C + 63) / 64};
    a.cnt = cnt;
    a.h = h;
    a.y = y;
    a.pq = (unsigned char*)pq;
    a.q_off = (int64_t)mlp_pq_bytes(T, F);
    a.wait_ns = debug_wait_ns();
    a.err = err;
    const int NT = T <= 16 ? 16 : T <= 32 ? 32 : T <= 64 ? 64 : 128;
    SmMaps m;
    if (!make_map_box(&m.gate, Wg, C, F, 64, 64) || !make_map_box(&m.up, Wu, C, F, 64, 64) ||
        !make_map_box(&m.x, x, C, T, 64, NT))
        return cudaErrorInvalidValue;
    a.down_blocks = F % 64 == 0;
    if (a.down_blocks ? !map_blocks(&m.down, Wd, C, F, 64, 2) || !map_blocks(&m.h, h, T, F, NT, 2)
                      : !make_map_box(&m.down, Wd, F, C, 64, 64) || !make_map_box(&m.h, h, F, T, 64, NT))
        return cudaErrorInvalidValue;
    if (NT == 16) return sm_launch_act<16>(act, m, a, st);
    if (NT == 32) return sm_launch_act<32>(act, m, a, st);
    if (NT == 64) return sm_launch_act<64>(act, m, a, st);
    return sm_launch_act<128>(act, m, a, st);
}

}  // namespace xhc
