// The feed-forward block's forward for few tokens (a decode step), in one launch:
//   h = act(x W_gate^T) * (x W_up^T), then y = h W_down^T
// It is bound by reading the weights once, 6 C F bytes.  The weights are the MMA's A operand (128 rows of
// W_gate and of W_up, or of W_down, an M of 128 each), the tokens its N of 16 to 64: outputs transposed.
// Every SM streams an equal, contiguous share of the k-blocks of all weight tiles through a ring of about
// 200 KB, so that the bytes in flight do not depend on how the tiles fall.  A tile cut between CTAs leaves
// partial sums; at the product's end its CTAs wait for one another and each adds up its share of the tile's
// outputs, in the order of the CTAs.  (All of it by the last one to arrive: 24 tokens of C = 2048, F = 5632 took
// 199 us, as its loads were few at a time.)  The cut depends on C, F and the GPU alone: a token's
// bits do not depend on the other tokens or on their number.
// The second product needs all of h: the CTAs (one an SM, launched cooperatively, so all are there) meet at a
// counter.  Loads of W_down do not need h and fill the ring before that wait, so the stream of weights
// does not stop between the products.
#include <type_traits>

#include "k_mlp.cuh"

namespace xhc {

namespace {

constexpr int SM_NT = 192;                   // warp 0 TMA, warp 1 MMA, warps 2..5 epilogue
constexpr int SM_A = 128 * 64 * 2;           // a box of 128 weight rows and 64 k-elements; two a stage
constexpr int SM_CNT2 = 512;                 // first counter of the second product's tiles
constexpr int SM_ARRIVE = 640, SM_LEAVE = 641;
constexpr int SM_LEAST = 4;

template <int NT>
struct SmShape {
    static constexpr int B = NT * 64 * 2, STAGE = 2 * SM_A + 2 * B;
    static constexpr int STAGES = NT == 16 ? 6 : NT == 32 ? 5 : 4;
    static constexpr int SMEM = STAGES * STAGE + (2 * STAGES + 5) * 8 + 16 + 1024;
    static constexpr uint32_t COLS = 4 * NT;   // two accumulators of gate and up columns
};

// One of the two products as a stream of units (a stage each): unit g is k-step g % kb of weight tile g / kb;
// CTA c < P takes units [start(c), start(c + 1)).  Either s CTAs share each tile (P = s tiles), or (s = 0) the
// stream is cut into P equal parts wherever they fall.  (At most 512 tiles of 256 steps, 304 SMs.)
struct SmPhase {
    int kb, tiles, P, s;
    int per, more;   // s = 0: the first `more` CTAs take per + 1 units, the others per
    __device__ int start(int c) const {
        if (s == 0) return c * per + min(c, more);
        const int m = c / s;
        return m * kb + (c - m * s) * kb / s;
    }
    __device__ int owner(int g) const { return g < more * (per + 1) ? g / (per + 1) : more + (g - more * (per + 1)) / per; }
    // the first and the last CTA that have a part of tile m
    __device__ int first(int m) const { return s ? m * s : owner(m * kb); }
    __device__ int last(int m) const { return s ? m * s + s - 1 : owner(m * kb + kb - 1); }
};
struct SmMaps {
    CUtensorMap gate, up, down, x, h;
};
struct SmArgs {
    int T, C, F;
    SmPhase ph[2];
    float* part;           // [CTA][2][gate, up][T][128]
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
__device__ __forceinline__ float4 ld_l2(const float* p) {   // written by other SMs in this launch
    float4 v;
    asm volatile("ld.global.cg.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "l"(p));
    return v;
}

template <int NT, int ACT>
__global__ void __launch_bounds__(SM_NT, 1) k_mlp_small(const __grid_constant__ SmMaps maps, const __grid_constant__ SmArgs a) {
    using S = SmShape<NT>;
    constexpr int STAGES = S::STAGES;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + STAGES * S::STAGE);
    const uint32_t full = smem_u32(bars), empty = full + 8 * STAGES, accfull = empty + 8 * STAGES, accempty = accfull + 16,
                   drain = accempty + 16;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * STAGES + 5);
    __shared__ int s_abort;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = blockIdx.x;
    if (threadIdx.x == 0) {
        s_abort = 0;
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(full + 8 * s, 1);
            mbar_init(empty + 8 * s, 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(accfull + 8 * s, 1);
            mbar_init(accempty + 8 * s, 4);
        }
        mbar_init(drain, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(S::COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    if (threadIdx.x == 32) {
        for (const CUtensorMap* m : {&maps.gate, &maps.up, &maps.x, &maps.down, &maps.h})
            asm volatile("prefetch.tensormap [%0];" ::"l"((uint64_t)m) : "memory");
    }
    pdl_entry();

    auto give_up = [&](int code) {
        atomicExch(a.err, code);
        *(volatile int*)&s_abort = 1;
    };
    auto aborted = [&]() { return *(volatile int*)&s_abort != 0; };

    // waits until a counter reaches n
    auto wait_count = [&](const int* cnt, int n, int code) {
        uint64_t t0 = 0;
        for (uint32_t it = 0; ld_acquire(cnt) < n; ++it) {
            if ((it & 255u) != 255u) continue;   // reading the timer takes longer than a poll
            uint64_t now;
            asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(now));
            if (t0 == 0) t0 = now;
            if (now - t0 > a.wait_ns || aborted()) {
                give_up(code);
                return;
            }
        }
    };

    if (warp == 0) {
        // ---------------- TMA producer ----------------
        if (lane == 0) {
            int s = 0, issued = 0;
            uint32_t ph = 0;
            // the weights of unit g, or its tokens, into stage st
            auto load = [&](int f, int g, int st, bool weights) {
                const SmPhase& q = a.ph[f];
                const int m = g / q.kb * 128, kb = g % q.kb;
                const uint32_t sa = smem_u32(smem + st * S::STAGE), sb = sa + 2 * SM_A, bar = full + 8 * st;
                if (f == 0) {
                    if (weights) {
                        tma_load_2d(sa, &maps.gate, kb * 64, m, bar);
                        tma_load_2d(sa + SM_A, &maps.up, kb * 64, m, bar);
                    } else {
                        tma_load_2d(sb, &maps.x, kb * 64, 0, bar);
                    }
                } else if (weights) {
                    tma_load_2d(sa, &maps.down, kb * 128, m, bar);
                    tma_load_2d(sa + SM_A, &maps.down, kb * 128 + 64, m, bar);
                } else {
                    tma_load_2d(sb, &maps.h, kb * 128, 0, bar);
                    tma_load_2d(sb + S::B, &maps.h, kb * 128 + 64, 0, bar);
                }
            };
            for (int f = 0; f < 2 && !aborted(); ++f) {
                const SmPhase& q = a.ph[f];
                int g = c < q.P ? q.start(c) : 0;
                const int g1 = c < q.P ? q.start(c + 1) : 0;
                int ahead = 0;   // stages of the second product whose tokens are still to come
                const int s0 = s;
                for (int gw = g; gw < g1 && !aborted(); ++gw) {
                    if (issued >= STAGES && !mbar_wait(empty + 8 * s, ph ^ 1, a.wait_ns)) {
                        give_up(21);
                        break;
                    }
                    if (aborted()) break;
                    mbar_expect_tx(full + 8 * s, 2 * SM_A + (f ? 2 : 1) * S::B);
                    load(f, gw, s, true);
                    if (f == 0) {
                        load(f, gw, s, false);
                    } else if (ahead >= 0) {
                        ++ahead;
                        if (ahead == STAGES || gw + 1 == g1) {
                            // h is whole when every CTA has finished the first product
                            wait_count(a.cnt + SM_ARRIVE, (int)gridDim.x, 22);
                            // (given up: the tokens are loaded all the same, so that every stage begun is complete)
                            asm volatile("fence.proxy.async;" ::: "memory");
                            for (int j = 0, st = s0; j < ahead; ++j) {
                                load(1, g + j, st, false);
                                if (++st == STAGES) st = 0;
                            }
                            ahead = -1;
                        }
                    } else {
                        load(f, gw, s, false);
                    }
                    ++issued;
                    if (++s == STAGES) { s = 0; ph ^= 1u; }
                }
                if (aborted())   // stages whose tokens will not come any more
                    for (int j = 0, st = s0; j < ahead; ++j) {
                        load(1, g + j, st, false);
                        if (++st == STAGES) st = 0;
                    }
            }
            if (aborted()) {
                // a wait ran out: the copies in flight land before this memory is given back
                for (int q = 0; q < STAGES && q < issued; ++q) {
                    if (--s < 0) { s = STAGES - 1; ph ^= 1u; }
                    mbar_wait(full + 8 * s, ph, a.wait_ns);
                }
            }
        }
    } else if (warp == 1) {
        // ---------------- MMA issuer ----------------
        if (lane == 0) {
            const uint32_t idesc = idesc_bf16(128, NT);
            int s = 0, seg = 0;
            uint32_t ph = 0;
            for (int f = 0; f < 2 && !aborted(); ++f) {
                const SmPhase& q = a.ph[f];
                const int g1 = c < q.P ? q.start(c + 1) : 0;
                for (int g = c < q.P ? q.start(c) : 0; g < g1 && !aborted(); ++seg) {
                    const int end = min(g1, (g / q.kb + 1) * q.kb);
                    const uint32_t d = tmem + (uint32_t)((seg & 1) * 2 * NT);
                    if (seg >= 2 && !mbar_wait(accempty + 8 * (seg & 1), (uint32_t)((seg >> 1) & 1) ^ 1u, a.wait_ns)) {
                        give_up(23);
                        break;
                    }
                    tc_fence_after();
                    for (bool first = true; g < end; ++g, first = false) {
                        if (!mbar_wait(full + 8 * s, ph, a.wait_ns)) {
                            give_up(24);
                            break;
                        }
                        tc_fence_after();
                        const uint32_t sa = smem_u32(smem + s * S::STAGE), sb = sa + 2 * SM_A;
#pragma unroll
                        for (int kk = 0; kk < 4; ++kk) {
                            const uint32_t on = first && kk == 0 ? 0u : 1u;
                            mma_bf16(d, sw128_desc(sa + kk * 32), sw128_desc(sb + kk * 32), idesc, on);
                            if (f == 0) mma_bf16(d + NT, sw128_desc(sa + SM_A + kk * 32), sw128_desc(sb + kk * 32), idesc, on);
                            else mma_bf16(d, sw128_desc(sa + SM_A + kk * 32), sw128_desc(sb + S::B + kk * 32), idesc, 1u);
                        }
                        mma_commit(empty + 8 * s);
                        if (++s == STAGES) { s = 0; ph ^= 1u; }
                    }
                    if (aborted()) break;
                    mma_commit(accfull + 8 * (seg & 1));
                }
            }
            // all MMAs are done before the ring and TMEM are given back
            mma_commit(drain);
            if (!mbar_wait(drain, 0, a.wait_ns)) give_up(25);
        }
    } else {
        // ---------------- epilogue (warps 2..5) ----------------
        const int quarter = warp & 3, r = quarter * 32 + lane;   // weight row within the tile
        auto meet = [&]() { asm volatile("bar.sync 1, 128;" ::: "memory"); };
        // the final values of n (1 or 4) neighbouring outputs of token t, from `row` on: gate and up, or the output
        auto finish = [&](auto count, int f, int row, int t, float* v, float* u) {
            constexpr int n = decltype(count)::value;
            if (f == 0) {
                float p[n], q[n], h[n];
                mlp_factors<ACT, n>(v, u, p, q, h);
                if (n == 1) a.h[(int64_t)t * a.F + row] = f2bf(h[0]);
                else *reinterpret_cast<uint2*>(a.h + (int64_t)t * a.F + row) = make_uint2(pack2(h[0], h[1 % n]), pack2(h[2 % n], h[3 % n]));
                if (a.pq)
#pragma unroll
                    for (int e = 0; e < n; ++e) {
                        pq_put(a.pq, t, row + e, a.F, p[e]);
                        pq_put(a.pq + a.q_off, t, row + e, a.F, q[e]);
                    }
            } else if (n == 1) {
                a.y[(int64_t)t * a.C + row] = f2bf(v[0]);
            } else {
                *reinterpret_cast<uint2*>(a.y + (int64_t)t * a.C + row) = make_uint2(pack2(v[0], v[1 % n]), pack2(v[2 % n], v[3 % n]));
            }
        };
        int seg = 0;
        bool ok = true;
        for (int f = 0; f < 2 && ok; ++f) {
            const SmPhase& q = a.ph[f];
            const int g0 = c < q.P ? q.start(c) : 0, g1 = c < q.P ? q.start(c + 1) : 0;
            for (int g = g0; g < g1; ++seg) {
                const int m = g / q.kb, row = m * 128 + r;
                const int end = min(g1, (m + 1) * q.kb);
                const bool whole = end - g == q.kb, mine = row < (f ? a.C : a.F);
                const uint32_t d = tmem + (uint32_t)((seg & 1) * 2 * NT) + ((uint32_t)(quarter * 32) << 16);
                // all four warps go on or none: they meet below
                bool got = mbar_wait(accfull + 8 * (seg & 1), (uint32_t)((seg >> 1) & 1), a.wait_ns);
                int all;
                asm volatile("{\n .reg .pred p, q;\n setp.ne.s32 p, %1, 0;\n bar.red.and.pred q, 2, 128, p;\n selp.s32 %0, 1, 0, q;\n}\n"
                             : "=r"(all) : "r"(got && !aborted() ? 1 : 0) : "memory");
                if (!all) {
                    if (threadIdx.x == 64) give_up(26);
                    ok = false;
                    break;
                }
                tc_fence_after();
                float* mypart = a.part + ((int64_t)(c * 2 + (g == g0 ? 0 : 1)) * 2 * a.T) * 128 + r;
#pragma unroll 1
                for (int t0 = 0; t0 < a.T; t0 += 16) {
                    float v[16], u[16];
                    tmem_ld16(d + t0, v);
                    if (f == 0) tmem_ld16(d + NT + t0, u);
                    const int nt = min(16, a.T - t0);
                    if (whole) {
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            if (e < nt && mine) finish(std::integral_constant<int, 1>{}, f, row, t0 + e, v + e, u + e);
                    } else {
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            if (e < nt) {
                                mypart[(t0 + e) * 128] = v[e];
                                if (f == 0) mypart[(a.T + t0 + e) * 128] = u[e];
                            }
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(accempty + 8 * (seg & 1));
                if (!whole) {   // a part is left
                    meet();
                    if (threadIdx.x == 64) add_release(a.cnt + (f ? SM_CNT2 : 0) + m);
                }
                g = end;
            }
            // this CTA's share of the tiles that it has a part of: the first one and the last one it took
            for (int side = 0; side < 2 && ok && g0 < g1; ++side) {
                const int m = (side ? g1 - 1 : g0) / q.kb;
                const int b0 = m * q.kb, b1 = b0 + q.kb;
                if ((b0 >= g0 && b1 <= g1) || (side && g0 >= b0)) continue;   // whole, or done as the first one
                const int ca = q.first(m), n = q.last(m) - ca + 1;
                if (threadIdx.x == 64) wait_count(a.cnt + (f ? SM_CNT2 : 0) + m, n, 27);
                meet();
                const bool late = q.start(ca) < b0;   // the first of them began in the tile before: its second part
                // 4 rows of a token a slot; U slots of a thread at a time, for their loads to be in flight together
                constexpr int U = 4;
                const int slots = a.T * 32, o1 = slots * (c - ca + 1) / n, rows = f ? a.C : a.F;
                for (int o0 = slots * (c - ca) / n + (int)threadIdx.x - 64; o0 < o1; o0 += 128 * U) {
                    float v[U][4], u[U][4];
#pragma unroll
                    for (int j = 0; j < U; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[j][e] = u[j][e] = 0.f;
#pragma unroll 2
                    for (int k = ca; k < ca + n; ++k) {
                        const float* pt = a.part + (int64_t)(k * 2 + (late && k == ca ? 1 : 0)) * 2 * a.T * 128;
#pragma unroll
                        for (int j = 0; j < U; ++j) {
                            const int o = o0 + 128 * j;   // slot o's rows lie at 4 o
                            if (o >= o1) continue;
                            const float4 x = ld_l2(pt + o * 4);
                            v[j][0] += x.x; v[j][1] += x.y; v[j][2] += x.z; v[j][3] += x.w;
                            if (f == 0) {
                                const float4 z = ld_l2(pt + a.T * 128 + o * 4);
                                u[j][0] += z.x; u[j][1] += z.y; u[j][2] += z.z; u[j][3] += z.w;
                            }
                        }
                    }
#pragma unroll
                    for (int j = 0; j < U; ++j) {
                        const int o = o0 + 128 * j, row = m * 128 + (o & 31) * 4;
                        if (o < o1 && row < rows) finish(std::integral_constant<int, 4>{}, f, row, o >> 5, v[j], u[j]);
                    }
                }
            }
            if (f == 0) {
                // this CTA's part of h is written (given up: counted all the same, the others need not wait long)
                asm volatile("fence.proxy.async;" ::: "memory");   // it will be read by TMA
                meet();
                if (threadIdx.x == 64) add_release(a.cnt + SM_ARRIVE);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::COLS) : "memory");
    }
    // the last CTA to leave clears the counters for the next launch
    __shared__ int s_last;
    if (threadIdx.x == 0) s_last = atomicAdd(a.cnt + SM_LEAVE, 1) == (int)gridDim.x - 1;
    __syncthreads();
    if (s_last)
        for (int q = threadIdx.x; q < MLP_COUNTERS; q += SM_NT) a.cnt[q] = 0;
}

// Where whole CTAs of tiles nearly fill the GPU, a tile's CTAs share it evenly and each waits for one tile's parts
// only; else the stream is cut evenly.  A CTA takes SM_LEAST units at least: a part costs about as much as
// those (its sums leave and come back through L2, between two waits).
SmPhase sm_phase(int rows, int kb, int sms) {
    SmPhase p = {};
    p.kb = kb;
    p.tiles = (rows + 127) / 128;
    const int units = kb * p.tiles, cap = (kb + SM_LEAST - 1) / SM_LEAST;
    int s = sms / p.tiles;
    if (s > cap) s = cap;
    if (s >= 1 && (s == cap || 100 * s * p.tiles >= 85 * sms)) {
        p.s = s;
        p.P = s * p.tiles;
        return p;
    }
    p.P = units < sms ? units : sms;
    p.per = units / p.P;
    p.more = units - p.per * p.P;
    return p;
}

template <int NT, int ACT>
cudaError_t sm_launch(const SmMaps& maps, const SmArgs& a, cudaStream_t st) {
    auto* k = k_mlp_small<NT, ACT>;
    cudaError_t e = smem_optin((const void*)k, SmShape<NT>::SMEM);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(a.ph[0].P > a.ph[1].P ? a.ph[0].P : a.ph[1].P);
    cfg.blockDim = dim3(SM_NT);
    cfg.dynamicSmemBytes = SmShape<NT>::SMEM;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeCooperative;   // the CTAs wait for one another
    at[0].val.cooperative = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
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

// Up to 64 tokens where the weights are 12 MB or more, 16 where they are less: us a call here / with the tiles
// of k_mlp.cu, C = 4096, F = 11008: 80 / 104 at 64 tokens, 105 / 104 at 128; C = 1024, F = 2816: 17.6 / 29.7 at 1, 25.4 /
// 25.3 at 64; C = 264, F = 712: 13.4 / 13.3 at 1, 14.4 / 13.5 at 16, 21.3 / 13.8 at 64.
bool mlp_small(int64_t T, int C, int F) { return T <= ((int64_t)C * F >= (int64_t)1 << 21 ? 64 : 16); }

size_t mlp_small_part_bytes(int64_t T, int C, int F) {
    return mlp_small(T, C, F) ? (size_t)device_sms() * 2 * 2 * T * 128 * 4 : 0;
}

cudaError_t launch_mlp_small(int T, int C, int F, int act, const uint16_t* x, const uint16_t* Wg, const uint16_t* Wu,
                             const uint16_t* Wd, uint16_t* h, void* pq, uint16_t* y, float* part, int* cnt, int* err,
                             cudaStream_t st) {
    SmArgs a = {};
    a.T = T;
    a.C = C;
    a.F = F;
    a.ph[0] = sm_phase(F, (C + 63) / 64, device_sms());
    a.ph[1] = sm_phase(C, (F + 127) / 128, device_sms());
    a.part = part;
    a.cnt = cnt;
    a.h = h;
    a.y = y;
    a.pq = (unsigned char*)pq;
    a.q_off = (int64_t)mlp_pq_bytes(T, F);
    a.wait_ns = debug_wait_ns();
    a.err = err;
    const int NT = T <= 16 ? 16 : T <= 32 ? 32 : 64;
    SmMaps m;
    if (!make_map_box(&m.gate, Wg, C, F, 64, 128) || !make_map_box(&m.up, Wu, C, F, 64, 128) ||
        !make_map_box(&m.down, Wd, F, C, 64, 128) || !make_map_box(&m.x, x, C, T, 64, NT) || !make_map_box(&m.h, h, F, T, 64, NT))
        return cudaErrorInvalidValue;
    if (NT == 16) return sm_launch_act<16>(act, m, a, st);
    if (NT == 32) return sm_launch_act<32>(act, m, a, st);
    return sm_launch_act<64>(act, m, a, st);
}

}  // namespace xhc
