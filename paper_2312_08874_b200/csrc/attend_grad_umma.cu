// Gradient of softmax attention over whole sequences, 16-bit types, on the 5th-generation tensor cores.
//
// Two kernels of one form, so that every sum has one owner (no reductions in global memory; the same bits from call to call) at the price of making the
// logits twice (seven products a pair of tiles instead of five):
//   KEYS   a block owns 128 keys of a head and walks the tiles of 128 queries, of every head of the group, that see them:
//          S' = K Q^T, dP' = V dO^T, dV += P' dO, dK += dS' Q
//   else   it owns 128 queries and walks their keys:  S = Q K^T, dP = dO V^T, dQ += dS K
// Roles:
//   warps 0-7   a row and half of a tile's columns a thread: P = exp2(scale S - lse), dS = P (dP - D), both back to tensor memory in place of what they are made
//               of, as A operands.  The exponentials of one tile run beside the products of the other numbers of the tile before.
//   warp 8      issues the products
//   warp 9      TMA: the block's own rows once, then the columns' two operands
//   warp 10     rows behind a sequence become zero (they meet zeros in the sums, and need not be finite); KEYS: the queries' statistics
#include "attend_umma.cuh"

namespace aa {

namespace {

struct GradArgs {
    AttendArgs a;
    unsigned slots;
    RowMap q, k, v, dout;
};

constexpr int OFF_DEAD = 256, OFF_TMEM = 260, kThreads = 384;
template <int BOXES> struct GradUmma {
    static constexpr int kStages = BOXES == 1 ? 3 : 2, kOperand = BOXES * kTileBytes;
    static constexpr int OFF_X = 1024, OFF_RING = OFF_X + 2 * kOperand, OFF_STAT = OFF_RING + kStages * 2 * kOperand, kSmem = OFF_STAT + kStages * 2 * kTileRows * 4 + 1024;
    static_assert(kSmem <= 232448, "shared memory");
    // mbarriers                        count            waiter
    static constexpr int BAR_X = 0,  // tx               issuer
        BAR_FULL = 1,                // [stages] tx      warp 10
        BAR_READY = BAR_FULL + kStages,      // [stages] warp 10   issuer, row warps
        BAR_FREE = BAR_READY + kStages,      // [stages] commit    producer, warp 10
        BAR_S = BAR_FREE + kStages,          // [2] commit         row warps
        BAR_T = BAR_S + 2,                   // commit             row warps
        BAR_P = BAR_T + 1,                   // row warps          issuer
        BAR_DS = BAR_P + 1,                  // row warps          issuer
        BAR_ACC = BAR_DS + 1,                // [2] commit         issuer, row warps at the end
        BAR_DRAIN = BAR_ACC + 2, kBars = BAR_DRAIN + 1;
    static_assert(8 * kBars <= OFF_DEAD, "mbarriers");
};
// tensor memory columns.  KEYS: S', dP', dV, dK; else S (twice), dP, dQ
constexpr uint32_t kCols = 128;

template <typename T, int BOXES, bool KEYS>
__global__ void __launch_bounds__(kThreads, 1) attend_grad_umma_kernel(const __grid_constant__ GradArgs u) {
    using G = GradUmma<BOXES>;
    constexpr int kStages = G::kStages, kFmt = Elem<T>::kIsBf16 ? 1 : 0;
    constexpr uint32_t TM_T = KEYS ? kCols : 2 * kCols, TM_V = 2 * kCols, TM_A = 3 * kCols;
    const AttendArgs& a = u.a;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const uint32_t base = smem_u32(smem);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int group = a.heads / a.kv_heads, wide = KEYS ? a.kv_heads : a.heads, mine = blockIdx.x % wide, hk = KEYS ? mine : mine / group;
    const unsigned slot = blockIdx.x / wide;
    int seq, tile;
    // (causal: the first keys, which most see, and the last queries, which see most, come first)
    if (!find_slot(KEYS ? a.k_offsets : a.q_offsets, a.sequences, KEYS ? a.M : a.N, 1, kTileRows, !KEYS && a.causal ? u.slots - 1 - slot : slot, &seq, &tile)) return;
    const Span q = span_of(a.q_offsets, a.q_lengths, a.N, seq), k = span_of(a.k_offsets, a.k_lengths, a.M, seq);
    const int rows = KEYS ? k.count : q.count, r0 = tile * kTileRows;
    if (r0 >= rows) return;
    // tiles of columns: `per` of every head, from `first` on
    const int ahead = k.count - q.count;                            // query i sees the keys up to i + ahead
    int first = 0, per;
    if (KEYS) {
        if (a.causal) first = max(0, r0 - ahead) / kTileRows;
        per = max(0, (q.count + kTileRows - 1) / kTileRows - first);
    } else {
        per = (visible_keys(a.causal, min(rows, r0 + kTileRows) - 1, q.count, k.count) + kTileRows - 1) / kTileRows;
    }
    const int total = KEYS ? per * group : per, steps = (a.d + 15) / 16;
    const Span x = KEYS ? k : q, y = KEYS ? q : k;                  // rows, columns

    Pipe pp;
    pp.status = a.status;
    pp.dead = reinterpret_cast<int*>(smem + OFF_DEAD);
    pp.bars = base;
    if (tid == 0) {
        *pp.dead = 0;
        for (int i = 0; i < G::kBars; ++i) mbar_init(pp.bars + 8 * i, i == G::BAR_P || i == G::BAR_DS ? 8u : 1u);
        mbar_fence_init();
    }
    if (warp == 8) tmem_alloc<512>(base + OFF_TMEM);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    pp.tmem = *reinterpret_cast<const volatile uint32_t*>(smem + OFF_TMEM);
    float* stats = reinterpret_cast<float*>(smem + G::OFF_STAT);   // [stages][lse | D][128]
    const float kappa_seq = KEYS && is_f16<T> ? grad_factor(__uint_as_float(grad_most(a, seq, hk)[0]), __uint_as_float(grad_most(a, seq, hk)[1])) : 1.f;

    if (warp == 9) {
        // ------------------------------------------------------------------ producer
        if (lane == 0 && total) {
            mbar_arrive_expect_tx(pipe_bar(pp, G::BAR_X), 2 * G::kOperand);
            for (int b = 0; b < BOXES; ++b) {
                load_rows(base + G::OFF_X + b * kTileBytes, KEYS ? u.k : u.q, 64 * b, x.first + r0, mine, x.batch, pipe_bar(pp, G::BAR_X));
                load_rows(base + G::OFF_X + G::kOperand + b * kTileBytes, KEYS ? u.v : u.dout, 64 * b, x.first + r0, mine, x.batch, pipe_bar(pp, G::BAR_X));
            }
            int t = 0, head = hk * group;
            for (int j = 0; j < total && !pipe_dead(pp); ++j) {
                const int s = j % kStages, row = y.first + (first + t) * kTileRows;
                if (j >= kStages) wait_spin(pp, G::BAR_FREE + s, j / kStages - 1, kAttendTimeout);
                const uint32_t bar = pipe_bar(pp, G::BAR_FULL + s), dst = base + G::OFF_RING + s * 2 * G::kOperand;
                mbar_arrive_expect_tx(bar, 2 * G::kOperand);
                for (int b = 0; b < BOXES; ++b) {
                    load_rows(dst + b * kTileBytes, KEYS ? u.q : u.k, 64 * b, row, KEYS ? head : hk, y.batch, bar);
                    load_rows(dst + G::kOperand + b * kTileBytes, KEYS ? u.dout : u.v, 64 * b, row, KEYS ? head : hk, y.batch, bar);
                }
                if (++t == per) { t = 0; ++head; }
            }
        }
        __syncwarp();
    } else if (warp == 10) {
        // ------------------------------------------------------------------ rows behind the sequence; statistics of the columns
        int t = 0, head = hk * group;
        for (int j = 0; j < total && !pipe_dead(pp); ++j) {
            const int s = j % kStages, c0 = (first + t) * kTileRows, left = y.count - c0;
            if (KEYS) {
                if (j >= kStages) wait_spin(pp, G::BAR_FREE + s, j / kStages - 1, kAttendTimeout);
                const float2* st = reinterpret_cast<const float2*>(a.ws) + ((long long)q.batch * a.heads + head) * a.N + q.first + c0;
                float* to = stats + s * 2 * kTileRows;
#pragma unroll
                for (int i = 0; i < kTileRows / 32; ++i) {
                    const int c = 32 * i + lane;
                    // (a column that is none: a probability of zero)
                    const float2 v = c < left ? __ldg(st + c) : make_float2(INFINITY, 0.f);
                    to[c] = v.x - (is_f16<T> ? kHeldP : 0.f);
                    to[kTileRows + c] = v.y * kappa_seq;
                }
            }
            wait_spin(pp, G::BAR_FULL + s, j / kStages, kAttendTimeout);
            if (left < kTileRows) {
                clear_rows(base + G::OFF_RING + s * 2 * G::kOperand, BOXES, left, lane);
                clear_rows(base + G::OFF_RING + s * 2 * G::kOperand + G::kOperand, BOXES, left, lane);
                fence_proxy_async();
            }
            __syncwarp();
            if (lane == 0) pipe_arrive(pp, G::BAR_READY + s);
            if (++t == per) { t = 0; ++head; }
        }
        __syncwarp();
    } else if (warp == 8) {
        // ------------------------------------------------------------------ products
        const uint32_t id_s = umma_idesc(kFmt, 128, 128, 0), id_a = umma_idesc(kFmt, 128, steps * 16, 1), elected = elect_lane();
        auto ring = [&](int j, int which) { return base + G::OFF_RING + (j % kStages) * 2 * G::kOperand + which * G::kOperand; };
        auto logits = [&](int j) {
            wait_spin(pp, G::BAR_READY + j % kStages, j / kStages, kAttendTimeout);
            tc_fence_after_sync();
            mma_rows<BOXES>(elected, pp.tmem + (KEYS ? 0 : (j & 1) * kCols), base + G::OFF_X, ring(j, 0), id_s, steps);
            umma_commit_e<false>(elected, pipe_bar(pp, G::BAR_S + (KEYS ? 0 : j & 1)));
        };
        auto slopes = [&](int j) {
            mma_rows<BOXES>(elected, pp.tmem + TM_T, base + G::OFF_X + G::kOperand, ring(j, 1), id_s, steps);
            umma_commit_e<false>(elected, pipe_bar(pp, G::BAR_T));
        };
        auto sums = [&](uint32_t acc, uint32_t operand, int j, int which) { mma_sum<BOXES>(elected, acc, operand, operand + 64, ring(j, which), id_a, j > 0); };
        if (total) {
            wait_spin(pp, G::BAR_X, 0, kAttendTimeout);
            logits(0);
            slopes(0);
        }
        for (int j = 0; j < total && !pipe_dead(pp); ++j) {
            if (KEYS) {
                wait_spin(pp, G::BAR_P, j, kAttendTimeout);
                tc_fence_after_sync();
                sums(pp.tmem + TM_V, pp.tmem, j, 1);
                umma_commit_e<false>(elected, pipe_bar(pp, G::BAR_ACC));
                if (j + 1 < total) {
                    wait_spin(pp, G::BAR_ACC, j, kAttendTimeout);            // (the next logits take the place of the probabilities)
                    logits(j + 1);
                }
            } else if (j + 1 < total) {
                logits(j + 1);                                               // (the logits two tiles ago have been read: dS of the tile before is there)
            }
            wait_spin(pp, G::BAR_DS, j, kAttendTimeout);
            tc_fence_after_sync();
            sums(pp.tmem + TM_A, pp.tmem + TM_T, j, 0);
            umma_commit_e<false>(elected, pipe_bar(pp, G::BAR_FREE + j % kStages));
            umma_commit_e<false>(elected, pipe_bar(pp, G::BAR_ACC + 1));
            if (j + 1 < total) {
                wait_spin(pp, G::BAR_ACC + 1, j, kAttendTimeout);
                tc_fence_after_sync();
                slopes(j + 1);
            }
        }
        umma_drain_w(pp, G::BAR_DRAIN);
        __syncwarp();
    } else if (warp < 8) {
        // ------------------------------------------------------------------ P and dS
        const int w = warp >> 2, local = 32 * (warp & 3) + lane, row = r0 + local;
        const uint32_t lanes = ((uint32_t)(32 * (warp & 3)) << 16) + 64 * w;       // (this thread's row, and the first of its columns)
        const float c1 = a.scale * kLog2e;
        float lse = 0.f, dot = 0.f, kappa = kappa_seq;
        int limit = 0;                             // rows are queries: keys that this one sees; keys: the first query that sees it
        if (KEYS) {
            limit = a.causal ? row - ahead : 0;
        } else if (row < rows) {
            const long long at = ((long long)q.batch * a.heads + mine) * a.N + q.first + row;
            const float2 st = __ldg(reinterpret_cast<const float2*>(a.ws) + at);
            if (is_f16<T>) kappa = grad_factor(grad_norms(a)[at], __uint_as_float(grad_most(a, seq, hk)[1]));
            lse = st.x - (is_f16<T> ? kHeldP : 0.f);
            dot = st.y * kappa;
            limit = visible_keys(a.causal, row, q.count, k.count);
        }
        int t = 0;
        for (int j = 0; j < total; ++j) {
            const int s = j % kStages, c0 = (first + t) * kTileRows;
            if (++t == per) t = 0;
            const bool masked = KEYS ? c0 + kTileRows > q.count || (a.causal && c0 < r0 + kTileRows - 1 - ahead)
                                     : c0 + kTileRows > visible_keys(a.causal, r0, q.count, k.count);
            const float4* st = reinterpret_cast<const float4*>(stats + s * 2 * kTileRows + 64 * w);
            if (KEYS) wait_soon(pp, G::BAR_READY + s, j / kStages);
            wait_soon(pp, G::BAR_S + (KEYS ? 0 : j & 1), KEYS ? j : j >> 1);
            tc_fence_after_sync();
            const uint32_t ts = pp.tmem + (KEYS ? 0 : (j & 1) * kCols) + lanes, tt = pp.tmem + TM_T + lanes;
            float2 p[32];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t o[32];
                tmem_ld32(ts + 32 * h, o);
                tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    float4 l = make_float4(lse, lse, lse, lse);
                    if (KEYS) l = st[8 * h + i];
                    const float2 e0 = ffma2(make_float2(__uint_as_float(o[4 * i]), __uint_as_float(o[4 * i + 1])), make_float2(c1, c1), make_float2(-l.x, -l.y));
                    const float2 e1 = ffma2(make_float2(__uint_as_float(o[4 * i + 2]), __uint_as_float(o[4 * i + 3])), make_float2(c1, c1), make_float2(-l.z, -l.w));
                    p[16 * h + 2 * i] = make_float2(fast_exp2(e0.x), fast_exp2(e0.y));
                    p[16 * h + 2 * i + 1] = make_float2(fast_exp2(e1.x), fast_exp2(e1.y));
                }
            }
            if (masked) {
                const int at = c0 + 64 * w;
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    const int c = at + 2 * i;
                    if (KEYS ? c < limit || c >= q.count : c >= limit) p[i].x = 0.f;
                    if (KEYS ? c + 1 < limit || c + 1 >= q.count : c + 1 >= limit) p[i].y = 0.f;
                }
            }
            if (KEYS) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t o[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[i] = pack2<T>(p[16 * h + i].x, p[16 * h + i].y);
                    tmem_st16(ts + 16 * h, o);
                }
                tmem_st_wait();
                tc_fence_before_sync();
                pipe_arrive_warp(pp, G::BAR_P, lane);
            }
            wait_soon(pp, G::BAR_T, j);
            tc_fence_after_sync();
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t o[32], z[16];
                tmem_ld32(tt + 32 * h, o);
                tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    float4 d = make_float4(dot, dot, dot, dot);
                    if (KEYS) d = st[32 + 8 * h + i];
                    const float2 kk = make_float2(kappa, kappa);
                    float2 e0 = make_float2(__uint_as_float(o[4 * i]), __uint_as_float(o[4 * i + 1])), e1 = make_float2(__uint_as_float(o[4 * i + 2]), __uint_as_float(o[4 * i + 3]));
                    if (is_f16<T>) {
                        e0 = ffma2(e0, kk, make_float2(-d.x, -d.y));
                        e1 = ffma2(e1, kk, make_float2(-d.z, -d.w));
                    } else {
                        e0 = fadd2(e0, make_float2(-d.x, -d.y));
                        e1 = fadd2(e1, make_float2(-d.z, -d.w));
                    }
                    e0 = fmul2(e0, p[16 * h + 2 * i]);
                    e1 = fmul2(e1, p[16 * h + 2 * i + 1]);
                    if (masked) {                                            // (0 * NaN)
                        if (p[16 * h + 2 * i].x == 0.f) e0.x = 0.f;
                        if (p[16 * h + 2 * i].y == 0.f) e0.y = 0.f;
                        if (p[16 * h + 2 * i + 1].x == 0.f) e1.x = 0.f;
                        if (p[16 * h + 2 * i + 1].y == 0.f) e1.y = 0.f;
                    }
                    z[2 * i] = pack2<T>(e0.x, e0.y);
                    z[2 * i + 1] = pack2<T>(e1.x, e1.y);
                }
                tmem_st16(tt + 16 * h, z);
            }
            tmem_st_wait();
            tc_fence_before_sync();
            pipe_arrive_warp(pp, G::BAR_DS, lane);
        }
        if (total) {
            if (KEYS) wait_soon(pp, G::BAR_ACC, total - 1);
            wait_soon(pp, G::BAR_ACC + 1, total - 1);
            tc_fence_after_sync();
        }
        // either half of the warps stores one of the two results, or half of the channels
        const uint32_t mine_lanes = (uint32_t)(32 * (warp & 3)) << 16;
        const float back = is_f16<T> ? kHeldBack : 1.f, factor = KEYS && w ? back : a.scale * back / kappa;
        void* out = KEYS ? (w ? a.dv : a.dk) : a.dq;
        const TokLayout& lo = KEYS ? (w ? a.ldv : a.ldk) : a.ldq;
        T* to = static_cast<T*>(out) + x.batch * lo.sb + mine * lo.sh + (long long)(x.first + row) * lo.st;
        const uint32_t acc = pp.tmem + (KEYS && w ? TM_V : TM_A) + mine_lanes;
#pragma unroll
        for (int h = KEYS ? 0 : BOXES * w; h < (KEYS ? 2 * BOXES : BOXES * (w + 1)); ++h) {
            uint32_t o[32] = {};
            if (total) {
                tmem_ld32(acc + 32 * h, o);
                tmem_ld_wait();
            }
            if (row >= rows) continue;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int c = 32 * h + 8 * g;
                if (c >= a.d) continue;
                float f[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(o[8 * g + i]) * factor;
                *reinterpret_cast<uint4*>(to + c) = pack16<T>(f);
            }
        }
        tc_fence_before_sync();
    }
    __syncthreads();
    if (warp == 8) {
        tc_fence_after_sync();
        tmem_dealloc<512>(pp.tmem);
    }
}

template <typename T, int BOXES, bool KEYS> cudaError_t run(GradArgs u, cudaStream_t st) {
    using G = GradUmma<BOXES>;
    static std::atomic<unsigned long long> done{0};
    if (cudaError_t e = allow_smem(attend_grad_umma_kernel<T, BOXES, KEYS>, done, G::kSmem)) return e;
    u.slots = (unsigned)(KEYS ? slots_of(u.a.k_offsets != nullptr, u.a.sequences, u.a.M, 1, kTileRows) : slots_of(u.a.q_offsets != nullptr, u.a.sequences, u.a.N, 1, kTileRows));
    attend_grad_umma_kernel<T, BOXES, KEYS><<<(unsigned)((long long)u.slots * (KEYS ? u.a.kv_heads : u.a.heads)), kThreads, G::kSmem, st>>>(u);
    return cudaGetLastError();
}
template <typename T, int BOXES> cudaError_t run_both(const GradArgs& u, cudaStream_t st) {
    if (cudaError_t e = run<T, BOXES, true>(u, st)) return e;
    return run<T, BOXES, false>(u, st);
}

}  // namespace

cudaError_t launch_attend_grad_umma(int dtype, const AttendArgs& a, cudaStream_t st) {
    GradArgs u;
    u.a = a;
    if (!make_row_map(&u.q, a.q, a.lq, a.batch, a.heads, a.N, a.d) || !make_row_map(&u.k, a.k, a.lk, a.batch, a.kv_heads, a.M, a.d) ||
        !make_row_map(&u.v, a.v, a.lv, a.batch, a.kv_heads, a.M, a.d) || !make_row_map(&u.dout, a.dout, a.ldo, a.batch, a.heads, a.N, a.d))
        return cudaErrorInvalidValue;
    if (dtype == 1) return a.d <= 64 ? run_both<__nv_bfloat16, 1>(u, st) : run_both<__nv_bfloat16, 2>(u, st);
    return a.d <= 64 ? run_both<__half, 1>(u, st) : run_both<__half, 2>(u, st);
}

}  // namespace aa
