// Gradient of softmax attention over whole sequences, 16-bit types, on the 5th-generation tensor cores.
//
// Two kernels of one form, so that every sum has one owner (no reductions in global memory; the same bits from call to call) at the price of making the
// logits twice (seven products a pair of tiles instead of five):
//   else   a block owns 128 queries of a head and walks their keys:  S = Q K^T, dP = dO V^T, dQ += dS K; bf16: it also makes D = rowsum(dO O) for the other one
//   KEYS   it owns 128 keys and walks the queries, of every head of the group, that see them:  S' = K Q^T, dP' = V dO^T, dV += P' dO, dK += dS' Q
// P = exp2(scale S - lse) and dS = P (dP - D) take the place in tensor memory of what they are made of, as A operands.  Up to 64 channels: two blocks an SM, tiles of 64
// columns; starts and ends of blocks overlap, and one block's exponentials run beside the other's products.  More channels: one block, tiles of 128 columns.  A thread
// has a row and 32 columns of a tile: what a tile costs besides its arithmetic (waits, arrivals, tensor memory) is shared by sixteen warps of an SM (by eight, with 64
// columns each: 8 heads of 4096 x 4096 x 128 257 us, 16 of 64 channels 354).
// Tried: tiles of 64 columns in turns for two groups of one block, 128 channels: 335 us (an instruction of 64 columns costs three quarters of one of 128).
// Bound by waits between products and rows (tensor pipe 56 % with 128 channels, 37 to 39 % with 64): 8 heads of 4096 x 4096 x 128 234 us (735 TFLOP/s of the five products), 16 of 64 channels
// 325 (528); 128 images of 196 tokens, 3 heads of 64, 71 (four short tiles a block).
// Roles after these warps: products; TMA (the block's own rows once, then the columns' two operands in a ring each); a warp that makes rows behind a sequence zero (they
// meet zeros in the sums, and need not be finite) and, KEYS, fetches the queries' statistics.
#include "attend_umma.cuh"

namespace aa {

namespace {

// Tiles of packed sequences in the order of their work, the most first: the tiles of few long sequences differ by as much as their number, and a long one that starts last
// keeps one SM busy alone.  Work of tile i of a sequence, in units of 128 columns: ROWS rows from ROWS i on meet
//   queries  the keys up to the last row's           keys  the queries from the first row's on
// Every lane holds up to four sequences; the work of the tile of rank `slot` is found by bisection on how many tiles have at least so much, then the tile among its equals.
// Some 600 cycles a block, so only where sequences are long (ranked_tiles).  Eight prompts of up to 4096 tokens, 16 heads of 128: 500 -> 483 us.  (The forward kernel's
// blocks are fewer and gain nothing by it: 538 -> 544 us for prompts of up to 8192.)
constexpr int kRanked = 128;
inline bool ranked_tiles(const AttendArgs& a, int rows_of_all) { return a.q_offsets && a.sequences > 1 && a.sequences <= kRanked && rows_of_all / a.sequences >= 512; }
template <int ROWS, bool KEYS> __device__ inline bool find_ranked(const AttendArgs& a, unsigned slot, int lane, int* seq, int* tile) {
    int tiles[kRanked / 32], nq[kRanked / 32], nk[kRanked / 32];
#pragma unroll
    for (int i = 0; i < kRanked / 32; ++i) {
        const int s = 32 * i + lane;
        tiles[i] = nq[i] = nk[i] = 0;
        if (s < a.sequences) {
            nq[i] = span_of(a.q_offsets, nullptr, a.N, s).count;
            nk[i] = span_of(a.k_offsets, nullptr, a.M, s).count;
            tiles[i] = ((KEYS ? nk[i] : nq[i]) + ROWS - 1) / ROWS;
        }
    }
    // tiles of sequence i with at least `units` of work: the first `n` or the last `n` of it
    auto at_least = [&](int i, int units) {
        if (units <= 0 || !tiles[i]) return tiles[i];
        const int ahead = nk[i] - nq[i], need = (units - 1) * 128 + 1;           // columns
        if (!a.causal) return (KEYS ? nq[i] : nk[i]) >= need ? tiles[i] : 0;
        if (KEYS) {                                                              // nq - max(0, k0 - ahead) >= need
            const int most = min(nq[i] - need, nq[i] - need + ahead);            // (k0 = 0 has nq + min(0, ahead))
            return most < 0 ? 0 : min(tiles[i], max(0, nq[i] - need + ahead) / ROWS + 1);      // k0 <= nq - need + ahead
        }
        if (nk[i] < need) return 0;
        // min(nq, (t + 1) ROWS) + ahead >= need: the last tile has all keys
        const int t = max(0, (need - ahead + ROWS - 1) / ROWS - 1);
        return tiles[i] - min(tiles[i] - 1, t);
    };
    auto count = [&](int units) {
        int c = 0;
#pragma unroll
        for (int i = 0; i < kRanked / 32; ++i) c += at_least(i, units);
        return __reduce_add_sync(0xffffffffu, c);
    };
    if ((unsigned)count(0) <= slot) return false;
    int lo = 0, hi = (max(a.N, a.M) + 127) / 128 + 1;                            // count(lo) > slot >= count(hi)
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if ((unsigned)count(mid) > slot) lo = mid;
        else hi = mid;
    }
    int left = (int)slot - count(hi), found = -1, at = 0;                        // rank among the tiles with just `lo` units
#pragma unroll
    for (int i = 0; i < kRanked / 32; ++i) {
        const int some = at_least(i, lo), more = at_least(i, hi), mine = some - more;
        int upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += v;
        }
        const int before = upto - mine;
        if (found < 0 && left >= before && left < upto) {
            found = 32 * i + lane;
            at = !a.causal || KEYS ? more + left - before : tiles[i] - 1 - more - (left - before);
        }
        left -= __shfl_sync(0xffffffffu, upto, 31);
    }
    const unsigned who = __ballot_sync(0xffffffffu, found >= 0);
    if (!who) return false;
    *seq = __shfl_sync(0xffffffffu, found, __ffs(who) - 1);
    *tile = __shfl_sync(0xffffffffu, at, __ffs(who) - 1);
    return true;
}
// A block's sequence and tile; by the first warp where tiles are ranked (`pick`: two words of shared memory)
template <int ROWS, bool KEYS> __device__ __forceinline__ bool block_tile(const AttendArgs& a, bool ranked, unsigned slot, unsigned slots, int* pick, int* seq, int* tile) {
    if (!ranked)       // (causal: the last queries, which see most, come first, and the first keys, which most see)
        return find_slot(KEYS ? a.k_offsets : a.q_offsets, a.sequences, KEYS ? a.M : a.N, 1, ROWS, !KEYS && a.causal ? slots - 1 - slot : slot, seq, tile);
    if (threadIdx.x < 32) {
        int s = -1, t = 0;
        if (!find_ranked<ROWS, KEYS>(a, slot, threadIdx.x, &s, &t)) s = -1;
        if (threadIdx.x == 0) {
            pick[0] = s;
            pick[1] = t;
        }
    }
    __syncthreads();
    *seq = pick[0];
    *tile = pick[1];
    return pick[0] >= 0;
}
struct GradArgs {
    AttendArgs a;
    unsigned slots;
    bool ranked;
    RowMap q, k, v, dout;
};

constexpr int OFF_DEAD = 512, OFF_TMEM = 516, OFF_PICK = 520;
template <int BOXES, bool KEYS> struct GradUmma {
    static constexpr int COLS = 64 * BOXES, GROUPS = 2 * BOXES, kThreads = 128 * GROUPS + 128, kBlocks = BOXES == 1 ? 2 : 1, kColBytes = COLS * 128;
    static constexpr uint32_t kTmem = 256 * BOXES;
    // registers: of the block's threads x kStart at launch
    static constexpr int kStart = BOXES == 1 ? 80 : 96, kRowRegs = BOXES == 1 ? 96 : 104, kRoleRegs = BOXES == 1 ? 48 : 64;
    static_assert(128 * GROUPS * kRowRegs + 128 * kRoleRegs <= kThreads * kStart && kThreads * kStart * kBlocks <= 65536, "registers");
    // stages of the operand that the logits and the last sum read, and of the other one
    static constexpr int kStages = BOXES == 1 ? 4 : KEYS ? 2 : 3, kStats = kStages, kStages1 = BOXES == 1 ? 4 : 2, kOwn = BOXES * kTileBytes, kOperand = BOXES * kColBytes;
    static constexpr int OFF_DOT = 1024, OFF_X = 2048, OFF_RING = OFF_X + 2 * kOwn, OFF_RING1 = OFF_RING + kStages * kOperand, OFF_STAT = OFF_RING1 + kStages1 * kOperand,
                         kSmem = OFF_STAT + (KEYS ? kStats * 2 * COLS * 4 : 0) + 1024;
    static_assert(kSmem * kBlocks <= 232448, "shared memory");
    // mbarriers                             count            waiter
    static constexpr int BAR_X = 0,               // tx               issuer
        BAR_FULL = 1,                             // [stages] tx      last warp
        BAR_READY = BAR_FULL + kStages,           // [stages] 1       issuer, rows
        BAR_FREE = BAR_READY + kStages,           // [stages] commit  producer, last warp
        BAR_FULL1 = BAR_FREE + kStages,           // the same of the other operand
        BAR_READY1 = BAR_FULL1 + kStages1,
        BAR_FREE1 = BAR_READY1 + kStages1,
        BAR_S = BAR_FREE1 + kStages1,             // commit           rows
        BAR_T = BAR_S + 1,                        // [2] commit       rows (KEYS: one buffer)
        BAR_P = BAR_T + 2,                        // rows' warps      issuer: KEYS: P is there; else: S has been read
        BAR_DS = BAR_P + 1,                       // [2] rows' warps  issuer: in turns; without KEYS all may be a tile ahead of it, and a wait knows a phase only from its neighbours
        BAR_V = BAR_DS + 2,                       // commit           issuer
        BAR_A = BAR_V + 1,                        // commit           issuer
        BAR_END = BAR_A + 1,                      // commit, once: everybody
        BAR_PIECE = BAR_END + 1,                  // commit           rows: the last sum of a piece (of BAR_A they may be two phases behind)
        kBars = BAR_PIECE + 1;
    static_assert(8 * kBars <= OFF_DEAD, "mbarriers");
};

// LONG: sums may be longer than a piece (the others do without their code: 128 images of 196 tokens 79.4 us with it, 75.8 without)
template <typename T, int BOXES, bool KEYS, bool LONG>
__global__ void __launch_bounds__(GradUmma<BOXES, KEYS>::kThreads, GradUmma<BOXES, KEYS>::kBlocks) attend_grad_umma_kernel(const __grid_constant__ GradArgs u) {
    using G = GradUmma<BOXES, KEYS>;
    constexpr int kStages = G::kStages, kStages1 = G::kStages1, COLS = G::COLS, kFmt = Elem<T>::kIsBf16 ? 1 : 0;
    // tensor memory columns.  KEYS: S, dP, dV, dK; else S, dP twice, dQ
    constexpr uint32_t TM_T = COLS, TM_V = 2 * COLS, TM_A = 3 * COLS;
    constexpr bool kDot = !KEYS && !is_f16<T>;
    constexpr int kPiece = kPieceKeys / COLS;                       // tiles of a piece of the results' sums
    const AttendArgs& a = u.a;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const uint32_t base = smem_u32(smem);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, role = warp - 4 * G::GROUPS;
    const int group = a.heads / a.kv_heads, wide = KEYS ? a.kv_heads : a.heads, mine = blockIdx.x % wide, hk = KEYS ? mine : mine / group;
    const unsigned slot = blockIdx.x / wide;
    int seq, tile;
    if (!block_tile<kTileRows, KEYS>(a, u.ranked, slot, u.slots, reinterpret_cast<int*>(smem + OFF_PICK), &seq, &tile)) return;
    const Span q = span_of(a.q_offsets, a.q_lengths, a.N, seq), k = span_of(a.k_offsets, a.k_lengths, a.M, seq);
    const int rows = KEYS ? k.count : q.count, r0 = tile * kTileRows;
    if (r0 >= rows) return;
    // tiles of columns: `per` of every head, from `first` on
    const int ahead = k.count - q.count;                            // query i sees the keys up to i + ahead
    int first = 0, per;
    if (KEYS) {
        if (a.causal) first = max(0, r0 - ahead) / COLS;
        per = max(0, (q.count + COLS - 1) / COLS - first);
    } else {
        per = (visible_keys(a.causal, min(rows, r0 + kTileRows) - 1, q.count, k.count) + COLS - 1) / COLS;
    }
    const int total = KEYS ? per * group : per, steps = (a.d + 15) / 16;
    const Span x = KEYS ? k : q, y = KEYS ? q : k;                  // rows, columns

    Pipe pp;
    pp.status = a.status;
    pp.dead = reinterpret_cast<int*>(smem + OFF_DEAD);
    pp.bars = base;
    auto load = [&](int j, int which, int row, int head) {          // one operand of a tile of columns (by one lane)
        const int s = j % (which ? kStages1 : kStages);
        const uint32_t bar = pipe_bar(pp, (which ? G::BAR_FULL1 : G::BAR_FULL) + s), dst = base + (which ? G::OFF_RING1 : G::OFF_RING) + s * G::kOperand;
        mbar_arrive_expect_tx(bar, G::kOperand);
        for (int b = 0; b < BOXES; ++b)
            load_rows(dst + b * G::kColBytes, which ? (KEYS ? u.dout : u.v) : (KEYS ? u.q : u.k), 64 * b, row, KEYS ? head : hk, y.batch, bar);
    };
    if (role == 1) {                                                // the first loads are on their way while the block is set up
        if (lane == 0) *pp.dead = 0;
        for (int i = lane; i < G::kBars; i += 32) mbar_init(pp.bars + 8 * i, i >= G::BAR_P && i < G::BAR_V ? 4u * G::GROUPS : 1u);
        mbar_fence_init();
        __syncwarp();
        if (lane == 0 && total) {
            constexpr int kParts = kTileRows / COLS;               // (boxes of COLS rows)
            mbar_arrive_expect_tx(pipe_bar(pp, G::BAR_X), 2 * G::kOwn);
            for (int b = 0; b < kParts * BOXES; ++b) {
                const int ch = 64 * (b / kParts), row = x.first + r0 + COLS * (b % kParts);
                load_rows(base + G::OFF_X + b * G::kColBytes, KEYS ? u.k : u.q, ch, row, mine, x.batch, pipe_bar(pp, G::BAR_X));
                load_rows(base + G::OFF_X + G::kOwn + b * G::kColBytes, KEYS ? u.v : u.dout, ch, row, mine, x.batch, pipe_bar(pp, G::BAR_X));
            }
            load(0, 0, y.first + first * COLS, hk * group);
            load(0, 1, y.first + first * COLS, hk * group);
        }
        __syncwarp();
    }
    if (role == 0) tmem_alloc<G::kTmem>(base + OFF_TMEM);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    pp.tmem = *reinterpret_cast<const volatile uint32_t*>(smem + OFF_TMEM);
    float* stats = reinterpret_cast<float*>(smem + G::OFF_STAT);   // [kStats][lse | D][COLS]
    const float kappa_seq = KEYS && is_f16<T> ? grad_factor(__uint_as_float(grad_most(a, seq, hk)[0]), __uint_as_float(grad_most(a, seq, hk)[1])) : 1.f;

    if (role >= 0) {
    set_regs_dec<G::kRoleRegs>();
    if (role == 1) {
        // ------------------------------------------------------------------ producer
        if (lane == 0) {
            int t = 0, head = hk * group;
            for (int j = 1; j < total && !pipe_dead(pp); ++j) {
                if (++t == per) { t = 0; ++head; }
                for (int which = 0; which < 2; ++which) {
                    const int stages = which ? kStages1 : kStages;
                    if (j >= stages) wait_spin(pp, (which ? G::BAR_FREE1 : G::BAR_FREE) + j % stages, j / stages - 1, kAttendTimeout);
                    load(j, which, y.first + (first + t) * COLS, head);
                }
            }
        }
        __syncwarp();
    } else if (role == 2) {
        // ------------------------------------------------------------------ rows behind the sequence; statistics of the columns
        int t = 0, head = hk * group;
        float2 next[COLS / 32];
        auto fetch = [&](int t, int head) {                          // (a tile ahead: the loads take longer than anything else here)
            const int c0 = (first + t) * COLS;
            const float2* st = reinterpret_cast<const float2*>(a.ws) + ((long long)q.batch * a.heads + head) * a.N + q.first + c0;
#pragma unroll
            for (int i = 0; i < COLS / 32; ++i)                      // (a column that is none: a probability of zero)
                next[i] = c0 + 32 * i + lane < q.count ? __ldg(st + 32 * i + lane) : make_float2(INFINITY, 0.f);
        };
        if (KEYS && total) fetch(t, head);
        for (int j = 0; j < total && !pipe_dead(pp); ++j) {
            const int s = j % kStages, s1 = j % kStages1, left = y.count - (first + t) * COLS;
            if (++t == per) { t = 0; ++head; }
            if (KEYS) {
                if (j >= G::kStats) wait_spin(pp, G::BAR_FREE + (j - G::kStats) % kStages, (j - G::kStats) / kStages, kAttendTimeout);      // (the last sum comes after all reads)
                float* to = stats + j % G::kStats * 2 * COLS;
#pragma unroll
                for (int i = 0; i < COLS / 32; ++i) {
                    to[32 * i + lane] = next[i].x - (is_f16<T> ? kHeldP : 0.f);
                    to[COLS + 32 * i + lane] = next[i].y * kappa_seq;
                }
                if (j + 1 < total) fetch(t, head);
            }
            wait_spin(pp, G::BAR_FULL + s, j / kStages, kAttendTimeout);
            if (left < COLS) {
                clear_rows<COLS>(base + G::OFF_RING + s * G::kOperand, BOXES, left, lane);
                fence_proxy_async();
            }
            __syncwarp();
            if (lane == 0) pipe_arrive(pp, G::BAR_READY + s);
            __syncwarp();
            wait_spin(pp, G::BAR_FULL1 + s1, j / kStages1, kAttendTimeout);
            if (left < COLS) {
                clear_rows<COLS>(base + G::OFF_RING1 + s1 * G::kOperand, BOXES, left, lane);
                fence_proxy_async();
            }
            __syncwarp();
            if (lane == 0) pipe_arrive(pp, G::BAR_READY1 + s1);
            __syncwarp();
        }
        __syncwarp();
    } else if (role == 0) {
        // ------------------------------------------------------------------ products
        const uint32_t id_s = umma_idesc(kFmt, 128, COLS, 0), id_a = umma_idesc(kFmt, 128, steps * 16, 1), elected = elect_lane();
        auto ring = [&](int j) { return base + G::OFF_RING + (j % kStages) * G::kOperand; };
        auto ring1 = [&](int j) { return base + G::OFF_RING1 + (j % kStages1) * G::kOperand; };
        auto slope_at = [&](int j) { return pp.tmem + TM_T + (KEYS ? 0 : (j & 1) * COLS); };
        auto logits = [&](int j) {
            wait_spin(pp, G::BAR_READY + j % kStages, j / kStages, kAttendTimeout);
            tc_fence_after_sync();
            mma_rows<BOXES, COLS>(elected, pp.tmem, base + G::OFF_X, ring(j), id_s, steps);
            umma_commit_e<false>(elected, pipe_bar(pp, G::BAR_S));
        };
        auto slopes = [&](int j) {
            wait_spin(pp, G::BAR_READY1 + j % kStages1, j / kStages1, kAttendTimeout);
            tc_fence_after_sync();
            mma_rows<BOXES, COLS>(elected, slope_at(j), base + G::OFF_X + G::kOwn, ring1(j), id_s, steps);
            umma_commit_e<false>(elected, pipe_bar(pp, G::BAR_T + (KEYS ? 0 : j & 1)));
            if (!KEYS) umma_commit_e<false>(elected, pipe_bar(pp, G::BAR_FREE1 + j % kStages1));
        };
        if (total) {
            wait_spin(pp, G::BAR_X, 0, kAttendTimeout);
            logits(0);
            slopes(0);
        }
        for (int j = 0; j < total && !pipe_dead(pp); ++j) {
            wait_spin(pp, G::BAR_P, j, kAttendTimeout);                      // (KEYS: P; else S has been read)
            tc_fence_after_sync();
            if (KEYS) {
                mma_sum<BOXES, COLS, 32>(elected, pp.tmem + TM_V, pp.tmem, ring1(j), id_a, LONG ? j % kPiece != 0 : j > 0);
                umma_commit_e<false>(elected, pipe_bar(pp, G::BAR_FREE1 + j % kStages1));
                umma_commit_e<false>(elected, pipe_bar(pp, G::BAR_V));
                if (j + 1 < total) {
                    wait_spin(pp, G::BAR_V, j, kAttendTimeout);              // (the next logits take the place of the probabilities)
                    logits(j + 1);
                }
            } else if (j + 1 < total) {
                logits(j + 1);
                if (j > 0) wait_spin(pp, G::BAR_A, j - 1, kAttendTimeout);   // (the next slopes that of dS of two tiles ago)
                slopes(j + 1);
            }
            wait_spin(pp, G::BAR_DS + (j & 1), j >> 1, kAttendTimeout);
            tc_fence_after_sync();
            mma_sum<BOXES, COLS, 32>(elected, pp.tmem + TM_A, slope_at(j), ring(j), id_a, LONG ? j % kPiece != 0 : j > 0);
            umma_commit_e<false>(elected, pipe_bar(pp, G::BAR_FREE + j % kStages));
            umma_commit_e<false>(elected, pipe_bar(pp, G::BAR_A));
            if (LONG && (j + 1) % kPiece == 0) umma_commit_e<false>(elected, pipe_bar(pp, G::BAR_PIECE));
            if (KEYS && j + 1 < total) {
                wait_spin(pp, G::BAR_A, j, kAttendTimeout);
                slopes(j + 1);
            }
        }
        umma_drain_w(pp, G::BAR_END);
        __syncwarp();
    }
    } else {
        // ------------------------------------------------------------------ P and dS
        set_regs_inc<G::kRowRegs>();
        const int w = warp >> 2, local = 32 * (warp & 3) + lane, row = r0 + local;
        const uint32_t lanes = (uint32_t)(32 * (warp & 3)) << 16;
        const uint32_t elected = elect_lane();
        const float c1 = a.scale * kLog2e;
        float lse = 0.f, dot = 0.f, kappa = kappa_seq;
        int limit = 0;                             // rows are queries: keys that this one sees; keys: the first query that sees it
        float2* dots = reinterpret_cast<float2*>(smem + G::OFF_DOT);         // (one group makes the rows' statistics, all read them)
        if (kDot) {
            float2 st = make_float2(0.f, 0.f);
            if (w == 0 && row < rows) {
                const long long at = ((long long)q.batch * a.heads + mine) * a.N + q.first + row;
                const T* o = static_cast<const T*>(a.out) + q.batch * a.lo.sb + mine * a.lo.sh + (long long)(q.first + row) * a.lo.st;
                const T* g = static_cast<const T*>(a.dout) + q.batch * a.ldo.sb + mine * a.ldo.sh + (long long)(q.first + row) * a.ldo.st;
                st = make_float2(a.lse[at] * kLog2e, 0.f);
#pragma unroll 4
                for (int c = 0; c < a.d; c += 8) {
                    float f[8], h[8];
                    unpack16<T>(__ldg(reinterpret_cast<const uint4*>(o + c)), f);
                    unpack16<T>(__ldg(reinterpret_cast<const uint4*>(g + c)), h);
#pragma unroll
                    for (int e = 0; e < 8; ++e) st.y = fmaf(f[e], h[e], st.y);
                }
                reinterpret_cast<float2*>(a.ws)[at] = st;
            }
            if (w == 0) dots[local] = st;
            asm volatile("bar.sync 1, %0;\n" ::"n"(128 * G::GROUPS) : "memory");
        }
        if (KEYS) {
            limit = a.causal ? row - ahead : 0;
        } else if (row < rows) {
            float2 st;
            if (kDot) {
                st = dots[local];
            } else {
                const long long at = ((long long)q.batch * a.heads + mine) * a.N + q.first + row;
                st = __ldg(reinterpret_cast<const float2*>(a.ws) + at);
                kappa = grad_factor(grad_norms(a)[at], __uint_as_float(grad_most(a, seq, hk)[1]));
            }
            lse = st.x - (is_f16<T> ? kHeldP : 0.f);
            dot = st.y * kappa;
            limit = visible_keys(a.causal, row, q.count, k.count);
        }
        const int whole = KEYS ? 0 : visible_keys(a.causal, r0, q.count, k.count);         // keys that every row sees
        // a thread's share of the results' channels is 32 at a time of dK and dV, or of dQ; of a long sum the pieces so far (in local memory, touched once a piece)
        constexpr int kParts = KEYS ? 2 : 1;
        auto result = [&](int i) {                                  // in tensor memory
            const int part = KEYS ? 2 * w + i : w;
            return pp.tmem + (part / (2 * BOXES) ? TM_V : TM_A) + lanes + 32 * (part % (2 * BOXES));
        };
        volatile float kept[LONG ? kParts : 1][LONG ? 32 : 1];
        int t = 0;
        for (int j = 0; j < total; ++j) {
            if (LONG && j > 0 && j % kPiece == 0) {
                wait_soon(pp, G::BAR_PIECE, j / kPiece - 1);
                tc_fence_after_sync();
#pragma unroll
                for (int i = 0; i < kParts; ++i) {
                    uint32_t o[32];
                    tmem_ld32(result(i), o);
                    tmem_ld_wait();
#pragma unroll
                    for (int e = 0; e < 32; ++e) kept[LONG ? i : 0][LONG ? e : 0] = j == kPiece ? __uint_as_float(o[e]) : kept[LONG ? i : 0][LONG ? e : 0] + __uint_as_float(o[e]);
                }
            }
            const int s = j % kStages, tile0 = (first + t) * COLS, c0 = tile0 + 32 * w;       // (this thread's columns)
            if (++t == per) t = 0;
            const bool masked = KEYS ? tile0 + COLS > q.count || (a.causal && tile0 < r0 + kTileRows - 1 - ahead) : tile0 + COLS > whole;
            const float4* st = reinterpret_cast<const float4*>(stats + j % G::kStats * 2 * COLS + 32 * w);
            if (KEYS) wait_soon(pp, G::BAR_READY + s, j / kStages);
            wait_soon(pp, G::BAR_S, j);
            tc_fence_after_sync();
            const uint32_t ts = pp.tmem + lanes + 32 * w, tt = pp.tmem + TM_T + (KEYS ? 0 : (j & 1) * COLS) + lanes + 32 * w;
            uint32_t o[32], z[16];
            tmem_ld32(ts, o);
            tmem_ld_wait();
            if (!KEYS) {
                tc_fence_before_sync();
                arrive_warp_e<false>(elected, pipe_bar(pp, G::BAR_P));
            }
            float2 p[16];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float4 l = make_float4(lse, lse, lse, lse);
                if (KEYS) l = st[i];
                const float2 e0 = ffma2(make_float2(__uint_as_float(o[4 * i]), __uint_as_float(o[4 * i + 1])), make_float2(c1, c1), make_float2(-l.x, -l.y));
                const float2 e1 = ffma2(make_float2(__uint_as_float(o[4 * i + 2]), __uint_as_float(o[4 * i + 3])), make_float2(c1, c1), make_float2(-l.z, -l.w));
                p[2 * i] = make_float2(fast_exp2(e0.x), fast_exp2(e0.y));
                p[2 * i + 1] = make_float2(fast_exp2(e1.x), fast_exp2(e1.y));
            }
            if (masked) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int c = c0 + 2 * i;
                    if (KEYS ? c < limit || c >= q.count : c >= limit) p[i].x = 0.f;
                    if (KEYS ? c + 1 < limit || c + 1 >= q.count : c + 1 >= limit) p[i].y = 0.f;
                }
            }
            if (KEYS) {
#pragma unroll
                for (int i = 0; i < 16; ++i) z[i] = pack2<T>(p[i].x, p[i].y);
                tmem_st16(ts, z);
                tmem_st_wait();
                tc_fence_before_sync();
                arrive_warp_e<false>(elected, pipe_bar(pp, G::BAR_P));
            }
            wait_soon(pp, G::BAR_T + (KEYS ? 0 : j & 1), KEYS ? j : j >> 1);
            tc_fence_after_sync();
            tmem_ld32(tt, o);
            tmem_ld_wait();
            if (!KEYS && j == 0 && whole <= COLS) {
                // Rows whose keys are all in this tile (short sequences, the first rows of a causal one): D = sum P dP.  Out of the result, which is rounded, it would be off
                // by as much as the slopes of two or three keys differ (sequences of two: error of dQ and dK 2.4 of a rounding, so 1.5).
                float2 sum2 = make_float2(0.f, 0.f);
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    sum2 = make_float2(p[i].x != 0.f ? fmaf(p[i].x, __uint_as_float(o[2 * i]), sum2.x) : sum2.x, p[i].y != 0.f ? fmaf(p[i].y, __uint_as_float(o[2 * i + 1]), sum2.y) : sum2.y);
                float* share = reinterpret_cast<float*>(smem + G::OFF_DOT);          // two groups' shares of 128 rows, in place of the statistics, which all have read
                float own = sum2.x + sum2.y;
                auto meet = [] { asm volatile("bar.sync 1, %0;\n" ::"n"(128 * G::GROUPS) : "memory"); };
                if (kDot) meet();
                if (G::GROUPS > 2) {
                    if (w >= 2) share[128 * (w - 2) + local] = own;
                    meet();
                    if (w < 2) own += share[128 * w + local];
                    meet();
                }
                if (w < 2) share[128 * w + local] = own;
                meet();
                if (limit <= COLS) {
                    dot = (share[local] + share[128 + local]) * (is_f16<T> ? kHeldBack : 1.f);
                    if (w == 0 && row < rows) a.ws[2 * (((long long)q.batch * a.heads + mine) * a.N + q.first + row) + 1] = dot;
                    dot *= kappa;
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float4 d = make_float4(dot, dot, dot, dot);
                if (KEYS) d = st[COLS / 4 + i];
                const float2 kk = make_float2(kappa, kappa);
                float2 e0 = make_float2(__uint_as_float(o[4 * i]), __uint_as_float(o[4 * i + 1])), e1 = make_float2(__uint_as_float(o[4 * i + 2]), __uint_as_float(o[4 * i + 3]));
                if (is_f16<T>) {
                    e0 = ffma2(e0, kk, make_float2(-d.x, -d.y));
                    e1 = ffma2(e1, kk, make_float2(-d.z, -d.w));
                } else {
                    e0 = fadd2(e0, make_float2(-d.x, -d.y));
                    e1 = fadd2(e1, make_float2(-d.z, -d.w));
                }
                e0 = fmul2(e0, p[2 * i]);
                e1 = fmul2(e1, p[2 * i + 1]);
                z[2 * i] = pack2<T>(e0.x, e0.y);
                z[2 * i + 1] = pack2<T>(e1.x, e1.y);
            }
            if (masked) {                                                    // (0 * NaN)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    if (p[i].x == 0.f) z[i] &= 0xffff0000u;
                    if (p[i].y == 0.f) z[i] &= 0xffffu;
                }
            }
            tmem_st16(tt, z);
            tmem_st_wait();
            tc_fence_before_sync();
            arrive_warp_e<false>(elected, pipe_bar(pp, G::BAR_DS + (j & 1)));
        }
        wait_soon(pp, G::BAR_END, 0);
        tc_fence_after_sync();
        // every group stores its share of the results' channels, 32 at a time: dK and dV, or dQ
        const float back = is_f16<T> ? kHeldBack : 1.f;
#pragma unroll
        for (int i = 0; i < kParts; ++i) {
            const int part = KEYS ? 2 * w + i : w, r = part / (2 * BOXES), h = part % (2 * BOXES);
            // (a query that sees one key has P = 1, whatever its logit: no gradient but that of the value)
            const float factor = r ? back : (KEYS ? k.count : limit) == 1 ? 0.f : a.scale * back / kappa;
            void* out = KEYS ? (r ? a.dv : a.dk) : a.dq;
            const TokLayout& lo = KEYS ? (r ? a.ldv : a.ldk) : a.ldq;
            T* to = static_cast<T*>(out) + x.batch * lo.sb + mine * lo.sh + (long long)(x.first + r0 + 32 * (warp & 3)) * lo.st + 32 * h;       // the warp's first row
            uint32_t o[32] = {};
            if (total) {
                tmem_ld32(result(i), o);
                tmem_ld_wait();
                if (LONG && total > kPiece)
#pragma unroll
                    for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(kept[LONG ? i : 0][LONG ? e : 0] + __uint_as_float(o[e]));
            }
            // through a place of the warp's own among the block's rows, which nothing reads any more (nor, without columns, has loaded): 64 bytes a row
            unsigned char* stage = smem + G::OFF_X + (i * 4 * G::GROUPS + warp) * 2048;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                float f[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(o[8 * g + e]) * factor;
                *reinterpret_cast<uint4*>(stage + lane * 64 + ((g ^ ((lane >> 1) & 3)) << 4)) = pack16<T>(f);
            }
            __syncwarp();
            const int chunk = lane & 3;
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const int line = 8 * n + (lane >> 2);
                if (r0 + 32 * (warp & 3) + line < rows && 32 * h + 8 * chunk < a.d)
                    *reinterpret_cast<uint4*>(to + (long long)line * lo.st + 8 * chunk) = *reinterpret_cast<const uint4*>(stage + line * 64 + ((chunk ^ ((line >> 1) & 3)) << 4));
            }
        }
        tc_fence_before_sync();
    }
    __syncthreads();
    if (role == 0) {
        tc_fence_after_sync();
        tmem_dealloc<G::kTmem>(pp.tmem);
    }
}

template <typename T, int BOXES, bool KEYS, bool LONG> cudaError_t run_form(const GradArgs& u, cudaStream_t st) {
    using G = GradUmma<BOXES, KEYS>;
    static std::atomic<unsigned long long> done{0};
    if (cudaError_t e = allow_smem(attend_grad_umma_kernel<T, BOXES, KEYS, LONG>, done, G::kSmem)) return e;
    attend_grad_umma_kernel<T, BOXES, KEYS, LONG><<<(unsigned)((long long)u.slots * (KEYS ? u.a.kv_heads : u.a.heads)), G::kThreads, G::kSmem, st>>>(u);
    return cudaGetLastError();
}
template <typename T, int BOXES, bool KEYS> cudaError_t run(GradArgs u, cudaStream_t st) {
    u.ranked = ranked_tiles(u.a, KEYS ? u.a.M : u.a.N);
    u.slots = (unsigned)(KEYS ? slots_of(u.a.k_offsets != nullptr, u.a.sequences, u.a.M, 1, kTileRows) : slots_of(u.a.q_offsets != nullptr, u.a.sequences, u.a.N, 1, kTileRows));
    // (a head of a group adds its whole tiles of columns; of packed sequences the longest may have all rows)
    const long long columns = KEYS ? ((long long)u.a.N + kTileRows) * (u.a.heads / u.a.kv_heads) : u.a.M;
    return columns > kPieceKeys ? run_form<T, BOXES, KEYS, true>(u, st) : run_form<T, BOXES, KEYS, false>(u, st);
}
template <typename T, int BOXES> cudaError_t run_both(const GradArgs& u, cudaStream_t st) {
    if (cudaError_t e = run<T, BOXES, false>(u, st)) return e;
    return run<T, BOXES, true>(u, st);
}

}  // namespace

cudaError_t launch_attend_grad_umma(int dtype, const AttendArgs& a, cudaStream_t st) {
    GradArgs u;
    u.a = a;
    const int box = a.d <= 64 ? 64 : 128;
    if (!make_row_map(&u.q, a.q, a.lq, a.batch, a.heads, a.N, a.d, box) || !make_row_map(&u.k, a.k, a.lk, a.batch, a.kv_heads, a.M, a.d, box) ||
        !make_row_map(&u.v, a.v, a.lv, a.batch, a.kv_heads, a.M, a.d, box) || !make_row_map(&u.dout, a.dout, a.ldo, a.batch, a.heads, a.N, a.d, box))
        return cudaErrorInvalidValue;
    if (dtype == 1) return a.d <= 64 ? run_both<__nv_bfloat16, 1>(u, st) : run_both<__nv_bfloat16, 2>(u, st);
    return a.d <= 64 ? run_both<__half, 1>(u, st) : run_both<__half, 2>(u, st);
}

}  // namespace aa
