// Softmax attention over whole sequences, forward, 16-bit types, on the 5th-generation tensor cores.
//
// A block takes two tiles of 128 queries of a head and walks the keys in tiles of 128 that both share.  Roles:
//   warps 0-3, 4-7  a tile each: thread = query.  Logits come out of tensor memory into registers, 128 at a time; probabilities go back to tensor memory as the
//                   A operand of P V.  The exponents' reference moves only when a logit exceeds it by more than kSlack: then the thread
//                   rescales its row of the result in tensor memory.  Sums over long axes come in pieces (kPieceKeys).  Sums in fp32, of unrounded probabilities;
//                   probabilities are rounded to the type (half a step each; sums over many keys see less, unless the keys are equal, which are rounded alike).
//   warps 8, 11     issue the products of a tile of queries each: the logits of its next keys while its probabilities are made (up to 64 channels; above, the
//                   logits take the place of the probabilities)
//   warp 9          TMA: queries, keys and values
//   warp 10         looks after the values of tiles that not every query sees whole: rows behind the sequence become zero, and so do numbers that are
//                   not finite (0 * infinity is NaN); the queries that do see these get their NaN at the end
// Results are stored by rows of the sequence alone.
//
// Bound by the row warps up to 64 channels (special-function unit 69 % busy; 16 heads of 16384 x 16384 x 64 1451 to 1473 us, 746 to 758 TFLOP/s), by the chain products - exponentials - products above
// (tensor pipe 51 %; 8 heads of 8192 x 8192 x 128 281 us, 977 TFLOP/s; causal, 16 heads on 4 of keys 273, 1007), and by starts and ends of blocks on short sequences, one block an SM.
#include "attend_umma.cuh"


namespace aa {

namespace {

struct UmmaArgs {
    AttendArgs a;
    unsigned slots;
    RowMap q, k, v;
};

template <int BOXES> struct FwdGeom {
    static constexpr int kStages = BOXES == 1 ? 4 : 2, kOperand = BOXES * kTileBytes;
    // shared memory (bytes from a 1024-aligned base)
    static constexpr int OFF_BAD = 512, OFF_Q = 1024, OFF_K = OFF_Q + 2 * kOperand, OFF_V = OFF_K + kStages * kOperand, kSmem = OFF_V + kStages * kOperand + 1024;
    static_assert(OFF_BAD + BOXES * 64 * 4 <= OFF_Q && kSmem <= 232448, "shared memory");
    // tensor memory columns: logits, probabilities (two channels' boxes: in place of the logits), results; of the first tile, the second one `step` further
    static constexpr uint32_t TM_S = 0, kS = 128, TM_P = BOXES == 1 ? 256 : 0, kP = BOXES == 1 ? 64 : 128, TM_O = BOXES == 1 ? 384 : 256, kO = 64 * BOXES;
    // mbarriers
    static constexpr int BAR_Q = 0, BAR_KFULL = 1, BAR_KFREE = BAR_KFULL + kStages, BAR_VFULL = BAR_KFREE + kStages, BAR_VREADY = BAR_VFULL + kStages,
                         BAR_VFREE = BAR_VREADY + kStages, BAR_S = BAR_VFREE + kStages, BAR_READ = BAR_S + 2, BAR_P = BAR_READ + 2, BAR_O = BAR_P + 2,
                         BAR_MENDED = BAR_O + 2, BAR_DRAIN = BAR_MENDED + 1, kBars = BAR_DRAIN + 2;
    static_assert(8 * kBars <= 256, "mbarriers");
};
constexpr int OFF_DEAD = 256, OFF_TMEM = 260;
constexpr int kThreads = 384;
constexpr int kRowRegs = 208, kRoleRegs = 80;       // 256 x 208 + 128 x 80 of the 384 x 168 that the block starts with
static_assert(256 * kRowRegs + 128 * kRoleRegs <= kThreads * 168, "registers");

// Turns of two warps, one of each tile, that share a scheduler: the exponentials of one run beside the products and maxima of the other.  In step with each other both
// would wait for the tensor cores, and then both for the special-function unit (8 heads of 8192 x 8192 x 128: 325 -> 283 us, 16 of 64 channels 476 -> 421).
__device__ __forceinline__ void bar_sync_pair(int id) { asm volatile("bar.sync %0, 64;\n" ::"r"(id) : "memory"); }
__device__ __forceinline__ void bar_arrive_pair(int id) { asm volatile("bar.arrive %0, 64;\n" ::"r"(id) : "memory"); }

template <typename T, int BOXES>
__global__ void __launch_bounds__(kThreads, 1) attend_umma_kernel(const __grid_constant__ UmmaArgs u) {
    using G = FwdGeom<BOXES>;
    constexpr int kStages = G::kStages, kFmt = Elem<T>::kIsBf16 ? 1 : 0;
    const AttendArgs& a = u.a;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const uint32_t base = smem_u32(smem);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int head = blockIdx.x % a.heads, hk = head / (a.heads / a.kv_heads);
    const unsigned slot = blockIdx.x / a.heads;
    int seq, tile;
    // (causal: the last queries, which see most, first)
    if (!find_slot(a.q_offsets, a.sequences, a.N, 1, 2 * kTileRows, a.causal ? u.slots - 1 - slot : slot, &seq, &tile)) return;
    const Span q = span_of(a.q_offsets, a.q_lengths, a.N, seq), k = span_of(a.k_offsets, a.k_lengths, a.M, seq);
    const int q0 = tile * 2 * kTileRows;
    if (q0 >= q.count) return;
    // key tiles of either tile of queries, and the first of them that not every query of it sees whole
    int n[2], part[2];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        const int first = q0 + w * kTileRows, last = min(q.count, first + kTileRows) - 1;
        n[w] = first < q.count ? (visible_keys(a.causal, last, q.count, k.count) + kTileRows - 1) / kTileRows : 0;
        part[w] = first < q.count ? visible_keys(a.causal, first, q.count, k.count) / kTileRows : INT_MAX;
    }
    const int tiles = max(n[0], n[1]), steps = (a.d + 15) / 16;

    Pipe pp;
    pp.status = a.status;
    pp.dead = reinterpret_cast<int*>(smem + OFF_DEAD);
    pp.bars = base;
    int* first_bad = reinterpret_cast<int*>(smem + G::OFF_BAD);
    auto fetch = [&](int j, int kind) {                             // keys or values of a tile (by one lane)
        const int s = j % kStages;
        const uint32_t bar = pipe_bar(pp, (kind ? G::BAR_VFULL : G::BAR_KFULL) + s), dst = base + (kind ? G::OFF_V : G::OFF_K) + s * G::kOperand;
        mbar_arrive_expect_tx(bar, G::kOperand);
        for (int b = 0; b < BOXES; ++b) load_rows(dst + b * kTileBytes, kind ? u.v : u.k, 64 * b, k.first + j * kTileRows, hk, k.batch, bar);
    };
    if (warp == 9) {                                                // the first loads are on their way while the block is set up
        if (lane == 0) *pp.dead = 0;
        for (int i = lane; i < G::kBars; i += 32)
            mbar_init(pp.bars + 8 * i, i >= G::BAR_READ && i < G::BAR_O ? 4u : (i >= G::BAR_KFREE && i < G::BAR_VFULL) || (i >= G::BAR_VFREE && i < G::BAR_S) ? 2u : 1u);
        mbar_fence_init();
        __syncwarp();
        if (lane == 0 && tiles) {
            const int both = n[1] ? 2 : 1;
            mbar_arrive_expect_tx(pipe_bar(pp, G::BAR_Q), both * G::kOperand);
            for (int w = 0; w < both; ++w)
                for (int b = 0; b < BOXES; ++b)
                    load_rows(base + G::OFF_Q + w * G::kOperand + b * kTileBytes, u.q, 64 * b, q.first + q0 + w * kTileRows, head, q.batch, pipe_bar(pp, G::BAR_Q));
            for (int j = 0; j < min(tiles, kStages); ++j)
                for (int kind = 0; kind < 2; ++kind) fetch(j, kind);
        }
        __syncwarp();
    }
    if (tid < 64 * BOXES) first_bad[tid] = INT_MAX;
    if (warp == 8) tmem_alloc<512>(base + OFF_TMEM);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    pp.tmem = *reinterpret_cast<const volatile uint32_t*>(smem + OFF_TMEM);

    if (warp >= 8) {
    set_regs_dec<kRoleRegs>();
    if (warp == 9) {
        // ------------------------------------------------------------------ producer
        if (lane == 0)
            for (int j = kStages; j < tiles && !pipe_dead(pp); ++j)
                for (int kind = 0; kind < 2; ++kind) {
                    wait_spin(pp, (kind ? G::BAR_VFREE : G::BAR_KFREE) + j % kStages, j / kStages - 1, kAttendTimeout);
                    fetch(j, kind);
                }
        __syncwarp();
    } else if (warp == 10) {
        // ------------------------------------------------------------------ values that not every query sees
        for (int j = 0; j < tiles && !pipe_dead(pp); ++j) {
            const int s = j % kStages;
            const uint32_t v = base + G::OFF_V + s * G::kOperand;
            wait_spin(pp, G::BAR_VFULL + s, j / kStages, kAttendTimeout);
            const bool masked = (j < n[0] && j >= part[0]) || (j < n[1] && j >= part[1]);
            if (masked) {
                const int left = min(kTileRows, k.count - j * kTileRows);
                clear_rows<kTileRows>(v, BOXES, left, lane);
                __syncwarp();
                // an exponent of ones, infinity or NaN, carries into the sign bit; eight loads at a time (one by one they took longer than a tile)
                constexpr uint32_t kExp = Elem<T>::kIsBf16 ? 0x7f807f80u : 0x7c007c00u, kOne = Elem<T>::kIsBf16 ? 0x00800080u : 0x04000400u;
                for (int at = lane * 16; at < BOXES * kTileBytes; at += 8 * 512) {
                    uint4 x[8];
                    uint32_t bad = 0;
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = *reinterpret_cast<const uint4*>(smem + (v - base) + at + 512 * i);
#pragma unroll
                    for (int i = 0; i < 8; ++i) bad |= ((x[i].x & kExp) + kOne) | ((x[i].y & kExp) + kOne) | ((x[i].z & kExp) + kOne) | ((x[i].w & kExp) + kOne);
                    if (!(bad & 0x80008000u)) continue;
                    for (int i = 0; i < 8; ++i) {
                        const int here = at + 512 * i, row = here % kTileBytes / 128, c0 = 64 * (here / kTileBytes) + (((here >> 4) & 7) ^ (row & 7)) * 8;
                        unsigned short* e = reinterpret_cast<unsigned short*>(smem + (v - base) + here);
                        for (int n = 0; n < 8; ++n)
                            if ((e[n] & (kExp & 0xffffu)) == (kExp & 0xffffu)) {
                                e[n] = 0;
                                atomicMin(first_bad + c0 + n, j * kTileRows + row);
                            }
                    }
                }
                fence_proxy_async();
            }
            __syncwarp();
            if (lane == 0) pipe_arrive(pp, G::BAR_VREADY + s);
        }
        __syncwarp();
        if (lane == 0) pipe_arrive(pp, G::BAR_MENDED);
        __syncwarp();
    } else {
        // ------------------------------------------------------------------ products of one tile of queries
        const int w = warp == 8 ? 0 : 1;
        const uint32_t id_s = umma_idesc(kFmt, 128, 128, 0), id_o = umma_idesc(kFmt, 128, steps * 16, 1), elected = elect_lane();
        const uint32_t tp = pp.tmem + G::TM_P + w * G::kP;
        auto logits = [&](int j) {
            const int s = j % kStages;
            wait_spin(pp, G::BAR_KFULL + s, j / kStages, kAttendTimeout);
            tc_fence_after_sync();
            mma_rows<BOXES, kTileRows>(elected, pp.tmem + G::TM_S + w * G::kS, base + G::OFF_Q + w * G::kOperand, base + G::OFF_K + s * G::kOperand, id_s, steps);
            umma_commit_e<false>(elected, pipe_bar(pp, G::BAR_S + w));
            umma_commit_e<false>(elected, pipe_bar(pp, G::BAR_KFREE + s));
        };
        if (n[w]) {
            wait_spin(pp, G::BAR_Q, 0, kAttendTimeout);
            logits(0);
        }
        for (int j = 0; j < n[w] && !pipe_dead(pp); ++j) {
            const int s = j % kStages;
            if (BOXES == 1 && j + 1 < n[w]) {
                wait_spin(pp, G::BAR_READ + w, j, kAttendTimeout);
                logits(j + 1);
            }
            wait_spin(pp, G::BAR_VREADY + s, j / kStages, kAttendTimeout);
            wait_spin(pp, G::BAR_P + w, j, kAttendTimeout);
            tc_fence_after_sync();
            mma_sum<BOXES, kTileRows, kTileRows>(elected, pp.tmem + G::TM_O + w * G::kO, tp, base + G::OFF_V + s * G::kOperand, id_o, j % (kPieceKeys / kTileRows) != 0);
            umma_commit_e<false>(elected, pipe_bar(pp, G::BAR_O + w));
            umma_commit_e<false>(elected, pipe_bar(pp, G::BAR_VFREE + s));
            if (BOXES == 2 && j + 1 < n[w]) {
                wait_spin(pp, G::BAR_O + w, j, kAttendTimeout);              // (the logits take the place of the probabilities)
                logits(j + 1);
            }
        }
        // tiles that only the other one needs: released as they come
        for (int j = n[w]; j < tiles && !pipe_dead(pp); ++j) {
            const int s = j % kStages;
            wait_spin(pp, G::BAR_KFULL + s, j / kStages, kAttendTimeout);
            wait_spin(pp, G::BAR_VREADY + s, j / kStages, kAttendTimeout);
            if (lane == 0) {
                pipe_arrive(pp, G::BAR_KFREE + s);
                pipe_arrive(pp, G::BAR_VFREE + s);
            }
            __syncwarp();
        }
        umma_drain_w(pp, G::BAR_DRAIN + w);
        __syncwarp();
    }
    } else {
        // ------------------------------------------------------------------ softmax: thread = query
        set_regs_inc<kRowRegs>();
        const int w = warp >> 2, row = 32 * (warp & 3) + lane, token = q0 + w * kTileRows + row;
        const int limit = visible_keys(a.causal, min(token, q.count - 1), q.count, k.count);
        const uint32_t lanes = (uint32_t)(32 * (warp & 3)) << 16, elected = elect_lane();
        const uint32_t ts = pp.tmem + G::TM_S + w * G::kS + lanes, tp = pp.tmem + G::TM_P + w * G::kP + lanes, to = pp.tmem + G::TM_O + w * G::kO + lanes;
        const float c1 = a.scale * kLog2e;
        float ref = -INFINITY;
        float2 sum[2] = {};
        // a long axis: sums of the pieces so far, relative to `kept_ref` (in local memory: 512 bytes at most, touched once a piece)
        volatile float kept[64 * BOXES];
        float kept_sum = 0.f, kept_ref = -INFINITY;
        for (int j = 0; j < n[w]; ++j) {
            if (j > 0 && j % (kPieceKeys / kTileRows) == 0) {
                wait_soon(pp, G::BAR_O + w, j - 1);
                tc_fence_after_sync();
                const float f = kept_ref == ref ? 1.f : fast_exp2(kept_ref - ref);       // (no visible key so far: -inf both)
                kept_ref = ref;
                kept_sum = fmaf(kept_sum, f, (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y));
                sum[0] = sum[1] = make_float2(0.f, 0.f);
#pragma unroll 1
                for (int h = 0; h < 2 * BOXES; ++h) {
                    uint32_t o[32];
                    tmem_ld32(to + 32 * h, o);
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 32; ++i) kept[32 * h + i] = j == kPieceKeys / kTileRows ? __uint_as_float(o[i]) : fmaf(kept[32 * h + i], f, __uint_as_float(o[i]));
                }
            }
            wait_soon(pp, G::BAR_S + w, j);
            tc_fence_after_sync();
            uint32_t o[4][32];
#pragma unroll
            for (int h = 0; h < 4; ++h) tmem_ld32(ts + 32 * h, o[h]);
            tmem_ld_wait();
            float2 x[64];
#pragma unroll
            for (int i = 0; i < 64; ++i) x[i] = make_float2(__uint_as_float(o[i >> 4][2 * (i & 15)]), __uint_as_float(o[i >> 4][2 * (i & 15) + 1]));
            if (BOXES == 1) {
                tc_fence_before_sync();
                arrive_warp_e<false>(elected, pipe_bar(pp, G::BAR_READ + w));
            }
            if (j >= part[w]) {
                const int left = limit - j * kTileRows;
#pragma unroll
                for (int i = 0; i < 64; ++i) {
                    if (2 * i >= left) x[i].x = -INFINITY;
                    if (2 * i + 1 >= left) x[i].y = -INFINITY;
                }
            }
            float top[4];                                                        // (four chains: one of 64 would take longer than the rest)
#pragma unroll
            for (int i = 0; i < 4; ++i) top[i] = max_nan(x[i].x, x[i].y);
#pragma unroll
            for (int i = 4; i < 64; ++i) top[i & 3] = max3_nan(top[i & 3], x[i].x, x[i].y);
            const float m = max_nan(max3_nan(top[0], top[1], top[2]), top[3]) * c1;
            const bool grow = !(m <= ref + kSlack<T>);                                // (a NaN makes its row NaN)
            if (__any_sync(0xffffffffu, grow)) {
                const float next = grow ? m : ref, f = grow ? fast_exp2(ref - next) : 1.f;      // (exp2(-inf) = 0)
                ref = next;
                sum[0] = fmul2(sum[0], make_float2(f, f));
                sum[1] = fmul2(sum[1], make_float2(f, f));
                if (j > 0) {
                    wait_soon(pp, G::BAR_O + w, j - 1);
                    tc_fence_after_sync();
#pragma unroll
                    for (int h = 0; h < 2 * BOXES; ++h) {
                        uint32_t o[32];
                        tmem_ld32(to + 32 * h, o);
                        tmem_ld_wait();
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                        tmem_st32(to + 32 * h, o);
                    }
                }
            }
            const float nr = ref == -INFINITY ? 0.f : kHeld<T> - ref;
            uint32_t p[4][16];
            if ((w == 0 ? j > 0 && j <= n[1] : j < n[0])) bar_sync_pair(1 + (warp & 3) + 4 * w);
            // groups of eight pairs: exponentials of one, sums and roundings of the one before
            float2 v[2][8], part_sum[2];                                         // (a tile's own sum: 128 keys more on a long one would lose their last bits)
#pragma unroll
            for (int g = 0; g <= 8; ++g) {
                if (g < 8) {
                    float2 e[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) e[i] = ffma2(x[8 * g + i], make_float2(c1, c1), make_float2(nr, nr));
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[g & 1][i] = make_float2(fast_exp2(e[i].x), fast_exp2(e[i].y));
                }
                if (g == 8 && (w == 0 ? j < n[1] : j + 1 < n[0])) bar_arrive_pair(5 + (warp & 3) - 4 * w);
                if (g > 0) {
                    const int k = g - 1;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        part_sum[i & 1] = k == 0 && i < 2 ? v[0][i] : fadd2(part_sum[i & 1], v[k & 1][i]);
                        p[k >> 1][8 * (k & 1) + i] = pack2<T>(v[k & 1][i].x, v[k & 1][i].y);
                    }
                    if (BOXES == 2 && (k & 1)) tmem_st16(tp + 8 * (k - 1), p[k >> 1]);
                }
            }
            sum[0] = fadd2(sum[0], part_sum[0]);
            sum[1] = fadd2(sum[1], part_sum[1]);
            if (BOXES == 1) {
                if (j > 0) {                                                     // P V of the keys before has read its probabilities
                    wait_soon(pp, G::BAR_O + w, j - 1);
                    tc_fence_after_sync();
                }
#pragma unroll
                for (int h = 0; h < 4; ++h) tmem_st16(tp + 16 * h, p[h]);
            }
            tmem_st_wait();
            tc_fence_before_sync();
            arrive_warp_e<false>(elected, pipe_bar(pp, G::BAR_P + w));
        }
        const bool live = token < q.count;
        if (n[w]) {
            wait_soon(pp, G::BAR_O + w, n[w] - 1);
            wait_soon(pp, G::BAR_MENDED, 0);
            tc_fence_after_sync();
        }
        const bool pieces = n[w] > kPieceKeys / kTileRows;
        const float before = kept_ref == ref ? 1.f : fast_exp2(kept_ref - ref);
        const float total = fmaf(kept_sum, pieces ? before : 0.f, (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y)), inv = limit > 0 ? 1.f / total : 0.f;
        T* out = static_cast<T*>(a.out) + q.batch * a.lo.sb + head * a.lo.sh + (long long)(q.first + q0 + w * kTileRows + 32 * (warp & 3)) * a.lo.st;      // the warp's first row
        // Through the queries' place in shared memory, which nothing reads any more (rows 16 bytes a lane took 2900 cycles for 64 channels), a box at a time; a tile without
        // keys has loads of its queries in flight, maybe, but only zeros to store.
#pragma unroll
        for (int b = 0; b < BOXES; ++b) {
            unsigned char* stage = smem + G::OFF_Q + w * G::kOperand + b * kTileBytes + 32 * (warp & 3) * 128;
            if (n[w]) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t o[32];
                    tmem_ld32(to + 64 * b + 32 * h, o);
                    tmem_ld_wait();
                    if (pieces)
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(fmaf(kept[64 * b + 32 * h + i], before, __uint_as_float(o[i])));
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        float f[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) f[i] = limit > 0 ? __uint_as_float(o[8 * g + i]) * inv : 0.f;
                        if (part[0] < n[0] || part[1] < n[1])
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                if (first_bad[64 * b + 32 * h + 8 * g + i] < limit) f[i] = NAN;
                        *reinterpret_cast<uint4*>(stage + lane * 128 + (((4 * h + g) ^ (lane & 7)) << 4)) = pack16<T>(f);
                    }
                }
                __syncwarp();
            }
            const int chunk = lane & 7, rows = q.count - (q0 + w * kTileRows + 32 * (warp & 3));
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int r = 4 * i + (lane >> 3);
                if (r < rows && 64 * b + 8 * chunk < a.d)
                    *reinterpret_cast<uint4*>(out + (long long)r * a.lo.st + 64 * b + 8 * chunk) =
                        n[w] ? *reinterpret_cast<const uint4*>(stage + r * 128 + ((chunk ^ (r & 7)) << 4)) : make_uint4(0u, 0u, 0u, 0u);
            }
        }
        if (live && a.lse) a.lse[((long long)q.batch * a.heads + head) * a.N + q.first + token] = limit > 0 ? (ref - kHeld<T> + log2f(total)) * kLn2 : -INFINITY;
        tc_fence_before_sync();
    }
    __syncthreads();
    if (warp == 8) {
        tc_fence_after_sync();
        tmem_dealloc<512>(pp.tmem);
    }
}

template <typename T, int BOXES> cudaError_t run(const UmmaArgs& u, cudaStream_t st) {
    using G = FwdGeom<BOXES>;
    static std::atomic<unsigned long long> done{0};
    if (cudaError_t e = allow_smem(attend_umma_kernel<T, BOXES>, done, G::kSmem)) return e;
    attend_umma_kernel<T, BOXES><<<(unsigned)((long long)u.slots * u.a.heads), kThreads, G::kSmem, st>>>(u);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attend_umma(int dtype, const AttendArgs& a, cudaStream_t st) {
    UmmaArgs u;
    u.a = a;
    u.slots = (unsigned)slots_of(a.q_offsets != nullptr, a.sequences, a.N, 1, 2 * kTileRows);
    if (!make_row_map(&u.q, a.q, a.lq, a.batch, a.heads, a.N, a.d) || !make_row_map(&u.k, a.k, a.lk, a.batch, a.kv_heads, a.M, a.d) ||
        !make_row_map(&u.v, a.v, a.lv, a.batch, a.kv_heads, a.M, a.d))
        return cudaErrorInvalidValue;
    if (dtype == 1) return a.d <= 64 ? run<__nv_bfloat16, 1>(u, st) : run<__nv_bfloat16, 2>(u, st);
    return a.d <= 64 ? run<__half, 1>(u, st) : run<__half, 2>(u, st);
}

}  // namespace aa
