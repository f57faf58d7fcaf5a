// Softmax attention over whole sequences on mma.sync: fp32 tensors as sums of three bf16 terms, and few queries over many keys in any type; statistics for the gradients.
//
// A row is a query of one head; the heads that share keys stand side by side (row = query * group + head), so that single tokens fill a tile's rows
// with their heads.  fp32, forward: WR warps own 16 rows each, WK of them share the rows and take turns at blocks of 32 keys; logits, probabilities and
// results stay in registers, the softmax keeps a running maximum and sum in fp32.  The gradient of fp32 tensors has one kernel for both directions: rows
// are queries (dQ) or keys (dK, dV, whose columns are the queries of all heads of the group, so no share of theirs is added up elsewhere).
//
// fp32: a product of two numbers is six products of their terms (what is left out is below 2^-24), small ones first; sums over the columns leave the
// tensor core after 32 of them and join in fp32 registers, since its accumulators cut off what lies below the last bit, and in pieces of kPieceBlocks such blocks, since a
// sum of thousands loses bits in fp32, too.  Bound by the rate of mma.sync: 16 heads of
// 1024 x 1024 x 64 100 us (43 TFLOP/s of fp32), gradient 295; 8 heads of 4096 x 4096 x 128 1278 (54).
//
// Few rows on a long axis: shares of `chunk` keys a block, whose states (maximum, sum, result) a second kernel joins in order.  Bound by HBM then: one token of 16 heads over 16
// caches of 8192 to 16384 keys, 4 heads of 128, 74 us (5.6 TB/s).
#include "attend_umma.cuh"
#include "bwd_terms.cuh"

#include <algorithm>

namespace aa {

namespace {

// `COUNT` rows of DK fp32 channels (d of them exist, the others are zero) -> three planes of bf16 terms at `dst`, by THREADS threads; row(i): address or null
// (zeros).  Loads in batches of four: one at a time, their latencies were most of a small call (196 tokens, 3 heads of 64: 16.4 -> 12.3 us).
template <int DK, int THREADS, int COUNT, typename F> __device__ __forceinline__ void load_tile(int me, unsigned char* dst, uint32_t plane, int d, F row) {
    constexpr int kPitch = TileGeom<DK>::kPitch, kGroups = DK / 8, kItems = COUNT * kGroups, kBatch = 4;
#pragma unroll 1
    for (int base = me; base < kItems; base += kBatch * THREADS) {
        float4 f[kBatch][2];
#pragma unroll
        for (int n = 0; n < kBatch; ++n) {
            const int i = base + n * THREADS, c = i % kGroups * 8;
            const float* src = i < kItems ? row(i / kGroups) : nullptr;
            f[n][0] = f[n][1] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (src && c < d) f[n][0] = __ldg(reinterpret_cast<const float4*>(src + c));
            if (src && c + 4 < d) f[n][1] = __ldg(reinterpret_cast<const float4*>(src + c + 4));
        }
#pragma unroll
        for (int n = 0; n < kBatch; ++n) {
            const int i = base + n * THREADS;
            if (i >= kItems) continue;
            const float4 a = f[n][0], b = f[n][1];
            const float x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
            uint32_t w[3][4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                uint32_t t[3];
                split_pair<__nv_bfloat16, 3>(x[2 * k], x[2 * k + 1], t);
#pragma unroll
                for (int m = 0; m < 3; ++m) w[m][k] = t[m];
            }
            unsigned char* to = dst + i / kGroups * kPitch + i % kGroups * 16;
#pragma unroll
            for (int m = 0; m < 3; ++m) *reinterpret_cast<uint4*>(to + m * plane) = make_uint4(w[m][0], w[m][1], w[m][2], w[m][3]);
        }
    }
}

// s (16 x 32) = rows . columns^T; a, b: this lane's ldmatrix addresses of the warp's rows and of the block of 32 column rows
template <typename E, int NT, int DK> __device__ __forceinline__ void block_logits(float (&s)[4][4], uint32_t a, uint32_t a_plane, uint32_t b, uint32_t b_plane) {
    constexpr int P = TileGeom<DK>::kPitch;
    float small[4][4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[j][e] = small[j][e] = 0.f;
#pragma unroll
    for (int ks = 0; ks < DK / 16; ++ks) {
        uint32_t x[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n) ldsm4(x[n], a + n * a_plane + ks * 32);
#pragma unroll
        for (int j2 = 0; j2 < 2; ++j2) {
            uint32_t y[NT][4];
#pragma unroll
            for (int n = 0; n < NT; ++n) ldsm4(y[n], b + n * b_plane + j2 * 16 * P + ks * 32);
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int sum = NT - 1; sum >= 0; --sum)
#pragma unroll
                    for (int n = 0; n <= sum; ++n) mma_acc<E>(sum ? small[2 * j2 + e] : s[2 * j2 + e], x[sum - n], y[n][2 * e], y[n][2 * e + 1]);
        }
    }
    if constexpr (NT > 1) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[j][e] += small[j][e];
    }
}
// acc (16 x DK) += p (16 x 32, as terms) . columns; b: this lane's transposing ldmatrix address
template <typename E, int NT, int DK> __device__ __forceinline__ void block_product(float (&acc)[DK / 8][4], const uint32_t (&p)[NT][2][4], uint32_t b, uint32_t b_plane) {
    constexpr int P = TileGeom<DK>::kPitch;
#pragma unroll
    for (int c = 0; c < DK / 16; ++c) {
        float t[2][4];
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i) t[e][i] = 0.f;
        uint32_t y[NT][2][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) ldsm4t(y[n][ks], b + n * b_plane + ks * 16 * P + c * 32);
#pragma unroll
        for (int sum = NT - 1; sum >= 0; --sum)
#pragma unroll
            for (int n = 0; n <= sum; ++n)
#pragma unroll
                for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                    for (int e = 0; e < 2; ++e) mma_acc<E>(t[e], p[sum - n][ks], y[n][ks][2 * e], y[n][ks][2 * e + 1]);
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[2 * c + e][i] += t[e][i];
    }
}
// 16 x 32 fp32 numbers in accumulator layout -> terms as an A operand
template <typename E, int NT> __device__ __forceinline__ void block_operand(const float (&s)[4][4], uint32_t (&p)[NT][2][4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t w[NT];
            split_pair<E, NT>(s[j][2 * h], s[j][2 * h + 1], w);
#pragma unroll
            for (int n = 0; n < NT; ++n) p[n][j >> 1][(j & 1) * 2 + h] = w[n];
        }
}
// Values that are not finite, in a block of which some rows see only a part: zero in shared memory (0 * infinity is NaN), and first_bad keeps
// for every channel the first key that has one, so that the rows that do see it become NaN at the end.
template <typename E, int NT, int DK, int THREADS> __device__ void clean_values(int me, unsigned char* v, uint32_t plane, int keys, int k0, int* first_bad) {
    constexpr int kPitch = TileGeom<DK>::kPitch;
    for (int i = me; i < keys * DK; i += THREADS) {
        E* at = reinterpret_cast<E*>(v + i / DK * kPitch) + i % DK;
        bool bad = false;
#pragma unroll
        for (int n = 0; n < NT; ++n) bad |= !(fabsf(Elem<E>::to_f32(*reinterpret_cast<E*>(reinterpret_cast<unsigned char*>(at) + n * plane))) < INFINITY);
        if (bad) {
#pragma unroll
            for (int n = 0; n < NT; ++n) *reinterpret_cast<E*>(reinterpret_cast<unsigned char*>(at) + n * plane) = Elem<E>::from_f32(0.f);
            atomicMin(first_bad + i % DK, k0 + i / DK);
        }
    }
}

// Blocks of 32 columns that a sum in fp32 takes before it joins the others: equal numbers on a growing sum are rounded the same way each time, up to 2^-25 of it (65536 keys of
// 2^-35 of one: result and log-sum-exp off by 1.4e-4 without pieces, 2^20 by 2e-3).
constexpr int kPieceBlocks = 128;

// ------------------------------------------------------------------------------------------------ forward
template <int DK, int WR, int WK> struct RowsGeom {
    static constexpr int NT = 3, kRows = 16 * WR, kStep = 32 * WK, kThreads = 32 * WR * WK, kPitch = TileGeom<DK>::kPitch;
    static constexpr uint32_t kQPlane = kRows * kPitch, kPlane = kStep * kPitch;
    static constexpr int kStage = 2 * NT * (int)kPlane;
    static constexpr int kJoin = WK > 1 ? WK * kRows * (DK + 4) * 4 : 0;                  // states of the warps that share rows
    static constexpr int kRing = kStage > kJoin ? kStage : kJoin, kSmem = NT * (int)kQPlane + kRing + DK * 4;
};

// Partial state of a row and share: [row of the tensor][share]: maximum (log2 units) and sum; results behind them
__device__ __forceinline__ long long row_index(const AttendArgs& a, const Span& q, int token, int head) {
    return ((long long)q.batch * a.N + q.first + token) * a.heads + head;
}

// Two channels of row r of a tile, once its state is known: the result, or a share's partial state
template <typename T> __device__ __forceinline__ void put_pair(const AttendArgs& a, const Span& q, const Span& k, int hk, int end, const int* first_bad, int r, int c, float v0, float v1,
                                                               float sum, float top) {
    const int group = a.heads / a.kv_heads, token = r / group, head = hk * group + r % group, lim = min(end, visible_keys(a.causal, token, q.count, k.count));
    if (first_bad[c] < lim) v0 = NAN;
    if (first_bad[c + 1] < lim) v1 = NAN;
    if (gridDim.z == 1) {
        const float inv = lim > 0 ? 1.f / sum : 0.f;
        T* to = static_cast<T*>(a.out) + q.batch * a.lo.sb + head * a.lo.sh + (long long)(q.first + token) * a.lo.st + c;
        if constexpr (sizeof(T) == 2) *reinterpret_cast<uint32_t*>(to) = pack2<T>(v0 * inv, v1 * inv);
        else *reinterpret_cast<float2*>(to) = make_float2(v0 * inv, v1 * inv);
        if (c == 0 && a.lse) a.lse[((long long)q.batch * a.heads + head) * a.N + q.first + token] = lim > 0 ? (top + log2f(sum)) * kLn2 : -INFINITY;
    } else {
        const long long at = row_index(a, q, token, head) * gridDim.z + blockIdx.z, all = (long long)a.batch * a.N * a.heads * gridDim.z;
        *reinterpret_cast<float2*>(a.ws + (2 * all + 3) / 4 * 4 + at * a.d + c) = make_float2(v0, v1);
        if (c == 0) *reinterpret_cast<float2*>(a.ws + 2 * at) = make_float2(top, sum);
    }
}
// The states of WK warps that share rows meet in shared memory: [WK][ROWS][DK + 4], results, maximum, sum
template <typename T, int DK, int ROWS, int WK, int THREADS>
__device__ __forceinline__ void join_warps(const AttendArgs& a, const Span& q, const Span& k, int hk, int end, const int* first_bad, const float* join, int row0, int rows) {
    for (int i = threadIdx.x; i < ROWS * (DK / 2); i += THREADS) {
        const int r = i / (DK / 2), c = i % (DK / 2) * 2;
        if (row0 + r >= rows || c >= a.d) continue;
        float top = -INFINITY, sum = 0.f, v0 = 0.f, v1 = 0.f;
#pragma unroll
        for (int w = 0; w < WK; ++w) top = fmaxf(top, join[(w * ROWS + r) * (DK + 4) + DK]);
        const float b = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int w = 0; w < WK; ++w) {
            const float* s = join + (w * ROWS + r) * (DK + 4);
            const float f = fast_exp2(s[DK] - b);
            sum = fmaf(f, s[DK + 1], sum);
            v0 = fmaf(f, s[c], v0);
            v1 = fmaf(f, s[c + 1], v1);
        }
        put_pair<T>(a, q, k, hk, end, first_bad, row0 + r, c, v0, v1, sum, top);
    }
}

template <int DK, int WR, int WK>
__global__ void __launch_bounds__(32 * WR * WK) attend_rows_kernel(const __grid_constant__ AttendArgs a) {
    using T = float;
    using E = __nv_bfloat16;
    using G = RowsGeom<DK, WR, WK>;
    constexpr int NT = G::NT, P = G::kPitch;
    extern __shared__ __align__(128) unsigned char smem[];
    unsigned char* ring = smem + NT * G::kQPlane;
    int* first_bad = reinterpret_cast<int*>(smem + NT * G::kQPlane + G::kRing);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, wr = warp % WR, wk = warp / WR, g = lane >> 2, t = lane & 3;
    const int group = a.heads / a.kv_heads, hk = blockIdx.y;
    int seq, tile;
    if (!find_slot(a.q_offsets, a.sequences, a.N, group, G::kRows, blockIdx.x, &seq, &tile)) return;
    const Span q = span_of(a.q_offsets, a.q_lengths, a.N, seq), k = span_of(a.k_offsets, a.k_lengths, a.M, seq);
    const int rows = q.count * group, row0 = tile * G::kRows;      // (the host refuses more than 31 bits of them)
    if (row0 >= rows) return;
    const int last = min(rows, row0 + G::kRows) - 1;
    const int k_all = visible_keys(a.causal, last / group, q.count, k.count);            // of the tile's last query
    const int share = blockIdx.z, begin = (int)min((long long)k_all, (long long)share * a.chunk);
    const int end = (int)min((long long)k_all, (long long)begin + a.chunk);
    if (share > 0 && begin >= k_all) return;
    const int k_whole = visible_keys(a.causal, row0 / group, q.count, k.count);    // keys that every row sees

    const T* kp = static_cast<const T*>(a.k) + k.batch * a.lk.sb + hk * a.lk.sh + (long long)k.first * a.lk.st;
    const T* vp = static_cast<const T*>(a.v) + k.batch * a.lv.sb + hk * a.lv.sh + (long long)k.first * a.lv.st;
    load_tile<DK, G::kThreads, G::kRows>(tid, smem, G::kQPlane, a.d, [&](int r) -> const T* {
        const int i = row0 + r;
        return i < rows ? static_cast<const T*>(a.q) + q.batch * a.lq.sb + (hk * group + i % group) * a.lq.sh + (long long)(q.first + i / group) * a.lq.st : nullptr;
    });
    for (int c = tid; c < DK; c += G::kThreads) first_bad[c] = INT_MAX;
    const int steps = (end - begin + G::kStep - 1) / G::kStep;
    // warps that share their keys fetch them together; one that has its own (WK > 1) waits for no other
    constexpr int LOADERS = WK > 1 ? 32 : G::kThreads, OWN = WK > 1 ? 32 : G::kStep;
    const int me = WK > 1 ? lane : tid;
    unsigned char* mine = ring + (WK > 1 ? wk * 32 * P : 0);
    auto meet = [&] {
        if (WK > 1) __syncwarp();
        else __syncthreads();
    };

    int limit[2], row[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        row[h] = row0 + wr * 16 + g + 8 * h;
        limit[h] = row[h] < rows ? min(end, visible_keys(a.causal, row[h] / group, q.count, k.count)) : 0;
    }
    const float c1 = a.scale * kLog2e;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, o[DK / 8][4];
#pragma unroll
    for (int c = 0; c < DK / 8; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[c][e] = 0.f;
    __syncthreads();                               // (the queries, and first_bad)
    const uint32_t qa = smem_u32(smem) + wr * 16 * P + val_lane_offset<DK>(lane);

    // a long axis: sums of the pieces so far, relative to kept_m (in local memory, touched once a piece)
    volatile float kept[DK / 8][4];
    float kept_m[2] = {-INFINITY, -INFINITY}, kept_l[2] = {0.f, 0.f};
    int pieces = 0;
    for (int s = 0; s < steps; ++s) {
        const int k0 = begin + s * G::kStep + (WK > 1 ? wk * 32 : 0);
        if (k0 >= end) break;                      // (of a warp with its own keys)
        if (s && s % kPieceBlocks == 0) {
            float f[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                f[h] = kept_m[h] == m[h] ? 1.f : fast_exp2(kept_m[h] - m[h]);          // (no visible key so far: -inf both)
                kept_m[h] = m[h];
                kept_l[h] = fmaf(kept_l[h], f[h], l[h]);
                l[h] = 0.f;
            }
#pragma unroll
            for (int c = 0; c < DK / 8; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    kept[c][e] = pieces ? fmaf(kept[c][e], f[e >> 1], o[c][e]) : o[c][e];
                    o[c][e] = 0.f;
                }
            ++pieces;
        }
        if (s) meet();
        load_tile<DK, LOADERS, OWN>(me, mine, G::kPlane, a.d, [&](int r) -> const T* { return k0 + r < end ? kp + (long long)(k0 + r) * a.lk.st : nullptr; });
        load_tile<DK, LOADERS, OWN>(me, mine + NT * G::kPlane, G::kPlane, a.d, [&](int r) -> const T* { return k0 + r < end ? vp + (long long)(k0 + r) * a.lv.st : nullptr; });
        meet();
        if (k0 + OWN > k_whole) {
            clean_values<E, NT, DK, LOADERS>(me, mine + NT * G::kPlane, G::kPlane, min(OWN, end - k0), k0, first_bad);
            meet();
        }
        const uint32_t kb = smem_u32(mine);
        float x[4][4];
        block_logits<E, NT, DK>(x, qa, G::kQPlane, kb + key_lane_offset<DK>(lane), G::kPlane);
        if (k0 + 32 > min(limit[0], limit[1])) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (k0 + 8 * j + 2 * t + (e & 1) >= limit[e >> 1]) x[j][e] = -INFINITY;
        }
        float f[2], base[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float n = -INFINITY;
#pragma unroll
            for (int j = 0; j < 4; ++j) n = max3(n, x[j][2 * h], x[j][2 * h + 1]);
            n = fmaxf(m[h], quad_max(n) * c1);
            base[h] = n == -INFINITY ? 0.f : n;                          // (no visible key so far)
            f[h] = m[h] == -INFINITY ? 0.f : fast_exp2(m[h] - base[h]);
            m[h] = n;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[j][e] = fast_exp2(fmaf(x[j][e], c1, -base[e >> 1]));
#pragma unroll
        for (int h = 0; h < 2; ++h) {              // (the block's own sum first: eight small numbers on a long one would lose their last bits)
            float t = x[0][2 * h] + x[0][2 * h + 1];
#pragma unroll
            for (int j = 1; j < 4; ++j) t += x[j][2 * h] + x[j][2 * h + 1];
            l[h] = fmaf(l[h], f[h], t);
        }
#pragma unroll
        for (int c = 0; c < DK / 8; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[c][e] *= f[e >> 1];
        uint32_t p[NT][2][4];
        block_operand<E, NT>(x, p);
        block_product<E, NT, DK>(o, p, kb + NT * G::kPlane + val_lane_offset<DK>(lane), G::kPlane);
    }
    if (pieces) {
        float f[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            f[h] = kept_m[h] == m[h] ? 1.f : fast_exp2(kept_m[h] - m[h]);
            l[h] = fmaf(kept_l[h], f[h], l[h]);
        }
#pragma unroll
        for (int c = 0; c < DK / 8; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[c][e] = fmaf(kept[c][e], f[e >> 1], o[c][e]);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) l[h] = quad_sum(l[h]);
    __syncthreads();                               // (first_bad is complete; the ring may be written)
    auto finish = [&](int r, int c, float v0, float v1, float sum, float top) { put_pair<T>(a, q, k, hk, end, first_bad, r, c, v0, v1, sum, top); };
    if constexpr (WK == 1) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (row[h] >= rows) continue;
#pragma unroll
            for (int c = 0; c < DK / 8; ++c)
                if (8 * c + 2 * t < a.d) finish(row[h], 8 * c + 2 * t, o[c][2 * h], o[c][2 * h + 1], l[h], m[h]);
        }
    } else {
        float* join = reinterpret_cast<float*>(ring);                    // [WK][rows][DK + 4]: results, maximum, sum
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float* to = join + (wk * G::kRows + wr * 16 + g + 8 * h) * (DK + 4);
#pragma unroll
            for (int c = 0; c < DK / 8; ++c) *reinterpret_cast<float2*>(to + 8 * c + 2 * t) = make_float2(o[c][2 * h], o[c][2 * h + 1]);
            if (t == 0) { to[DK] = m[h]; to[DK + 1] = l[h]; }
        }
        __syncthreads();
        join_warps<T, DK, G::kRows, WK, G::kThreads>(a, q, k, hk, end, first_bad, join, row0, rows);
    }
}

// Few queries over many keys, 16-bit types: sixteen rows a block, four warps that take turns at sixteen keys each.  Bound by HBM: every warp has a ring of its own that
// TMA fills (100 KB in flight a SM; a turn ahead in registers was 64 KB and 4.5 TB/s), takes its keys and values from there into registers, 16 bytes a lane, and
// hands the stage back before it computes:
//   logits   lane (g, t) takes the channels 32 i + 8 t .. + 7 of key g: two steps of the product's sum, whose channels may come in any order if the queries' do so, too
//   P V      lane (g, t) takes the channels 8 g .. 8 g + 7 of the keys 2 t, 2 t + 1, 2 t + 8, 2 t + 9; byte permutes make the pairs of keys that the product wants,
//            and column n of its tile i is channel 8 n + i
// The exponents' reference moves only when a logit exceeds it by more than kSlack.
constexpr int kFewWarps = 4, kFewStages = 3, kFewKeys = 16;
struct FewArgs {
    AttendArgs a;
    RowMap k, v;
};
template <int DK> struct FewKV {
    uint4 k[2][DK / 32], v[4][DK / 64];
};
template <typename T, int DK> __global__ void __launch_bounds__(32 * kFewWarps) attend_few_kernel(const __grid_constant__ FewArgs f) {
    constexpr int WK = kFewWarps, kRows = 16, KI = DK / 32, VI = DK / 64, kBox = kFewKeys * 128, kStage = 2 * VI * kBox;
    const AttendArgs& a = f.a;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    float* join = reinterpret_cast<float*>(smem);                       // [WK][16][DK + 4], once the rings are done with
    __shared__ int first_bad[DK];
    __shared__ __align__(8) unsigned long long bars[WK * kFewStages];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const int group = a.heads / a.kv_heads, hk = blockIdx.y;
    int seq, tile;
    if (!find_slot(a.q_offsets, a.sequences, a.N, group, kRows, blockIdx.x, &seq, &tile)) return;
    const Span q = span_of(a.q_offsets, a.q_lengths, a.N, seq), k = span_of(a.k_offsets, a.k_lengths, a.M, seq);
    const int rows = q.count * group, row0 = tile * kRows;
    if (row0 >= rows) return;
    const int last = min(rows, row0 + kRows) - 1, k_all = visible_keys(a.causal, last / group, q.count, k.count);
    const int begin = (int)min((long long)k_all, (long long)blockIdx.z * a.chunk), end = (int)min((long long)k_all, (long long)begin + a.chunk);
    if (blockIdx.z > 0 && begin >= k_all) return;
    const int k_whole = visible_keys(a.causal, row0 / group, q.count, k.count);          // keys that every row sees
    for (int c = tid; c < DK; c += 32 * WK) first_bad[c] = INT_MAX;
    pdl_release_next();                            // (of a launch that does not depend on this one nothing is said by it)
    if (tid == 0) {
        for (int i = 0; i < WK * kFewStages; ++i) mbar_init(smem_u32(bars + i), 1);
        mbar_fence_init();
    }
    __syncthreads();
    const uint32_t ring = smem_u32(smem) + warp * kFewStages * kStage, bar = smem_u32(bars + warp * kFewStages);
    const int k0 = begin + kFewKeys * warp, turns = k0 < end ? (end - k0 + WK * kFewKeys - 1) / (WK * kFewKeys) : 0;
    auto fetch = [&](int i) {                                           // (by one lane)
        const uint32_t to = ring + (i % kFewStages) * kStage, full = bar + 8 * (i % kFewStages);
        const int row = k.first + k0 + i * WK * kFewKeys;
        mbar_arrive_expect_tx(full, kStage);
#pragma unroll
        for (int b = 0; b < VI; ++b) {
            load_rows(to + b * kBox, f.k, 64 * b, row, hk, k.batch, full);
            load_rows(to + (VI + b) * kBox, f.v, 64 * b, row, hk, k.batch, full);
        }
    };
    if (lane == 0)
        for (int i = 0; i < min(turns, kFewStages); ++i) fetch(i);

    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
    uint4 x[2][KI];                                                     // queries: rows g and g + 8, channels 32 i + 8 t
    int limit[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int r = row0 + g + 8 * h;
        limit[h] = r < rows ? min(end, visible_keys(a.causal, r / group, q.count, k.count)) : 0;
        const T* src = static_cast<const T*>(a.q) + q.batch * a.lq.sb + (hk * group + r % group) * a.lq.sh + (long long)(q.first + r / group) * a.lq.st;
#pragma unroll
        for (int i = 0; i < KI; ++i) x[h][i] = r < rows && 32 * i + 8 * t < a.d ? __ldg(reinterpret_cast<const uint4*>(src + 32 * i + 8 * t)) : zero;
    }
    auto take = [&](FewKV<DK>& f, int i) {
        const unsigned char* from = smem + (ring - smem_u32(smem)) + (i % kFewStages) * kStage;
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int c = 0; c < KI; ++c) f.k[n][c] = *reinterpret_cast<const uint4*>(from + (c >> 1) * kBox + (8 * n + g) * 128 + (((4 * (c & 1) + t) ^ g) << 4));
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            const int key = 2 * t + (n & 1) + 8 * (n >> 1);
#pragma unroll
            for (int c = 0; c < VI; ++c) f.v[n][c] = *reinterpret_cast<const uint4*>(from + (VI + c) * kBox + key * 128 + ((g ^ (key & 7)) << 4));
        }
    };
    const float c1 = a.scale * kLog2e;
    float ref[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, o[VI][8][4];
#pragma unroll
    for (int i = 0; i < VI; ++i)
#pragma unroll
        for (int n = 0; n < 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[i][n][e] = 0.f;
    auto use = [&](FewKV<DK>& f, int k0) {
        float s[2][4];
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int i = 0; i < KI; ++i) {
                const uint32_t a0[4] = {x[0][i].x, x[1][i].x, x[0][i].y, x[1][i].y}, a1[4] = {x[0][i].z, x[1][i].z, x[0][i].w, x[1][i].w};
                if (i == 0) mma_set<T>(s[n], a0, f.k[n][i].x, f.k[n][i].y);
                else mma_acc<T>(s[n], a0, f.k[n][i].x, f.k[n][i].y);
                mma_acc<T>(s[n], a1, f.k[n][i].z, f.k[n][i].w);
            }
        if (k0 + 16 > k_whole || k0 + 16 > end) {                       // (some rows do not see all: see clean_values)
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (k0 + 8 * n + 2 * t + (e & 1) >= limit[e >> 1]) s[n][e] = -INFINITY;
#pragma unroll
            for (int n = 0; n < 4; ++n)
#pragma unroll
                for (int i = 0; i < VI; ++i) {
                    if (k0 + 2 * t + (n & 1) + 8 * (n >> 1) >= end) f.v[n][i] = zero;
                    uint32_t* w = reinterpret_cast<uint32_t*>(&f.v[n][i]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float2 p = unpack2<T>(w[e >> 1]);
                        if (!(fabsf(e & 1 ? p.y : p.x) < INFINITY)) {
                            w[e >> 1] &= e & 1 ? 0xffffu : 0xffff0000u;
                            atomicMin(first_bad + 64 * i + 8 * g + e, k0 + 2 * t + (n & 1) + 8 * (n >> 1));
                        }
                    }
                }
        }
        float m[2];
        bool grow = false;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            m[h] = fmaxf(fmaxf(s[0][2 * h], s[0][2 * h + 1]), fmaxf(s[1][2 * h], s[1][2 * h + 1])) * c1;
            grow |= m[h] > ref[h] + kSlack<T>;
        }
        if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float top = quad_max(m[h]);
                if (!(top > ref[h] + kSlack<T>)) continue;                 // (the same of a row's four lanes; no shuffles below)
                const float f = fast_exp2(ref[h] - top);                // (0 of a row without a key so far)
                ref[h] = top;
                l[h] *= f;
#pragma unroll
                for (int i = 0; i < VI; ++i)
#pragma unroll
                    for (int n = 0; n < 8; ++n) {
                        o[i][n][2 * h] *= f;
                        o[i][n][2 * h + 1] *= f;
                    }
            }
        }
        const float base[2] = {ref[0] == -INFINITY ? 0.f : ref[0] - kHeld<T>, ref[1] == -INFINITY ? 0.f : ref[1] - kHeld<T>};
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[n][e] = fast_exp2(fmaf(s[n][e], c1, -base[e >> 1]));
#pragma unroll
        for (int h = 0; h < 2; ++h) l[h] += (s[0][2 * h] + s[0][2 * h + 1]) + (s[1][2 * h] + s[1][2 * h + 1]);
        const uint32_t p[4] = {pack2<T>(s[0][0], s[0][1]), pack2<T>(s[0][2], s[0][3]), pack2<T>(s[1][0], s[1][1]), pack2<T>(s[1][2], s[1][3])};
#pragma unroll
        for (int i = 0; i < VI; ++i) {
            const uint32_t *v0 = reinterpret_cast<const uint32_t*>(&f.v[0][i]), *v1 = reinterpret_cast<const uint32_t*>(&f.v[1][i]);
            const uint32_t *v2 = reinterpret_cast<const uint32_t*>(&f.v[2][i]), *v3 = reinterpret_cast<const uint32_t*>(&f.v[3][i]);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                mma_acc<T>(o[i][2 * w], p, __byte_perm(v0[w], v1[w], 0x5410), __byte_perm(v2[w], v3[w], 0x5410));
                mma_acc<T>(o[i][2 * w + 1], p, __byte_perm(v0[w], v1[w], 0x7632), __byte_perm(v2[w], v3[w], 0x7632));
            }
        }
    };
    for (int i = 0; i < turns; ++i) {
        FewKV<DK> kv;
        if (!mbar_wait_bounded(bar + 8 * (i % kFewStages), (i / kFewStages) & 1, 1u << 22)) {
            if (a.status) atomicCAS(a.status, 0, kAttendTimeout);
            for (int n = i; n < min(turns, i + kFewStages); ++n) mbar_wait_bounded(bar + 8 * (n % kFewStages), (n / kFewStages) & 1, 1u << 22);      // (copies in flight)
            break;
        }
        take(kv, i);
        // The next copy must not overtake the loads: a vote on what they brought waits until it is in registers.
        uint32_t words = 0;
#pragma unroll
        for (int n = 0; n < 4; ++n) {
#pragma unroll
            for (int c = 0; c < VI; ++c) words |= kv.v[n][c].x;
#pragma unroll
            for (int c = 0; c < KI; ++c) words |= kv.k[n & 1][c].x;
        }
        words = __ballot_sync(0xffffffffu, words != 0);
        asm volatile("" ::"r"(words) : "memory");
        if (lane == 0 && i + kFewStages < turns) fetch(i + kFewStages);
        use(kv, k0 + i * WK * kFewKeys);
    }
    __syncthreads();                               // (the rings are done with)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        l[h] = quad_sum(l[h]);
        float* to = join + (warp * kRows + g + 8 * h) * (DK + 4);
#pragma unroll
        for (int i = 0; i < VI; ++i)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float4* d = reinterpret_cast<float4*>(to + 64 * i + 16 * t + 8 * e);
                d[0] = make_float4(o[i][0][2 * h + e], o[i][1][2 * h + e], o[i][2][2 * h + e], o[i][3][2 * h + e]);
                d[1] = make_float4(o[i][4][2 * h + e], o[i][5][2 * h + e], o[i][6][2 * h + e], o[i][7][2 * h + e]);
            }
        if (t == 0) {
            to[DK] = ref[h] - kHeld<T>;            // (what the exponents are relative to)
            to[DK + 1] = l[h];
        }
    }
    __syncthreads();
    join_warps<T, DK, kRows, WK, 32 * WK>(a, q, k, hk, end, first_bad, join, row0, rows);
}

// Joins the states of a row's shares: a block a row, its four warps take every fourth share, a lane four channels; the order is fixed.
template <typename T> __global__ void __launch_bounds__(128) attend_join_kernel(const __grid_constant__ AttendArgs a, int shares) {
    __shared__ float4 part[4][32];
    __shared__ float sums[4];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, group = a.heads / a.kv_heads, hk = blockIdx.y;
    int seq, r;
    const bool found = find_slot(a.q_offsets, a.sequences, a.N, group, 1, blockIdx.x, &seq, &r);
    const Span q = span_of(a.q_offsets, a.q_lengths, a.N, seq), k = span_of(a.k_offsets, a.k_lengths, a.M, seq);
    if (!found || r >= q.count * group) return;
    // (shares that a row's tile of 16 has: some may hold no key of this row, with a sum of zero)
    const int last = min(q.count * group, r / 16 * 16 + 16) - 1, k_all = visible_keys(a.causal, last / group, q.count, k.count);
    const int live = max(1, (int)((k_all + (long long)a.chunk - 1) / a.chunk));
    const int token = r / group, head = hk * group + r % group;
    const long long all = (long long)a.batch * a.N * a.heads * shares, at = row_index(a, q, token, head) * shares;
    const float2* state = reinterpret_cast<const float2*>(a.ws) + at;
    const float* acc = a.ws + (2 * all + 3) / 4 * 4 + at * a.d + 4 * lane;
    const bool mine = 4 * lane < a.d;
    pdl_wait_prior();
    float top = -INFINITY;
    for (int s = lane; s < live; s += 32) top = fmaxf(top, state[s].x);
#pragma unroll
    for (int i = 16; i; i >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, i));
    const float b = top == -INFINITY ? 0.f : top;
    float sum = 0.f;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int s = warp; s < live; s += 4) {
        const float2 st = state[s];
        const float f = fast_exp2(st.x - b);
        const float4 w = mine ? *reinterpret_cast<const float4*>(acc + (long long)s * a.d) : make_float4(0.f, 0.f, 0.f, 0.f);
        sum = fmaf(f, st.y, sum);
        v.x = fmaf(f, w.x, v.x); v.y = fmaf(f, w.y, v.y); v.z = fmaf(f, w.z, v.z); v.w = fmaf(f, w.w, v.w);
    }
    part[warp][lane] = v;
    if (lane == 0) sums[warp] = sum;
    __syncthreads();
    if (warp) return;
    sum = (sums[0] + sums[1]) + (sums[2] + sums[3]);
#pragma unroll
    for (int w = 1; w < 4; ++w) {
        v.x += part[w][lane].x; v.y += part[w][lane].y; v.z += part[w][lane].z; v.w += part[w][lane].w;
    }
    const bool some = visible_keys(a.causal, token, q.count, k.count) > 0;
    const float inv = some ? 1.f / sum : 0.f;
    if (mine) {
        T* to = static_cast<T*>(a.out) + q.batch * a.lo.sb + head * a.lo.sh + (long long)(q.first + token) * a.lo.st + 4 * lane;
        if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(to) = make_uint2(pack2<T>(v.x * inv, v.y * inv), pack2<T>(v.z * inv, v.w * inv));
        else *reinterpret_cast<float4*>(to) = make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
    }
    if (lane == 0 && a.lse) a.lse[((long long)q.batch * a.heads + head) * a.N + q.first + token] = some ? (top + log2f(sum)) * kLn2 : -INFINITY;
}

template <typename T> cudaError_t run_join(const AttendArgs& a, int shares, cudaStream_t st) {
    const long long slots = slots_of(a.q_offsets != nullptr, a.sequences, a.N, a.heads / a.kv_heads, 1);
    return launch_dependent(attend_join_kernel<T>, dim3((unsigned)slots, a.kv_heads), 128, 0, st, a, shares);
}
template <int DK, int WR, int WK> cudaError_t run_rows(const AttendArgs& a, int shares, cudaStream_t st) {
    using G = RowsGeom<DK, WR, WK>;
    static std::atomic<unsigned long long> done{0};
    if (cudaError_t e = allow_smem(attend_rows_kernel<DK, WR, WK>, done, G::kSmem)) return e;
    const long long slots = slots_of(a.q_offsets != nullptr, a.sequences, a.N, a.heads / a.kv_heads, G::kRows);
    attend_rows_kernel<DK, WR, WK><<<dim3((unsigned)slots, a.kv_heads, shares), G::kThreads, G::kSmem, st>>>(a);
    if (cudaError_t e = cudaGetLastError()) return e;
    return shares > 1 ? run_join<float>(a, shares, st) : cudaSuccess;
}
template <typename T, int DK> cudaError_t run_few(const AttendArgs& a, int shares, cudaStream_t st) {
    constexpr int kRing = kFewWarps * kFewStages * kFewKeys * 4 * DK, kJoin = kFewWarps * 16 * (DK + 4) * 4, kSmem = (kRing > kJoin ? kRing : kJoin) + 1024;
    FewArgs f;
    f.a = a;
    if (!make_row_map(&f.k, a.k, a.lk, a.batch, a.kv_heads, a.M, a.d, kFewKeys) || !make_row_map(&f.v, a.v, a.lv, a.batch, a.kv_heads, a.M, a.d, kFewKeys)) return cudaErrorInvalidValue;
    static std::atomic<unsigned long long> done{0};
    if (cudaError_t e = allow_smem(attend_few_kernel<T, DK>, done, kSmem)) return e;
    const long long slots = slots_of(a.q_offsets != nullptr, a.sequences, a.N, a.heads / a.kv_heads, 16);
    attend_few_kernel<T, DK><<<dim3((unsigned)slots, a.kv_heads, shares), 32 * kFewWarps, kSmem, st>>>(f);
    if (cudaError_t e = cudaGetLastError()) return e;
    return shares > 1 ? run_join<T>(a, shares, st) : cudaSuccess;
}

// Few rows a sequence: sixteen of them a block, whose four warps take turns at the keys.
bool few_rows(const AttendArgs& a) {
    const long long rows = (long long)a.N * (a.heads / a.kv_heads), sequences = a.q_offsets ? a.sequences : 1;
    return rows <= 16 * sequences && rows < (1LL << 28);
}
// Shares of the keys where blocks are too few to fill the GPU
int shares_of(const AttendArgs& a, bool few_16, int sm_count, int* chunk) {
    *chunk = std::max(1, a.M);
    if (!few_rows(a)) return 1;
    const long long blocks = slots_of(a.q_offsets != nullptr, a.sequences, a.N, a.heads / a.kv_heads, 16) * a.kv_heads;
    // One wave of blocks (two an SM; up to 64 channels of 16 bits, three): a block's start and end cost as much as some 1000 keys.  16 caches of up to 16384 keys, 4 heads
    // of keys of 128: one an SM 114 us, 2 75, 3 84, 4 83, 12 85; 8 heads of 64 over 8192: 70, 49, 49, 51, 51; one cache of 65536, 8 heads of 128: 56, 54, 64, 60, 74.
    // fp32, bound by its loads (with 128 channels one block fits an SM): 567, 574, 473, 418, 441 (lengths even out); 291, 296, 297, 300, 293; 265, 263, 283, 272, 312.
    const long long want = std::max(1LL, (a.d <= 64 && few_16 ? 3LL : 2LL) * sm_count / blocks);
    long long c = (a.M + want - 1) / want;
    c = std::min(std::max(256LL, (c + 127) / 128 * 128), 4LL * kPieceKeys);      // (four warps take a piece each, see kPieceKeys)
    *chunk = (int)std::min<long long>(c, a.M);
    return (a.M + *chunk - 1) / *chunk;
}

template <int WR, int WK> cudaError_t run_rows_of(const AttendArgs& a, int shares, cudaStream_t st) {
    if (a.d <= 32) return run_rows<32, WR, WK>(a, shares, st);
    if (a.d <= 64) return run_rows<64, WR, WK>(a, shares, st);
    if (a.d <= 96) return run_rows<96, WR, WK>(a, shares, st);
    return run_rows<128, WR, WK>(a, shares, st);
}

// ------------------------------------------------------------------------------------------------ backward
// (log2-sum-exp, D) of every row of a sequence, eight lanes a row, and for f16 what the powers of two that hold small gradients are made of: the norm of
// every row of dO, the largest of a sequence and head of keys, and the largest of the rows of V (blocks past the first `q_slots`).
template <typename T> __global__ void __launch_bounds__(256) attend_dot_kernel(const __grid_constant__ AttendArgs a, unsigned q_slots) {
    constexpr int V = Elem<T>::kVec;
    constexpr bool kNorms = is_f16<T>;
    const int group = a.heads / a.kv_heads, hk = blockIdx.y, lane8 = threadIdx.x & 7;
    const bool values = blockIdx.x >= q_slots;
    int seq, tile;
    if (!(values ? find_slot(a.k_offsets, a.sequences, a.M, 1, kDotRows, blockIdx.x - q_slots, &seq, &tile)
                 : find_slot(a.q_offsets, a.sequences, a.N, group, kDotRows, blockIdx.x, &seq, &tile))) return;
    const Span r = values ? span_of(a.k_offsets, a.k_lengths, a.M, seq) : span_of(a.q_offsets, a.q_lengths, a.N, seq);
    const int rows = r.count * (values ? 1 : group), first = tile * kDotRows;
    if (first >= rows) return;
    float most = 0.f;
    for (int i = first + (threadIdx.x >> 3); i < min(rows, first + kDotRows); i += 32) {       // (lanes of a row stay together)
        const int head = values ? hk : hk * group + i % group, at = r.first + (values ? i : i / group);
        const T* g = values ? static_cast<const T*>(a.v) + r.batch * a.lv.sb + head * a.lv.sh + (long long)at * a.lv.st
                            : static_cast<const T*>(a.dout) + r.batch * a.ldo.sb + head * a.ldo.sh + (long long)at * a.ldo.st;
        const T* o = values ? g : static_cast<const T*>(a.out) + r.batch * a.lo.sb + head * a.lo.sh + (long long)at * a.lo.st;
        float sum = 0.f, square = 0.f;
        for (int c = lane8 * V; c < a.d; c += 8 * V) {
            float x[V], y[V];
            unpack16<T>(__ldg(reinterpret_cast<const uint4*>(g + c)), x);
            unpack16<T>(__ldg(reinterpret_cast<const uint4*>(o + c)), y);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                sum = fmaf(x[e], y[e], sum);
                square = fmaf(x[e], x[e], square);
            }
        }
        const unsigned mask = 0xffu << (threadIdx.x & 24);
#pragma unroll
        for (int e = 4; e; e >>= 1) {
            sum += __shfl_xor_sync(mask, sum, e);
            if (kNorms) square += __shfl_xor_sync(mask, square, e);
        }
        if (lane8 == 0) {
            if (!values) {
                const long long row = ((long long)r.batch * a.heads + head) * a.N + at;
                reinterpret_cast<float2*>(a.ws)[row] = make_float2(a.lse[row] * kLog2e, sum);
                if (kNorms) grad_norms(a)[row] = sqrtf(square);
            }
            if (square < INFINITY) most = fmaxf(most, sqrtf(square));
        }
    }
    if (kNorms && most > 0.f) atomicMax(grad_most(a, seq, hk) + (values ? 1 : 0), __float_as_uint(most));      // (positive numbers keep their order; any order of arrival)
}

template <int DK> struct GradGeom {
    static constexpr int NT = 3, kRows = 64, kStep = 32, kPitch = TileGeom<DK>::kPitch;
    static constexpr uint32_t kRowPlane = kRows * kPitch, kPlane = kStep * kPitch;
    static constexpr int kSmem = 2 * NT * (int)(kRowPlane + kPlane) + kStep * 8;
};

// KEYS: rows are keys (x = K, y = V), columns queries (u = Q, w = dO); else rows are queries (x = Q, y = dO), columns keys (u = K, w = V).
// LONG: sums may be longer than a piece (the others do without its registers: 8 heads of 4096 x 4096 x 128 6.04 ms with them, 5.74 without).
template <int DK, bool KEYS, bool LONG>
__global__ void __launch_bounds__(128) attend_grad_kernel(const __grid_constant__ AttendArgs a) {
    using T = float;
    using G = GradGeom<DK>;
    using E = __nv_bfloat16;
    constexpr int NT = G::NT, P = G::kPitch;
    extern __shared__ __align__(128) unsigned char smem[];
    unsigned char *xs = smem, *ys = xs + NT * G::kRowPlane, *us = ys + NT * G::kRowPlane, *ws = us + NT * G::kPlane;
    float2* stats = reinterpret_cast<float2*>(ws + NT * G::kPlane);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const int group = a.heads / a.kv_heads, hk = blockIdx.y;
    int seq, tile;
    if (!find_slot(KEYS ? a.k_offsets : a.q_offsets, a.sequences, KEYS ? a.M : a.N, KEYS ? 1 : group, G::kRows, blockIdx.x, &seq, &tile)) return;
    const Span q = span_of(a.q_offsets, a.q_lengths, a.N, seq), k = span_of(a.k_offsets, a.k_lengths, a.M, seq);
    const int queries = q.count * group, rows = KEYS ? k.count : queries, row0 = tile * G::kRows;      // (the host refuses more than 31 bits of them)
    if (row0 >= rows) return;
    auto query = [&](const void* p, const TokLayout& l, int i) {
        return static_cast<const T*>(p) + q.batch * l.sb + (hk * group + i % group) * l.sh + (long long)(q.first + i / group) * l.st;
    };
    auto key = [&](const void* p, const TokLayout& l, int j) { return static_cast<const T*>(p) + k.batch * l.sb + hk * l.sh + (long long)(k.first + j) * l.st; };
    auto stat = [&](int i) {
        return __ldg(reinterpret_cast<const float2*>(a.ws) + ((long long)q.batch * a.heads + hk * group + i % group) * a.N + q.first + i / group);
    };
    load_tile<DK, 128, G::kRows>(tid, xs, G::kRowPlane, a.d, [&](int r) -> const T* { return row0 + r < rows ? (KEYS ? key(a.k, a.lk, row0 + r) : query(a.q, a.lq, row0 + r)) : nullptr; });
    load_tile<DK, 128, G::kRows>(tid, ys, G::kRowPlane, a.d, [&](int r) -> const T* { return row0 + r < rows ? (KEYS ? key(a.v, a.lv, row0 + r) : query(a.dout, a.ldo, row0 + r)) : nullptr; });
    // columns that some row of the tile meets
    int begin = 0, end;
    if (KEYS) {
        if (a.causal) begin = max(0, row0 - k.count + q.count) * group;
        end = queries;
    } else {
        end = visible_keys(a.causal, ((min(rows, row0 + G::kRows) - 1) / group), q.count, k.count);
    }
    const float c1 = a.scale * kLog2e;
    int row[2], limit[2];                          // rows are queries: the keys that they see; keys: the first column that sees them
    float2 st[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        row[h] = row0 + warp * 16 + g + 8 * h;
        if (KEYS) {
            limit[h] = row[h] >= rows ? INT_MAX : a.causal ? max(0, row[h] - k.count + q.count) * group : 0;
        } else {
            st[h] = row[h] < rows ? stat(row[h]) : make_float2(0.f, 0.f);
            limit[h] = row[h] < rows ? visible_keys(a.causal, row[h] / group, q.count, k.count) : 0;
        }
    }
    float acc[DK / 8][4], acc2[KEYS ? DK / 8 : 1][4];
#pragma unroll
    for (int c = 0; c < DK / 8; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            acc[c][e] = 0.f;
            if (KEYS) acc2[c][e] = 0.f;
        }
    const uint32_t xa = smem_u32(xs) + warp * 16 * P + val_lane_offset<DK>(lane), ya = xa + (uint32_t)(ys - xs);
    const uint32_t ub = smem_u32(us) + key_lane_offset<DK>(lane), wb = ub + (uint32_t)(ws - us);
    const uint32_t ut = smem_u32(us) + val_lane_offset<DK>(lane), wt = ut + (uint32_t)(ws - us);
    volatile float kept[LONG ? (KEYS ? 2 : 1) * DK / 8 : 1][4];    // of a long sum the pieces so far (in local memory, touched once a piece)
    int pieces = 0, blocks = 0;
    for (int c0 = begin; c0 < end; c0 += G::kStep) {
        if (c0 != begin) __syncthreads();
        if constexpr (LONG) {
            if (blocks++ == kPieceBlocks) {
                blocks = 1;
#pragma unroll
                for (int c = 0; c < DK / 8; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        kept[c][e] = pieces ? kept[c][e] + acc[c][e] : acc[c][e];
                        acc[c][e] = 0.f;
                        if constexpr (KEYS) {
                            kept[DK / 8 + c][e] = pieces ? kept[DK / 8 + c][e] + acc2[c][e] : acc2[c][e];
                            acc2[c][e] = 0.f;
                        }
                    }
                ++pieces;
            }
        }
        load_tile<DK, 128, G::kStep>(tid, us, G::kPlane, a.d, [&](int r) -> const T* { return c0 + r < end ? (KEYS ? query(a.q, a.lq, c0 + r) : key(a.k, a.lk, c0 + r)) : nullptr; });
        load_tile<DK, 128, G::kStep>(tid, ws, G::kPlane, a.d, [&](int r) -> const T* { return c0 + r < end ? (KEYS ? query(a.dout, a.ldo, c0 + r) : key(a.v, a.lv, c0 + r)) : nullptr; });
        if (KEYS && tid < G::kStep) stats[tid] = c0 + tid < end ? stat(c0 + tid) : make_float2(0.f, 0.f);
        __syncthreads();
        float x[4][4], y[4][4];
        block_logits<E, NT, DK>(x, xa, G::kRowPlane, ub, G::kPlane);
        block_logits<E, NT, DK>(y, ya, G::kRowPlane, wb, G::kPlane);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int c = 8 * j + 2 * t + (e & 1), h = e >> 1;
                const float2 s = KEYS ? stats[c] : st[h];
                const bool seen = KEYS ? c0 + c < end && c0 + c >= limit[h] : c0 + c < limit[h];
                const float p = seen ? fast_exp2(fmaf(x[j][e], c1, -s.x)) : 0.f;
                x[j][e] = p;
                // (a query that sees one key has P = 1, whatever its logit: no gradient but that of the value)
                y[j][e] = seen && (KEYS ? k.count : limit[h]) != 1 ? p * (y[j][e] - s.y) : 0.f;
            }
        uint32_t w[NT][2][4];
        block_operand<E, NT>(y, w);
        block_product<E, NT, DK>(acc, w, ut, G::kPlane);
        if constexpr (KEYS) {
            block_operand<E, NT>(x, w);
            block_product<E, NT, DK>(acc2, w, wt, G::kPlane);
        }
    }
    if constexpr (LONG) {
        if (pieces) {
#pragma unroll
            for (int c = 0; c < DK / 8; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    acc[c][e] += kept[c][e];
                    if constexpr (KEYS) acc2[c][e] += kept[DK / 8 + c][e];
                }
        }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if (row[h] >= rows) continue;
        auto put = [&](void* p, const TokLayout& l, int c, float v0, float v1) {
            T* to = static_cast<T*>(p) + (KEYS ? k.batch * l.sb + hk * l.sh + (long long)(k.first + row[h]) * l.st : q.batch * l.sb + (hk * group + row[h] % group) * l.sh + (long long)(q.first + row[h] / group) * l.st) + c;
            *reinterpret_cast<float2*>(to) = make_float2(v0, v1);
        };
#pragma unroll
        for (int c = 0; c < DK / 8; ++c) {
            if (8 * c + 2 * t >= a.d) continue;
            put(KEYS ? a.dk : a.dq, KEYS ? a.ldk : a.ldq, 8 * c + 2 * t, acc[c][2 * h] * a.scale, acc[c][2 * h + 1] * a.scale);
            if constexpr (KEYS) put(a.dv, a.ldv, 8 * c + 2 * t, acc2[c][2 * h], acc2[c][2 * h + 1]);
        }
    }
}

template <int DK, bool KEYS, bool LONG> cudaError_t run_grad_form(const AttendArgs& a, cudaStream_t st) {
    using G = GradGeom<DK>;
    static std::atomic<unsigned long long> done{0};
    if (cudaError_t e = allow_smem(attend_grad_kernel<DK, KEYS, LONG>, done, G::kSmem)) return e;
    const long long slots = KEYS ? slots_of(a.k_offsets != nullptr, a.sequences, a.M, 1, G::kRows) : slots_of(a.q_offsets != nullptr, a.sequences, a.N, a.heads / a.kv_heads, G::kRows);
    attend_grad_kernel<DK, KEYS, LONG><<<dim3((unsigned)slots, a.kv_heads), 128, G::kSmem, st>>>(a);
    return cudaGetLastError();
}
template <int DK, bool KEYS> cudaError_t run_grad(const AttendArgs& a, cudaStream_t st) {
    const long long columns = KEYS ? (long long)a.N * (a.heads / a.kv_heads) : a.M;        // (of packed sequences the longest may have all rows)
    return columns > 32LL * kPieceBlocks ? run_grad_form<DK, KEYS, true>(a, st) : run_grad_form<DK, KEYS, false>(a, st);
}
template <int DK> cudaError_t run_grads(const AttendArgs& a, cudaStream_t st) {
    if (cudaError_t e = run_grad<DK, true>(a, st)) return e;
    return run_grad<DK, false>(a, st);
}
template <typename T> cudaError_t run_dot(const AttendArgs& a, cudaStream_t st) {
    const long long q_slots = slots_of(a.q_offsets != nullptr, a.sequences, a.N, a.heads / a.kv_heads, kDotRows);
    const long long v_slots = is_f16<T> ? slots_of(a.k_offsets != nullptr, a.sequences, a.M, 1, kDotRows) : 0;
    if (is_f16<T>)
        if (cudaError_t e = cudaMemsetAsync(grad_most(a, 0, 0), 0, (size_t)a.sequences * a.kv_heads * 2 * sizeof(unsigned), st)) return e;
    attend_dot_kernel<T><<<dim3((unsigned)(q_slots + v_slots), a.kv_heads), 256, 0, st>>>(a, (unsigned)q_slots);
    return cudaGetLastError();
}

}  // namespace

size_t attend_workspace(int dtype, const AttendArgs& a, int sm_count) {
    int chunk;
    const int shares = shares_of(a, dtype != 0, sm_count, &chunk);
    return shares > 1 ? (size_t)a.batch * a.N * a.heads * shares * (a.d + 2) * sizeof(float) + 16 : 0;
}
size_t attend_backward_workspace(int dtype, const AttendArgs& a, int sm_count) {
    return (size_t)a.batch * a.N * a.heads * sizeof(float) * (dtype == 2 ? 3 : 2) + (dtype == 2 ? (size_t)a.sequences * a.kv_heads * 2 * sizeof(unsigned) : 0);
}

cudaError_t launch_attend(int dtype, AttendArgs a, int sm_count, cudaStream_t st, int* launches) {
    const int shares = shares_of(a, dtype != 0, sm_count, &a.chunk);
    *launches = shares > 1 ? 2 : 1;
    if (dtype != 0 && !few_rows(a)) return launch_attend_umma(dtype, a, st);
    if (dtype == 1) return a.d <= 64 ? run_few<__nv_bfloat16, 64>(a, shares, st) : run_few<__nv_bfloat16, 128>(a, shares, st);
    if (dtype == 2) return a.d <= 64 ? run_few<__half, 64>(a, shares, st) : run_few<__half, 128>(a, shares, st);
    // Sixteen rows a block and four warps on the keys, too, where 64 rows would leave half of the SMs idle (196 tokens, 3 heads of 64: 26.6 -> 16.4 us); elsewhere
    // every block of keys is split into terms for four times the rows.
    const long long blocks = slots_of(a.q_offsets != nullptr, a.sequences, a.N, a.heads / a.kv_heads, 64) * a.kv_heads;
    return few_rows(a) || 2 * blocks <= sm_count ? run_rows_of<1, 4>(a, shares, st) : run_rows_of<4, 1>(a, shares, st);
}
cudaError_t launch_attend_backward(int dtype, const AttendArgs& a, int sm_count, cudaStream_t st, int* launches) {
    *launches = dtype == 1 ? 2 : 3;
    if (dtype == 1) return launch_attend_grad_umma(dtype, a, st);      // (which makes its statistics itself)
    if (cudaError_t e = dtype == 0 ? run_dot<float>(a, st) : run_dot<__half>(a, st)) return e;
    if (dtype == 2) return launch_attend_grad_umma(dtype, a, st);
    if (a.d <= 32) return run_grads<32>(a, st);
    if (a.d <= 64) return run_grads<64>(a, st);
    if (a.d <= 96) return run_grads<96>(a, st);
    return run_grads<128>(a, st);
}

}  // namespace aa
