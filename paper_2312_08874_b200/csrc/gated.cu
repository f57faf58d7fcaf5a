// Gated feed-forward product on the 5th-generation tensor cores, and its gradient.
//
//     G = X Wg^T + bg,  U = X Wu^T + bu,  H = act(G) o U                       X [M][C], Wg and Wu [F][C], H [M][F]
//     dU = dH o act(G),  dG = dH o U o act'(G);  dX = dG Wg + dU Wu,  dWg = dG^T X,  dWu = dU^T X,  biases: column sums
//
// One pipelined product in four forms: a TMA warp fills a ring of operand tiles, one warp issues `tcgen05.mma` into two accumulators in tensor
// memory that take turns, eight warps read the finished one and do the rest.  Blocks are persistent over (tile, split) units.
//   kForward  tile of 128 rows x BN columns of G and the same of U: one instruction of 2 BN columns, whose B operand is a tile of Wg above one of
//             Wu; the epilogue applies biases, activation and product.  G and U never leave the chip.
//   kGrad     the same product again; the epilogue reads dH and writes dG and dU for the two forms that follow.
//   kInput    dX: A = dG, then dU (along their rows), B = Wg, then Wu, read as [hidden][channels] = MN-major: nothing is transposed.
//   kWeight   dWg above dWu: A = dG or dU read MN-major, B = X read MN-major; the sum runs over the rows of X, split over blocks where tiles are few.
// 16-bit operands enter as they are; dG and dU are rounded to the element type, as every operand of a product on the tensor cores is.  fp32: operands are sums of
// three bf16 terms, six pairs of terms, small ones first.
#include "bwd_terms.cuh"
#include "stream_common.cuh"

namespace aa {

namespace {

enum GatedMode { kForward, kGrad, kInput, kWeight };
constexpr int kEpiWarps = 8, kThreads = 32 * (kEpiWarps + 2);
constexpr int kATile = 128 * 128;                      // bytes of a [128][64] (or [64][128]) tile of 16-bit elements
constexpr int kStages = 4;
constexpr int OFF_RING = 1024;
constexpr int kTimeoutTile = 3, kTimeoutRole = 6;
// mbarriers: full [kStages], empty [kStages], accumulator ready [2], accumulator read [2], drain
constexpr int BAR_FULL = 0, BAR_EMPTY = kStages, BAR_ACC = 2 * kStages, BAR_READ = BAR_ACC + 2, BAR_DRAIN = BAR_READ + 2, kBars = BAR_DRAIN + 1;

struct GatedArgs {
    int M, C, F, act;
    int tiles_m, tiles_n, splits, chunks;              // chunks: 64 long, of the sum
    int n;                                             // columns of a tile (kInput, kWeight): a multiple of 16
    const void *bg, *bu, *dh;
    void *out0, *out1;                                 // H; dG and dU; dX; dWg and dWu
    float* part;                                       // [splits][rows][C], where splits > 1
    int* status;
    alignas(64) CUtensorMap a[2], b[2];
};

template <typename T> struct GatedTerms {              // element of the operands, terms and pairs of terms
    using E = T;
    static constexpr int kTerms = 1, kPairs = 1;
};
template <> struct GatedTerms<float> {
    using E = __nv_bfloat16;
    static constexpr int kTerms = 3, kPairs = 6;
};
__device__ __forceinline__ void term_pair(int i, int& a, int& b) {     // (2,0) (1,1) (0,2) (1,0) (0,1) (0,0)
    a = (0x001012 >> (4 * i)) & 3;
    b = (0x010210 >> (4 * i)) & 3;
}

// act(g) and, for the gradient, its derivative
struct Activated { float a, da; };
template <typename T, bool GRAD> __device__ __forceinline__ Activated activate(int act, float g) {
    Activated r;
    r.da = 0.f;
    if (act == 1) {                                                    // GELU: g Phi(g)
        const float cdf = 0.5f + 0.5f * erff(g * 0.70710678f);
        r.a = g * cdf;
        if (GRAD) r.da = fmaf(g * 0.39894228f, expf(-0.5f * g * g), cdf);
        return r;
    }
    // SiLU: g sigmoid(g).  GELU by tanh: g sigmoid(2 k (g + c g^3)), since 0.5 (1 + tanh z) = sigmoid(2 z)
    constexpr float k2 = 1.5957691216f, c = 0.044715f;
    const float g2 = fminf(g * g, 1e4f);                               // (far past where the sigmoid is 0 or 1: no infinity meets a zero)
    const float z = act == 2 ? k2 * g * fmaf(c, g2, 1.f) : g;
    const float s = 1.f / (1.f + expf(-z));
    r.a = g * s;
    if (GRAD) r.da = fmaf(g * (1.f - s), act == 2 ? s * k2 * fmaf(3.f * c, g2, 1.f) : s, s);
    return r;
}

// eight consecutive elements
template <typename T> __device__ __forceinline__ void load8(const T* p, float (&f)[8]) {
    constexpr int V = Elem<T>::kVec;
#pragma unroll
    for (int i = 0; i < 8; i += V) unpack16<T>(__ldg(reinterpret_cast<const uint4*>(p + i)), f + i);
}
template <typename T> __device__ __forceinline__ void store8(T* p, const float* f) {
    constexpr int V = Elem<T>::kVec;
#pragma unroll
    for (int i = 0; i < 8; i += V) *reinterpret_cast<uint4*>(p + i) = pack16<T>(f + i);
}
// eight values as operands of a later product: rounded to the element type, or (fp32) as three planes of terms
template <typename T> __device__ __forceinline__ void store_operand8(void* base, size_t plane, size_t at, const float* f) {
    using E = typename GatedTerms<T>::E;
    if constexpr (GatedTerms<T>::kTerms == 1) {
        store8<T>(static_cast<T*>(base) + at, f);
    } else {
        uint32_t o[3][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t w[3];
            split_pair<E, 3>(f[2 * i], f[2 * i + 1], w);
#pragma unroll
            for (int t = 0; t < 3; ++t) o[t][i] = w[t];
        }
#pragma unroll
        for (int t = 0; t < 3; ++t) *reinterpret_cast<uint4*>(static_cast<E*>(base) + t * plane + at) = make_uint4(o[t][0], o[t][1], o[t][2], o[t][3]);
    }
}

template <GatedMode MODE, int BN> struct GatedShape {
    static constexpr int kN = MODE <= kGrad ? 2 * BN : 256;            // columns of an accumulator
    static constexpr int kStage = kATile + kN * 128;
    static constexpr int kSmem = OFF_RING + kStages * kStage + 1024;
};

template <typename T, GatedMode MODE, int BN> __global__ void __launch_bounds__(kThreads, 1) gated_kernel(const __grid_constant__ GatedArgs p) {
    using S = GatedShape<MODE, BN>;
    using E = typename GatedTerms<T>::E;
    constexpr int kPairs = GatedTerms<T>::kPairs, kN = S::kN;
    extern __shared__ unsigned char smem_raw[];
    __shared__ int s_dead;
    __shared__ uint32_t s_tmem;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int units = p.tiles_m * p.tiles_n * p.splits;

    Pipe pp;
    pp.status = p.status;
    pp.dead = &s_dead;
    pp.bars = base;
    if (tid == 0) {
        s_dead = 0;
        for (int i = 0; i < kBars; ++i) mbar_init(pp.bars + 8 * i, i >= BAR_READ && i < BAR_DRAIN ? kEpiWarps : 1u);
        mbar_fence_init();
    }
    if (warp == 0) tmem_alloc<512>(smem_u32(&s_tmem));
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    pp.tmem = s_tmem;
    pdl_wait_prior();
    pdl_release_next();

    const int tiles_f = (p.F + 127) / 128, chunks_f = (p.F + 63) / 64;
    auto unit_of = [&](int u, int& mt, int& nt, int& k0, int& k1) {
        nt = u % p.tiles_n;
        const int v = u / p.tiles_n, split = v / p.tiles_m;
        mt = v - split * p.tiles_m;
        k0 = (int)((long long)p.chunks * split / p.splits);
        k1 = (int)((long long)p.chunks * (split + 1) / p.splits);
        return split;
    };

    if (warp == kEpiWarps) {
        // ------------------------------------------------------------------ producer
        if (lane == 0) {
            int stage = 0, round = 0;
            for (int u = blockIdx.x; u < units && !pipe_dead(pp); u += gridDim.x) {
                int mt, nt, k0, k1;
                unit_of(u, mt, nt, k0, k1);
                const int boxes = MODE <= kGrad ? 0 : (p.n + 63) / 64;
                for (int pair = 0; pair < kPairs; ++pair) {
                    int ta = 0, tb = 0;
                    if (kPairs > 1) term_pair(pair, ta, tb);
                    for (int k = k0; k < k1 && !pipe_dead(pp); ++k) {
                        if (round > 0) wait_spin(pp, BAR_EMPTY + stage, round - 1, kTimeoutRole);
                        const uint32_t bar = pipe_bar(pp, BAR_FULL + stage), da = base + OFF_RING + stage * S::kStage, db = da + kATile;
                        if constexpr (MODE <= kGrad) {
                            mbar_arrive_expect_tx(bar, S::kStage);
                            tma_load_3d(da, &p.a[0], 64 * k, 128 * mt, ta, bar);
                            tma_load_3d(db, &p.b[0], 64 * k, BN * nt, tb, bar);
                            tma_load_3d(db + BN * 128, &p.b[1], 64 * k, BN * nt, tb, bar);
                        } else if constexpr (MODE == kInput) {
                            const int op = k >= chunks_f, kk = k - op * chunks_f;
                            mbar_arrive_expect_tx(bar, kATile + boxes * 8192);
                            tma_load_3d(da, &p.a[op], 64 * kk, 128 * mt, ta, bar);
                            for (int j = 0; j < boxes; ++j) tma_load_3d(db + j * 8192, &p.b[op], p.n * nt + 64 * j, 64 * kk, tb, bar);
                        } else {
                            const int op = mt >= tiles_f, f0 = 128 * (mt - op * tiles_f);
                            mbar_arrive_expect_tx(bar, kATile + boxes * 8192);
                            tma_load_3d(da, &p.a[op], f0, 64 * k, ta, bar);
                            tma_load_3d(da + 8192, &p.a[op], f0 + 64, 64 * k, ta, bar);
                            for (int j = 0; j < boxes; ++j) tma_load_3d(db + j * 8192, &p.b[0], p.n * nt + 64 * j, 64 * k, tb, bar);
                        }
                        if (++stage == kStages) { stage = 0; ++round; }
                    }
                }
            }
            // no copy may be in flight at the block's end, whatever became of the other roles
            for (int s = 0; s < kStages; ++s) {
                const int last = s < stage ? round : round - 1;
                if (last >= 0) mbar_wait_bounded(pipe_bar(pp, BAR_FULL + s), last & 1, 1u << 16);
            }
        }
        __syncwarp();
    } else if (warp == kEpiWarps + 1) {
        // ------------------------------------------------------------------ products
        constexpr int fmt = Elem<E>::kIsBf16 ? 1 : 0;
        const uint32_t id = umma_idesc(fmt, 128, MODE <= kGrad ? kN : p.n, MODE >= kInput) | (MODE == kWeight ? 1u << 15 : 0u);
        const int total = MODE <= kGrad ? p.C : MODE == kInput ? p.F : p.M;
        int stage = 0, round = 0, ord = 0;
        for (int u = blockIdx.x; u < units && !pipe_dead(pp); u += gridDim.x, ++ord) {
            int mt, nt, k0, k1;
            unit_of(u, mt, nt, k0, k1);
            const int buf = ord & 1;
            if (ord >= 2) wait_spin(pp, BAR_READ + buf, (ord >> 1) - 1, kTimeoutRole);
            tc_fence_after_sync();
            const uint32_t d = pp.tmem + 256 * buf;
            uint32_t acc = 0;
            for (int pair = 0; pair < kPairs; ++pair)
                for (int k = k0; k < k1 && !pipe_dead(pp); ++k) {
                    wait_spin(pp, BAR_FULL + stage, round, kTimeoutTile);
                    tc_fence_after_sync();
                    const uint32_t at = base + OFF_RING + stage * S::kStage;
                    const uint64_t da = MODE == kWeight ? desc_mn(at, 8192) : umma_desc_sw128(at);
                    const uint64_t db = MODE <= kGrad ? umma_desc_sw128(at + kATile) : desc_mn(at + kATile, 8192);
                    const int kk = MODE == kInput && k >= chunks_f ? k - chunks_f : k;
                    const int steps = min(4, (total - 64 * kk + 15) / 16);
                    // descriptor addresses count 16 bytes: a step of 16 is 2 along a K-major row, 128 down MN-major ones
                    for (int s = 0; s < steps; ++s, acc = 1u) umma_ss_w(d, da + (MODE == kWeight ? 128 : 2) * s, db + (MODE <= kGrad ? 2 : 128) * s, id, acc);
                    umma_commit_w(pipe_bar(pp, BAR_EMPTY + stage));
                    if (++stage == kStages) { stage = 0; ++round; }
                }
            umma_commit_w(pipe_bar(pp, BAR_ACC + buf));
        }
        umma_drain_w(pp, BAR_DRAIN);
        __syncwarp();
    } else {
        // ------------------------------------------------------------------ epilogue
        const int q = warp & 3, half = warp >> 2;
        int ord = 0;
        for (int u = blockIdx.x; u < units; u += gridDim.x, ++ord) {
            int mt, nt, k0, k1;
            const int split = unit_of(u, mt, nt, k0, k1), buf = ord & 1;
            const uint32_t acc = pp.tmem + 256 * buf + ((uint32_t)(32 * q) << 16);
            wait_par(pp, BAR_ACC + buf, ord >> 1, kTimeoutTile);
            tc_fence_after_sync();
            auto release = [&] {
                tc_fence_before_sync();
                pipe_arrive_warp(pp, BAR_READ + buf, lane);
            };
            if constexpr (MODE <= kGrad) {
                const int row = 128 * mt + 32 * q + lane;
                const size_t plane = (size_t)p.M * p.F;
#pragma unroll
                for (int s = 0; s < BN / 32; ++s) {
                    const int col = half * (BN / 2) + 16 * s, f0 = BN * nt + col;
                    float g[16], v[16];
                    __syncwarp();
                    tmem_ld16(acc + col, g);
                    tmem_ld16(acc + BN + col, v);
                    tmem_ld_wait();
                    if (s == BN / 32 - 1) release();
#pragma unroll
                    for (int j = 0; j < 16; j += 8) {
                        const int f = f0 + j;
                        if (f >= p.F || row >= p.M) continue;
                        if (p.bg) {
                            float t[8];
                            load8<T>(static_cast<const T*>(p.bg) + f, t);
#pragma unroll
                            for (int i = 0; i < 8; ++i) g[j + i] += t[i];
                        }
                        if (p.bu) {
                            float t[8];
                            load8<T>(static_cast<const T*>(p.bu) + f, t);
#pragma unroll
                            for (int i = 0; i < 8; ++i) v[j + i] += t[i];
                        }
                        const size_t at = (size_t)row * p.F + f;
                        if constexpr (MODE == kForward) {
#pragma unroll
                            for (int i = 0; i < 8; ++i) v[j + i] *= activate<T, false>(p.act, g[j + i]).a;
                            store8<T>(static_cast<T*>(p.out0) + at, v + j);
                        } else {
                            float t[8];
                            load8<T>(static_cast<const T*>(p.dh) + at, t);
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                const Activated r = activate<T, true>(p.act, g[j + i]);
                                g[j + i] = t[i] * v[j + i] * r.da;
                                v[j + i] = t[i] * r.a;
                            }
                            store_operand8<T>(p.out0, plane, at, g + j);
                            store_operand8<T>(p.out1, plane, at, v + j);
                        }
                    }
                }
            } else {
                const int op = MODE == kWeight && mt >= tiles_f, limit = MODE == kWeight ? p.F : p.M;
                const int row = 128 * (mt - op * tiles_f) + 32 * q + lane;
                const int blocks = (p.n + 31) / 32;
                for (int b = half; b < blocks; b += 2) {
                    float v[32];
                    __syncwarp();
                    tmem_ld32(acc + 32 * b, reinterpret_cast<uint32_t(&)[32]>(v));
                    tmem_ld_wait();
                    if (b + 2 >= blocks) release();
#pragma unroll
                    for (int j = 0; j < 32; j += 8) {
                        const int in_tile = 32 * b + j, c = p.n * nt + in_tile;
                        if (in_tile >= p.n || c >= p.C || row >= limit) continue;
                        if (p.splits > 1) store8<float>(p.part + ((size_t)split * (MODE == kWeight ? 2 * (size_t)p.F : (size_t)p.M) + (size_t)op * p.F + row) * p.C + c, v + j);
                        else store8<T>(static_cast<T*>(op ? p.out1 : p.out0) + (size_t)row * p.C + c, v + j);
                    }
                }
                if (half >= blocks) release();
            }
            __syncwarp();
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 0) tmem_dealloc<512>(pp.tmem);
}

// fp32 -> three planes of bf16 terms, eight elements a thread
struct SplitArgs {
    const float* src[3];
    __nv_bfloat16* dst[3];
    size_t count[3];
};
__global__ void __launch_bounds__(256) split_terms_kernel(const __grid_constant__ SplitArgs p) {
    pdl_wait_prior();
    pdl_release_next();
    const size_t n = p.count[blockIdx.y], i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (i >= n) return;
    float f[8];
    load8<float>(p.src[blockIdx.y] + i, f);
    store_operand8<float>(p.dst[blockIdx.y], n, i, f);
}

// Sum of `splits` arrays of n fp32 values (a multiple of four) in their order; values from `first` on go to out1
template <typename T> __global__ void __launch_bounds__(256) gated_sum_kernel(const float* part, int splits, size_t n, size_t first, T* out0, T* out1) {
    pdl_wait_prior();
    pdl_release_next();
    const size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= n) return;
    float4 v = *reinterpret_cast<const float4*>(part + i);
    for (int s = 1; s < splits; ++s) {
        const float4 w = *reinterpret_cast<const float4*>(part + s * n + i);
        v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
    }
    T* dst = i < first ? out0 + i : out1 + (i - first);
    dst[0] = Elem<T>::from_f32(v.x); dst[1] = Elem<T>::from_f32(v.y); dst[2] = Elem<T>::from_f32(v.z); dst[3] = Elem<T>::from_f32(v.w);
}

// Column sums of dG and dU: a block takes 64 columns of one of them and a run of rows
constexpr int kColRows = 512;
template <typename T> __global__ void __launch_bounds__(256) gated_column_kernel(const void* dg, const void* du, int M, int F, float* part) {
    using E = typename GatedTerms<T>::E;
    __shared__ float s_sum[32][64];
    pdl_wait_prior();
    pdl_release_next();
    const int c = threadIdx.x & 7, r = threadIdx.x >> 3, f = 64 * blockIdx.x + 8 * c;
    const int r0 = kColRows * blockIdx.z, r1 = min(r0 + kColRows, M);
    const E* src = static_cast<const E*>(blockIdx.y ? du : dg);
    float sum[8] = {};
    if (f < F)
        for (int row = r0 + r; row < r1; row += 32)
#pragma unroll
            for (int t = 0; t < GatedTerms<T>::kTerms; ++t) {
                float v[8];
                load8<E>(src + ((size_t)t * M + row) * F + f, v);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[i] += v[i];
            }
#pragma unroll
    for (int i = 0; i < 8; ++i) s_sum[r][8 * c + i] = sum[i];
    __syncthreads();
    if (threadIdx.x < 64 && 64 * blockIdx.x + threadIdx.x < F) {
        float v = 0.f;
        for (int k = 0; k < 32; ++k) v += s_sum[k][threadIdx.x];
        part[((size_t)blockIdx.z * 2 + blockIdx.y) * F + 64 * blockIdx.x + threadIdx.x] = v;
    }
}

// Work of the two products with a long sum: tiles of at most 256 columns, split while tiles are fewer than SMs
struct GatedSplit { int tiles_m, tiles_n, n, chunks, splits; };
GatedSplit plan_split(int tiles_m, int chunks, int C, int sm_count) {
    GatedSplit s;
    s.tiles_m = tiles_m;
    s.tiles_n = (C + 255) / 256;
    s.n = ((C + s.tiles_n - 1) / s.tiles_n + 15) / 16 * 16;
    s.chunks = chunks;
    const long long tiles = (long long)tiles_m * s.tiles_n;
    s.splits = 1;
    if (tiles < sm_count) s.splits = (int)(sm_count / tiles);
    if (s.splits > chunks / 4) s.splits = chunks / 4;
    if (s.splits < 1) s.splits = 1;
    return s;
}
GatedSplit plan_input(int M, int C, int F, int sm_count) { return plan_split((M + 127) / 128, 2 * ((F + 63) / 64), C, sm_count); }
GatedSplit plan_weight(int M, int C, int F, int sm_count) { return plan_split(2 * ((F + 127) / 128), (M + 63) / 64, C, sm_count); }

// Workspace: terms of X, Wg, Wu (fp32) | dG | dU | shares of dX, dW, of the column sums
struct GatedWs { size_t x, wg, wu, dg, du, dx, dw, db, total; };
GatedWs gated_layout(int dtype, int M, int C, int F, bool backward, int sm_count) {
    GatedWs w;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at += (bytes + 255) / 256 * 256; return o; };
    const size_t terms = dtype == kF32 ? 3 : 0;
    w.x = take(terms * M * C * 2);
    w.wg = take(terms * F * C * 2);
    w.wu = take(terms * F * C * 2);
    w.dg = w.du = w.dx = w.dw = w.db = at;
    if (backward) {
        const size_t planes = (dtype == kF32 ? 3 : 1) * (size_t)M * F * 2;
        w.dg = take(planes);
        w.du = take(planes);
        const GatedSplit in = plan_input(M, C, F, sm_count), we = plan_weight(M, C, F, sm_count);
        w.dx = take(in.splits > 1 ? (size_t)in.splits * M * C * 4 : 0);
        w.dw = take(we.splits > 1 ? (size_t)we.splits * 2 * F * C * 4 : 0);
        w.db = take((size_t)((M + kColRows - 1) / kColRows) * 2 * F * 4);
    }
    w.total = at;
    return w;
}

template <typename T, GatedMode MODE, int BN> cudaError_t launch_mode(const GatedArgs& a, int sm_count, cudaStream_t st) {
    static std::atomic<unsigned long long> done{0};
    const cudaError_t e = allow_smem(gated_kernel<T, MODE, BN>, done, GatedShape<MODE, BN>::kSmem);
    if (e != cudaSuccess) return e;
    const long long units = (long long)a.tiles_m * a.tiles_n * a.splits;
    return launch_dependent(gated_kernel<T, MODE, BN>, dim3((unsigned)(units < sm_count ? units : sm_count)), kThreads, GatedShape<MODE, BN>::kSmem, st, a);
}

template <typename T> cudaError_t run_gated(const GatedCall& c, cudaStream_t st, int* launches) {
    constexpr int kTerms = GatedTerms<T>::kTerms;
    const GatedWs w = gated_layout(sizeof(T) == 4 ? kF32 : kBF16, c.M, c.C, c.F, c.dh != nullptr, c.sm_count);
    char* ws = static_cast<char*>(c.ws);
    const void *x = c.x, *wg = c.wg, *wu = c.wu;
    cudaError_t e;
    if (kTerms > 1) {
        SplitArgs s = {{static_cast<const float*>(x), static_cast<const float*>(wg), static_cast<const float*>(wu)},
                       {reinterpret_cast<__nv_bfloat16*>(ws + w.x), reinterpret_cast<__nv_bfloat16*>(ws + w.wg), reinterpret_cast<__nv_bfloat16*>(ws + w.wu)},
                       {(size_t)c.M * c.C, (size_t)c.F * c.C, (size_t)c.F * c.C}};
        const size_t most = s.count[0] > s.count[1] ? s.count[0] : s.count[1];
        if ((e = launch_dependent(split_terms_kernel, dim3((unsigned)((most + 2047) / 2048), 3), 256, 0, st, s)) != cudaSuccess) return e;
        ++*launches;
        x = s.dst[0]; wg = s.dst[1]; wu = s.dst[2];
    }
    GatedArgs a;
    memset(&a, 0, sizeof(a));
    a.M = c.M; a.C = c.C; a.F = c.F; a.act = c.act;
    a.bg = c.bg; a.bu = c.bu; a.dh = c.dh;
    a.status = c.status;
    // G and U.  Narrower tiles where 128 columns leave SMs without a tile.
    const int tm = (c.M + 127) / 128;
    int bn = 128;
    while (bn > 32 && (long long)tm * ((c.F + bn - 1) / bn) * 2 <= c.sm_count) bn /= 2;
    a.tiles_m = tm; a.tiles_n = (c.F + bn - 1) / bn; a.splits = 1; a.chunks = (c.C + 63) / 64;
    a.out0 = c.dh ? ws + w.dg : static_cast<char*>(c.h);
    a.out1 = ws + w.du;
    if (!make_map_3d_u16(&a.a[0], x, kTerms, c.M, c.C, 128) || !make_map_3d_u16(&a.b[0], wg, kTerms, c.F, c.C, bn) || !make_map_3d_u16(&a.b[1], wu, kTerms, c.F, c.C, bn)) return cudaErrorInvalidValue;
    if (c.dh) e = bn == 128 ? launch_mode<T, kGrad, 128>(a, c.sm_count, st) : bn == 64 ? launch_mode<T, kGrad, 64>(a, c.sm_count, st) : launch_mode<T, kGrad, 32>(a, c.sm_count, st);
    else e = bn == 128 ? launch_mode<T, kForward, 128>(a, c.sm_count, st) : bn == 64 ? launch_mode<T, kForward, 64>(a, c.sm_count, st) : launch_mode<T, kForward, 32>(a, c.sm_count, st);
    if (e != cudaSuccess) return e;
    ++*launches;
    if (!c.dh) return cudaSuccess;

    const void *dg = ws + w.dg, *du = ws + w.du;
    auto sum = [&](const float* part, int splits, size_t n, size_t first, void* out0, void* out1) {
        ++*launches;
        return launch_dependent(gated_sum_kernel<T>, dim3((unsigned)((n + 1023) / 1024)), 256, 0, st, part, splits, n, first, static_cast<T*>(out0), static_cast<T*>(out1));
    };
    if (c.dx) {
        const GatedSplit s = plan_input(c.M, c.C, c.F, c.sm_count);
        a.tiles_m = s.tiles_m; a.tiles_n = s.tiles_n; a.n = s.n; a.splits = s.splits; a.chunks = s.chunks;
        a.out0 = c.dx;
        a.part = reinterpret_cast<float*>(ws + w.dx);
        if (!make_map_3d_u16(&a.a[0], dg, kTerms, c.M, c.F, 128) || !make_map_3d_u16(&a.a[1], du, kTerms, c.M, c.F, 128) ||
            !make_map_3d_u16(&a.b[0], wg, kTerms, c.F, c.C, 64) || !make_map_3d_u16(&a.b[1], wu, kTerms, c.F, c.C, 64)) return cudaErrorInvalidValue;
        if ((e = launch_mode<T, kInput, 128>(a, c.sm_count, st)) != cudaSuccess) return e;
        ++*launches;
        if (s.splits > 1 && (e = sum(a.part, s.splits, (size_t)c.M * c.C, (size_t)c.M * c.C, c.dx, nullptr)) != cudaSuccess) return e;
    }
    if (c.dwg) {
        const GatedSplit s = plan_weight(c.M, c.C, c.F, c.sm_count);
        a.tiles_m = s.tiles_m; a.tiles_n = s.tiles_n; a.n = s.n; a.splits = s.splits; a.chunks = s.chunks;
        a.out0 = c.dwg; a.out1 = c.dwu;
        a.part = reinterpret_cast<float*>(ws + w.dw);
        if (!make_map_3d_u16(&a.a[0], dg, kTerms, c.M, c.F, 64) || !make_map_3d_u16(&a.a[1], du, kTerms, c.M, c.F, 64) || !make_map_3d_u16(&a.b[0], x, kTerms, c.M, c.C, 64)) return cudaErrorInvalidValue;
        if ((e = launch_mode<T, kWeight, 128>(a, c.sm_count, st)) != cudaSuccess) return e;
        ++*launches;
        if (s.splits > 1 && (e = sum(a.part, s.splits, 2 * (size_t)c.F * c.C, (size_t)c.F * c.C, c.dwg, c.dwu)) != cudaSuccess) return e;
    }
    if (c.dbg) {
        const int runs = (c.M + kColRows - 1) / kColRows;
        float* part = reinterpret_cast<float*>(ws + w.db);
        if ((e = launch_dependent(gated_column_kernel<T>, dim3((c.F + 63) / 64, 2, runs), 256, 0, st, dg, du, c.M, c.F, part)) != cudaSuccess) return e;
        ++*launches;
        if ((e = sum(part, runs, 2 * (size_t)c.F, c.F, c.dbg, c.dbu)) != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace

size_t gated_bytes(int dtype, int M, int C, int F, bool backward, int sm_count) { return gated_layout(dtype, M, C, F, backward, sm_count).total; }

cudaError_t launch_gated(int dtype, const GatedCall& c, cudaStream_t st, int* launches) {
    switch (dtype) {
        case kF32: return run_gated<float>(c, st, launches);
        case kBF16: return run_gated<__nv_bfloat16>(c, st, launches);
        case kF16: return run_gated<__half>(c, st, launches);
        default: return cudaErrorInvalidValue;
    }
}

}  // namespace aa
