// Gated feed-forward product on the 5th-generation tensor cores, and its gradient.
//
//     G = X Wg^T + bg,  U = X Wu^T + bu,  H = act(G) o U                       X [M][C], Wg and Wu [F][C], H [M][F]
//     dU = dH o act(G),  dG = dH o U o act'(G);  dX = dG Wg + dU Wu,  dWg = dG^T X,  dWu = dU^T X,  biases: column sums
//
// One pipelined product in three forms: two TMA warps fill a ring of operand tiles, one warp issues `tcgen05.mma` into two accumulators in tensor
// memory that take turns, sixteen warps read the finished one and do the rest.  A pair of blocks (cta_group::2) has a tile of 256 rows.
//   kForward   256 rows of 128 hidden units of G and U: one block of the pair holds a tile of Wg, the other one of Wu, so that one instruction of 256
//              columns makes both; the epilogue applies biases, activation and product.  G and U never leave the chip.
//   kGrad      the same product again; the epilogue reads dH, writes dG and dU for the third form and sums their columns before they are rounded.
//   kProducts  dX: A = dG, then dU (along their rows), B = Wg, then Wu, read as [hidden][channels] = MN-major: nothing is transposed.  dWg and dWu:
//              A = dG in one block of the pair, dU in the other, both MN-major, B = X MN-major.  Their sums are cut into chunks of 64, of which all pairs
//              have as many: whole tiles of dX, then a run of the other tiles; a pair writes what it has whole and leaves its share of what it has
//              not, and gated_finish_kernel adds the shares up in their order.
// 16-bit operands enter as they are; dG and dU are rounded to the element type, as every operand of a product on the tensor cores is (few rows, or where the
// caller asks for it: and what that leaves as a second term).  In f16 kGrad is launched twice: the second one ends at once unless dG and dU leave the type's range
// (gated_scale).  fp32: operands are sums of three bf16 terms, six pairs of terms, small ones first.
//
// What bounds it (us of a launch among others; rows x channels x hidden units):
//   kForward   32768 x 512 x 1368 bf16, SiLU: 88 to 92, 1.0 PFLOP/s.  Tensor pipe 75 % busy (a chunk of 64 takes 600 cycles of 512), clocks under the power
//              limit; the two products alone take 85 in the vendor's library.  8192 x 320 x 1280 f16, GELU: 18, 0.74 PFLOP/s: the epilogue (4000 cycles a tile,
//              products 2600), a first accumulator after 4.2 us, 1.1 us from the last store to the end.  The library's products alone: 19.
//   kGrad      8192 x 320 x 1280 f16 27 (its second launch 4), 25088 x 192 x 512 bf16 28: the epilogue, 7000 cycles a tile at half of the issue slots, and the same start and end.
//   kProducts  30 and 24: operands out of L2, 32 KB a block and chunk of 64 in 480 to 600 cycles (instructions for 160 or 192 columns take 320 or 384).
//   finishing  5.8 and 6.1: 16 MB of shares out of L2, a start.
// Tiles of 512 columns would halve what kProducts reads of A, and double the shares: 64.6 -> 69.8 us for 8192 x 320 x 1280.
#include "bwd_terms.cuh"
#include "pair.cuh"
#include "stream_common.cuh"

#include <type_traits>

namespace aa {

namespace {

enum GatedMode { kForward, kGrad, kProducts };
constexpr int kEpiWarps = 16, kThreads = 32 * (kEpiWarps + 3);
constexpr int kATile = 128 * 128;                      // bytes of a [128][64] (or [64][128]) tile of 16-bit elements
constexpr int kHalfPatch = 2048;                       // bytes of a warp's staged box of 32 x 32 16-bit values (fp32: two)
constexpr int kTimeoutTile = 3, kTimeoutRole = 6;
// mbarriers: full [kRing], empty [kRing], accumulator ready [2], accumulator read [2], drain, dH [warps]
constexpr int kRing = 6, BAR_FULL = 0, BAR_EMPTY = kRing, BAR_ACC = 2 * kRing, BAR_READ = BAR_ACC + 2, BAR_DRAIN = BAR_READ + 2, BAR_DH = BAR_DRAIN + 1, kBars = BAR_DH + kEpiWarps;
static_assert(kBars * 8 <= 1024, "barriers");

// kProducts' work: tiles of dX, of 256 rows, and of dWg and dWu, of 128 hidden units of both; n columns each.  Every pair has some of the first `whole`
// tiles of dX for itself; the other tiles of dX and those of the weights, cut into chunks, are a line of which it has a run, so long that all
// pairs have as many chunks.  Where only one of the two is asked for, the other's tiles are left out, and the cuts stay where they are: the bits of a
// gradient do not depend on what else is asked for.
struct GatedLine {
    int tiles_x, chunks_x, tiles_w, chunks_w, tiles_n, n, pairs, whole;
    int dx, dw;                                        // asked for
    __host__ __device__ long long total() const { return (long long)tiles_x * chunks_x + (long long)tiles_w * chunks_w; }
    __host__ __device__ int own(int pair) const { return (int)((long long)whole * pair / pairs); }           // first tile of a pair's own
    __host__ __device__ long long begin(int pair) const { return total() * pair / pairs - (long long)own(pair) * chunks_x; }
};
struct GatedArgs {
    int M, C, F, act;
    int tiles_m, tiles_n, chunks;                      // kForward, kGrad; chunks: 64 long, of the sum
    GatedLine line;
    const void *bg, *bu, *dh;
    void *out0, *out1;                                 // H; dG and dU: where they are written without staging
    int terms;                                         // kGrad, kProducts of 16-bit elements: of dG and dU (1 or 2)
    float* column;                                     // [slots][2][F]: shares of the column sums of dG and dU, or null
    float* largest;                                    // f16: [largest_parts] by kGrad's blocks: the largest |dG| and |dU|
    int largest_parts, again;                          // again: kGrad's second pass, where that is out of f16's range
    int* status;
    alignas(64) CUtensorMap a[2], b[2], x;             // operands; kProducts: a, b of dX (a of the weights, too), x: X
    alignas(64) CUtensorMap s[3], g, w[2], share;      // staged results: H; dG, dU; dX, dWg, dWu; dH; kProducts: dG and dU in boxes of 64 rows; shares of tiles
};

// Element of the operands, terms and pairs of terms; and how long a sum in tensor memory gets (kMost, kPiece, in chunks of 64).  The tensor cores cut off what
// lies below the last bit at every step of 16, always towards zero: 3e-8 of the sum a step, 1.9e-5 where 16384 channels are summed up in two halves.  Longer sums
// are cut into pieces, which the epilogue adds up in fp32: 16 bits 1024 steps, 3e-5 (f16 itself 2e-4); fp32 32 steps, 1e-6.
template <typename T> struct GatedTerms {
    using E = T;
    static constexpr int kTerms = 1, kPairs = 1, kMost = 256, kPiece = 256;
};
template <> struct GatedTerms<float> {
    using E = __nv_bfloat16;
    static constexpr int kTerms = 3, kPairs = 6, kMost = 16, kPiece = 8;
};
__device__ __forceinline__ void term_pair(int i, int& a, int& b) {     // (2,0) (1,1) (0,2) (1,0) (0,1) (0,0)
    a = (0x001012 >> (4 * i)) & 3;
    b = (0x010210 >> (4 * i)) & 3;
}

// act(g) and, for the gradient, its derivative, of a pair of values.  SiLU: g sigmoid(g).  GELU by tanh: g sigmoid(2 k (g + c g^3)), since
// 0.5 (1 + tanh z) = sigmoid(2 z).  GELU: g Phi(g).
constexpr float kTanh2 = 1.5957691216f, kTanhC = 0.044715f;            // 2 sqrt(2 / pi)
__device__ __forceinline__ float fast_rcp(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }
template <typename T, int ACT, bool GRAD> __device__ __forceinline__ void activate(float2 g, float2& a, float2& da) {
    da = both(0.f);
    if constexpr (sizeof(T) == 4) {                                    // fp32 accuracy
        const float gs[2] = {g.x, g.y};
        float r[2], d[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float x = gs[i];
            if (ACT == 1) {
                const float cdf = 0.5f + 0.5f * erff(x * 0.70710678f);
                r[i] = x * cdf;
                if (GRAD) d[i] = fmaf(x * 0.39894228f, expf(-0.5f * x * x), cdf);
            } else {
                const float x2 = fminf(x * x, 1e4f);                   // (far past where the sigmoid is 0 or 1: no infinity meets a zero)
                const float s = 1.f / (1.f + expf(ACT == 2 ? -kTanh2 * x * fmaf(kTanhC, x2, 1.f) : -x));
                r[i] = x * s;
                if (GRAD) d[i] = fmaf(x * (1.f - s), ACT == 2 ? s * kTanh2 * fmaf(3.f * kTanhC, x2, 1.f) : s, s);
            }
        }
        a = make_float2(r[0], r[1]);
        da = make_float2(d[0], d[1]);
    } else if constexpr (ACT == 1) {
        // Upper tail Q(x) = exp(-x^2 / 2) R(x), x = |g|, with R (half of a scaled complementary error function, smooth from 1/2 down) as a
        // polynomial on [0, 5], fitted with weight exp(-x^2 / 2): Q is within 3e-7 (a 16-bit result of size 1e-3 ends at 2e-6).  g Phi(g) =
        // max(g, 0) - x Q(x).  One special-function instruction, which the derivative shares; with the library's error function the epilogue
        // takes 3.4 times as long.
        const float2 x = make_float2(fminf(fabsf(g.x), 5.f), fminf(fabsf(g.y), 5.f));
        const float2 w = fmul2(fmul2(g, g), both(-0.72134752f));       // log2 of exp(-g^2 / 2)
        const float2 e = make_float2(fast_exp2(w.x), fast_exp2(w.y));
        float2 r = both(8.063080713e-06f);                             // -R
        r = ffma2(r, x, both(-1.519420184e-04f));
        r = ffma2(r, x, both(1.271162881e-03f));
        r = ffma2(r, x, both(-6.382808089e-03f));
        r = ffma2(r, x, both(2.223088220e-02f));
        r = ffma2(r, x, both(-5.949680135e-02f));
        r = ffma2(r, x, both(1.317728907e-01f));
        r = ffma2(r, x, both(-2.497522980e-01f));
        r = ffma2(r, x, both(3.989226222e-01f));
        r = ffma2(r, x, both(-4.999997318e-01f));
        if (GRAD) {
            const float2 h = ffma2(e, r, both(0.5f));                  // 1/2 - Q: Phi is that above 1/2, or below
            const float2 cdf = fadd2(both(0.5f), make_float2(copysignf(h.x, g.x), copysignf(h.y, g.y)));
            a = fmul2(g, cdf);
            da = ffma2(fmul2(g, both(0.39894228f)), e, cdf);
        } else {
            a = ffma2(x, fmul2(e, r), make_float2(fmaxf(g.x, 0.f), fmaxf(g.y, 0.f)));
        }
    } else {
        float2 z = fmul2(g, both(-kLog2e)), slope = both(1.f);
        if (ACT == 2) {
            const float2 q = fmul2(g, g), g2 = make_float2(fminf(q.x, 1e4f), fminf(q.y, 1e4f));
            z = fmul2(fmul2(g, both(-kLog2e * kTanh2)), ffma2(g2, both(kTanhC), both(1.f)));
            if (GRAD) slope = ffma2(g2, both(3.f * kTanhC * kTanh2), both(kTanh2));
        }
        const float2 s = make_float2(fast_rcp(1.f + fast_exp2(z.x)), fast_rcp(1.f + fast_exp2(z.y)));
        a = fmul2(g, s);
        if (GRAD) da = ffma2(fmul2(a, slope), ffma2(s, both(-1.f), both(1.f)), s);
    }
}
// f16: dG and dU leave its range before the results do (an infinity past 65504, fewer bits below 6e-5).  Where their largest lies outside [2, 65504], kGrad runs
// again and holds them times this power of two, which brings the largest to 2^14 and more, and kProducts divides by it.  From 2 on a row or a hidden unit
// whose gradients are a thousandth of the usual ones (a 32nd of the largest) keeps all bits.  8192 x 320 x 1280: 57.2 -> 61.2 us for the launch that ends at once
// and the sizes; scaled by a bound from the inputs (a pass over dH, X and the weights before kGrad): 72.7.  Called by whole warps.
__device__ __forceinline__ float gated_scale(const float* largest, int parts, int lane) {
    float m = 0.f;
    for (int i = lane; i < parts; i += 32) m = fmaxf(m, largest[i]);
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (m == 0.f || (m >= 2.f && m <= 65504.f)) return 1.f;
    return exp2f((float)max(-60, min(60, 14 - ilogbf(m))));
}
// m and the sizes of N values, of which infinities and NaN do not count
template <int N> __device__ __forceinline__ float largest_finite(float m, const float (&v)[N]) {
    static_assert(N % 2 == 0, "pairs");
    float n = m;
#pragma unroll
    for (int i = 0; i < N; i += 2) n = max3(n, fabsf(v[i]), fabsf(v[i + 1]));
    if (n < INFINITY) return n;
#pragma unroll 1
    for (int i = 0; i < N; ++i) {
        float a = 0.f;
#pragma unroll
        for (int k = 0; k < N; ++k) a = k == i ? fabsf(v[k]) : a;      // (no indexed registers)
        if (a < INFINITY) m = fmaxf(m, a);
    }
    return m;
}
// f(constant of the activation): the choice is made once a tile, not once a value
template <typename F> __device__ __forceinline__ void by_activation(int act, F f) {
    if (act == 1) f(std::integral_constant<int, 1>());
    else if (act == 2) f(std::integral_constant<int, 2>());
    else f(std::integral_constant<int, 0>());
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
// eight values as operands of a later product: rounded to the element type (and what that leaves in a second plane), or (fp32) as three planes of terms
template <typename T> __device__ __forceinline__ void store_operand8(void* base, size_t plane, size_t at, const float* f, bool second = false) {
    using E = typename GatedTerms<T>::E;
    if constexpr (GatedTerms<T>::kTerms == 1) {
        store8<T>(static_cast<T*>(base) + at, f);
        if (second) {
            float rest[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float r = f[i] - Elem<T>::to_f32(Elem<T>::from_f32(f[i]));
                rest[i] = r - r == 0.f ? r : 0.f;         // (an infinity leaves nothing, not NaN)
            }
            store8<T>(static_cast<T*>(base) + plane + at, rest);
        }
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
__device__ __forceinline__ void st_shared4(uint32_t at, uint4 v) { asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};\n" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory"); }
// 16 rows of 64 bytes each: 8 x 8 values a register, in the layout of tmem_ld_16x256b
__device__ __forceinline__ void ld_matrix4(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];\n" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void st_matrix4(uint32_t at, const uint32_t (&r)[4]) {
    asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1,%2,%3,%4};\n" ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
__device__ __forceinline__ float2 ld_shared_pair(uint32_t at) {
    float2 v;
    asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];\n" : "=f"(v.x), "=f"(v.y) : "r"(at) : "memory");
    return v;
}
// Sum over the lanes of 16 values each: lane l gets that of value l / 2
__device__ __forceinline__ float sum_lanes16(const float (&x)[16], int lane) {
    float y[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = x[i];
#pragma unroll
    for (int n = 8; n; n >>= 1) {
        const bool upper = lane & 2 * n;
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const float other = __shfl_xor_sync(0xffffffffu, upper ? y[i] : y[i + n], 2 * n);
            y[i] = (upper ? y[i + n] : y[i]) + other;
        }
    }
    return y[0] + __shfl_xor_sync(0xffffffffu, y[0], 1);
}

// A pair of blocks takes a tile of 256 rows, each of its blocks 128 of them and half of the B operand (BN = 128, and kProducts); a lone block a tile of
// 128 rows and 2 BN columns (BN = 64 or 32: small problems).
template <typename T, GatedMode MODE, int BN> struct GatedShape {
    static constexpr int kParts = MODE == kGrad && BN == 128 ? 2 : 1;                      // of a tile, which pairs may share
    static constexpr bool kPair = BN == 128, kStaged = MODE == kProducts || (kPair && sizeof(T) == 2);
    static constexpr int kBTile = kPair ? kATile : 2 * BN * 128;
    static constexpr int kStage = kATile + kBTile;
    static constexpr int kPatch = !kStaged ? 0 : MODE == kForward ? kHalfPatch : MODE == kGrad ? 3 * kHalfPatch : 2 * kHalfPatch;       // of a warp
    static constexpr int kStages = kStaged && MODE == kGrad ? 3 : 5;
    static constexpr int kOffPatch = 1024 + kStages * kStage, kOffBias = kOffPatch + kEpiWarps * kPatch;
    static constexpr int kSmem = kOffBias + (MODE <= kGrad && kStaged ? kEpiWarps * 256 : 0) + 1024;
};

// What block (or pair) `who` of `count` does, tile by tile.  kForward and kGrad: a run of tiles in the order of the rows, so that a run has few column
// ranges; kGrad's pairs share them evenly by halves of 64 hidden units, so that 5.3 tiles a pair take 5.5 instead of 6 tiles' time (8192 x 320 x 1280 f16
// 28.0 -> 26.9 us, 25088 x 192 x 512 bf16 29.1 -> 28.0).  Not kForward's: a half loads what a whole tile does (17.8 us both ways, 32768 x 512 x 1368 bf16
// 88.6 -> 90.2).  kProducts: its own tiles, then its run of the line.
struct Work {
    int mt, nt, k0, k1;
    int part;                                          // 0: a whole tile; else the half 1 or 2
    bool weight, whole;                                // kProducts: of dWg and dWu; the whole sum
    int slot;                                          // of a share
    bool cut, first, last;                             // a piece of a long sum: which one
};
// MOST (0: no sum of the launch is longer): a longer sum comes in pieces of at most PIECE chunks
template <GatedMode MODE, int PARTS, int MOST, int PIECE> struct Walk {
    const GatedArgs& p;
    long long at, first, end;
    int who, own, own_end, mt, nt, left;               // left, later: kForward and kGrad, whose loops have no room for 64-bit arithmetic
    bool later;                                        // the run begins with a tile's second half
    int each, until;                                   // of a long sum: chunks of a piece, the last one's end (0: none is under way)
    __device__ Walk(const GatedArgs& args, int who_, int count) : p(args), who(who_), each(0), until(0) {
        if (MODE == kProducts) {
            first = at = p.line.begin(who);
            end = p.line.begin(who + 1);
            own = p.line.own(who);
            own_end = p.line.dx ? p.line.own(who + 1) : own;
        } else {
            const long long units = (long long)PARTS * p.tiles_m * p.tiles_n;
            const long long begin = units * who / count, tile = begin / PARTS;
            left = (int)(units * (who + 1) / count - begin);
            later = begin % PARTS != 0;
            nt = (int)(tile / p.tiles_m);
            mt = (int)(tile - (long long)nt * p.tiles_m);
        }
    }
    __device__ bool next(Work& w) {                    // (w: as the call before left it)
        if (MOST == 0) return next_sum(w);
        if (until) {
            w.k0 = w.k1;
            w.k1 = min(w.k0 + each, until);
            w.first = false;
            w.last = w.k1 == until;
            if (w.last) until = 0;
            return true;
        }
        if (!next_sum(w)) return false;
        const int n = w.k1 - w.k0;
        w.cut = n > MOST;
        w.first = true;
        w.last = !w.cut;
        if (w.cut) {
            const int pieces = (n + PIECE - 1) / PIECE;
            each = (n + pieces - 1) / pieces;
            until = w.k1;
            w.k1 = w.k0 + each;
        }
        return true;
    }
    __device__ bool next_sum(Work& w) {
        if (MODE != kProducts) {
            if (left <= 0) return false;
            w.nt = nt; w.mt = mt;
            w.k0 = 0; w.k1 = p.chunks;
            w.part = later ? 2 : left < PARTS ? 1 : 0;
            left -= w.part ? 1 : PARTS;
            later = false;
            if (++mt == p.tiles_m) { mt = 0; ++nt; }
            return true;
        }
        const GatedLine& l = p.line;
        w.part = 0;
        int tile = 0, chunks = l.chunks_x;
        bool wanted = false;
        if (own < own_end) {
            tile = own++;
            w.k0 = 0;
            w.k1 = chunks;
            w.weight = false;
            wanted = true;
        }
        while (!wanted) {
            if (at >= end) return false;
            const long long rest = (long long)(l.tiles_x - l.whole) * l.chunks_x, left = end - at;
            w.weight = at >= rest;
            chunks = w.weight ? l.chunks_w : l.chunks_x;
            const long long here = w.weight ? at - rest : at;
            tile = (int)(here / chunks);
            w.k0 = (int)(here - (long long)tile * chunks);
            w.k1 = chunks - w.k0 < left ? chunks : (int)(w.k0 + left);
            if (!w.weight) tile += l.whole;
            w.slot = 2 * who + (at == first ? 0 : 1);
            at += w.k1 - w.k0;
            wanted = w.weight ? l.dw : l.dx;
        }
        w.mt = tile / l.tiles_n;
        w.nt = tile - w.mt * l.tiles_n;
        w.whole = w.k0 == 0 && w.k1 == chunks;
        return true;
    }
};

// LONG: some sum is longer than GatedTerms::kMost.  Its pieces come in the first accumulator, and the epilogue's warps keep their sum, each its own part, in the
// second one.
template <typename T, GatedMode MODE, int BN, bool LONG> __global__ void __launch_bounds__(kThreads, 1) gated_kernel(const __grid_constant__ GatedArgs p) {
    using S = GatedShape<T, MODE, BN>;
    using E = typename GatedTerms<T>::E;
    constexpr int kPairs = GatedTerms<T>::kPairs, kStages = S::kStages;
    constexpr bool PAIR = S::kPair;
    extern __shared__ unsigned char smem_raw[];
    __shared__ int s_dead, s_largest;
    __shared__ uint32_t s_tmem;
    constexpr bool kScaled = MODE >= kGrad && std::is_same<T, __half>::value;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t rank = PAIR ? cluster_rank() : 0u;
    const int who = PAIR ? blockIdx.x / 2 : blockIdx.x, count = PAIR ? gridDim.x / 2 : gridDim.x;

    if (MODE == kGrad && kScaled && p.again) {
        pdl_wait_prior();
        if (gated_scale(p.largest, p.largest_parts, lane) == 1.f) return;      // (all threads of all blocks; what follows waits for this kernel's end)
    }
    Pipe pp;
    pp.status = p.status;
    pp.dead = &s_dead;
    pp.bars = base;
    if (tid < kBars) mbar_init(pp.bars + 8 * tid, tid >= BAR_READ && tid < BAR_DRAIN ? (PAIR ? 2 : 1) * kEpiWarps : 1u);
    if (tid == 0) s_dead = s_largest = 0;
    if (warp <= (kBars - 1) / 32) mbar_fence_init();
    if (warp == kEpiWarps) {
        if (PAIR) tmem_alloc_pair<512>(smem_u32(&s_tmem));
        else tmem_alloc<512>(smem_u32(&s_tmem));
    }
    if (warp == kEpiWarps + 1 && lane == 0) {
        prefetch_map(&p.a[0]);
        prefetch_map(&p.b[PAIR && MODE != kProducts ? rank : 0]);
        if (MODE == kProducts) {
            prefetch_map(&p.a[1]);
            prefetch_map(&p.b[1]);
            prefetch_map(&p.w[rank]);
            prefetch_map(&p.x);
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    if (PAIR) cluster_sync();
    tc_fence_after_sync();
    pp.tmem = s_tmem;
    pdl_wait_prior();
    pdl_release_next();

    const int chunks_f = (p.F + 63) / 64;
    const int pairs = MODE == kProducts && kPairs == 1 ? p.terms : kPairs;
    // fp32: tensor memory cuts the last bit off at every step of a sum, which shows from some hundred summands on; the two accumulators have a half of the sum
    // each and are added in the epilogue, instead of taking turns.  Relative error with one accumulator, with two, and of sums in plain fp32: H of 64 x 640 x 2560
    // 1.2e-6, 0.6e-6, 0.7e-6, its dX 1.1e-6, 0.5e-6, 0.7e-6; dW of 30000 x 64 x 256 1.2e-6, 0.6e-6, 0.8e-6.  It costs H of 1568 x 192 x 512 0.7 of 11.5 us.
    constexpr bool kHalfSums = kPairs > 1;
    [[maybe_unused]] float scale = 1.f, largest = 0.f;
    Walk<MODE, S::kParts, LONG ? GatedTerms<T>::kMost : 0, GatedTerms<T>::kPiece> walk(p, who, count);
    Work t;
    // 16 bits, LONG: sums in one piece take turns with the accumulators (turn: whose it is next); how often each was in use
    int turn = 0, used0 = 0, used1 = 0;

    if (warp == kEpiWarps || warp == kEpiWarps + 2) {
        // ------------------------------------------------------------------ producers: one of A, one of B (a warp issues a load in some 130 cycles)
        const bool of_b = warp != kEpiWarps;
        int stage = 0, round = 0;
        const int half_n = p.line.n / 2, boxes = MODE <= kGrad ? 0 : (half_n + 63) / 64;       // of 64 columns
        const uint32_t bytes = MODE <= kGrad ? S::kStage : kATile + boxes * 8192;              // of this block's share
        const uint32_t full0 = PAIR ? in_block(pipe_bar(pp, BAR_FULL), 0) : pipe_bar(pp, BAR_FULL), elected = elect_lane();
        bool alive = true;
        while (alive && walk.next(t)) {
            for (int pair = 0; pair < pairs; ++pair) {
                int ta = pairs - 1 - pair, tb = 0;
                if (kPairs > 1) term_pair(pair, ta, tb);
                for (int k = t.k0; k < t.k1 && alive; ++k) {
                    if (round > 0 && !mbar_test(pipe_bar(pp, BAR_EMPTY + stage), (round - 1) & 1u)) {
                        wait_spin(pp, BAR_EMPTY + stage, round - 1, kTimeoutRole);
                        if (pipe_dead(pp)) { alive = false; break; }
                    }
                    const uint32_t bar = full0 + 8 * stage, da = base + 1024 + stage * S::kStage, db = da + kATile;
                    const int op = MODE == kProducts && !t.weight && k >= chunks_f, kk = k - op * chunks_f;
                    if (!of_b) {
                        if (rank == 0) mbar_arrive_expect_tx_e(elected, pipe_bar(pp, BAR_FULL + stage), (PAIR ? 2 : 1) * bytes);
                        if (MODE == kProducts && t.weight) {                                    // one block has dG's columns, the other dU's
                            tma_load_3d_e<PAIR>(elected, da, &p.w[rank], 128 * t.mt, 64 * k, ta, bar);
                            tma_load_3d_e<PAIR>(elected, da + 8192, &p.w[rank], 128 * t.mt + 64, 64 * k, ta, bar);
                        } else {
                            tma_load_3d_e<PAIR>(elected, da, &p.a[op], 64 * kk, (PAIR ? 256 : 128) * t.mt + 128 * rank, ta, bar);
                        }
                    } else if constexpr (MODE <= kGrad) {
                        if (PAIR) {
                            tma_load_3d_e<PAIR>(elected, db, &p.b[rank], 64 * k, BN * t.nt, tb, bar);     // one block has the gate's rows, the other the rest
                        } else {
                            tma_load_3d_e<PAIR>(elected, db, &p.b[0], 64 * k, BN * t.nt, tb, bar);
                            tma_load_3d_e<PAIR>(elected, db + BN * 128, &p.b[1], 64 * k, BN * t.nt, tb, bar);
                        }
                    } else {
                        const int c0 = p.line.n * t.nt + half_n * rank;
                        const CUtensorMap* map = t.weight ? &p.x : &p.b[op];
                        tma_load_3d_e<PAIR>(elected, db, map, c0, 64 * kk, tb, bar);
                        if (boxes > 1) tma_load_3d_e<PAIR>(elected, db + 8192, map, c0 + 64, 64 * kk, tb, bar);
                    }
                    if (++stage == kStages) { stage = 0; ++round; }
                }
            }
        }
        // no copy, and no arrival of the pair's products, may be under way at the block's end, whatever became of the other roles
        for (int s = 0; s < kStages; ++s) {
            const int last = s < stage ? round : round - 1;
            if (last < 0) continue;
            if (rank == 0) mbar_wait_bounded(pipe_bar(pp, BAR_FULL + s), last & 1, 1u << 16);
            if (!pipe_dead(pp)) mbar_wait_bounded(pipe_bar(pp, BAR_EMPTY + s), last & 1, 1u << 20);
        }
        __syncwarp();
    } else if (warp == kEpiWarps + 1) {
        // ------------------------------------------------------------------ products
        if (rank == 0) {
            constexpr int fmt = Elem<E>::kIsBf16 ? 1 : 0;
            const uint32_t id = umma_idesc(fmt, PAIR ? 256 : 128, MODE <= kGrad ? 2 * BN : p.line.n, MODE == kProducts);
            const uint32_t elected = elect_lane();
            int stage = 0, round = 0, ord = 0;
            bool alive = true, there = false;                          // whether the stage's tiles were seen to be there already
            for (; alive && walk.next(t); ++ord) {
                int buf = kHalfSums ? 0 : ord & 1, use = kHalfSums ? ord : ord >> 1;
                if (LONG && !kHalfSums) {
                    buf = t.cut ? 0 : turn;
                    use = buf ? used1++ : used0++;
                    if (!t.cut) turn ^= 1;
                    else if (t.last) ++used1;                          // the epilogue reads the sum of the pieces there
                }
                const int middle = LONG && t.cut ? t.k1 : (t.k0 + t.k1 + 1) >> 1;
                if (use > 0) wait_spin(pp, BAR_READ + buf, use - 1, kTimeoutRole);
                tc_fence_after_sync();
                uint32_t d = pp.tmem + 256 * buf;
                const bool weight = MODE == kProducts && t.weight;
                // half of a tile: 64 hidden units, those of each block's rows of B that begin at 0 or at 64
                const uint32_t id_here = S::kParts > 1 && t.part ? umma_idesc(fmt, 256, BN, 0) : id, b_at = kATile + (S::kParts > 1 && t.part == 2 ? 64 * 128 : 0);
                const int total = MODE <= kGrad ? p.C : weight ? p.M : p.F;
                uint32_t acc = 0;
                for (int pair = 0; pair < pairs; ++pair)
                    for (int k = t.k0; k < t.k1 && alive; ++k) {
                        if (!there) {
                            wait_spin(pp, BAR_FULL + stage, round, kTimeoutTile);
                            alive = !pipe_dead(pp);
                        }
                        tc_fence_after_sync();
                        if (kHalfSums) {
                            d = pp.tmem + (k < middle ? 0 : 256);
                            acc = pair > 0 || (k != t.k0 && k != middle);
                        }
                        const uint32_t at = base + 1024 + stage * S::kStage, empty = pipe_bar(pp, BAR_EMPTY + stage);
                        const int kk = MODE == kProducts && !weight && k >= chunks_f ? k - chunks_f : k, left = total - 64 * kk;
                        if (++stage == kStages) { stage = 0; ++round; }
                        there = mbar_test(pipe_bar(pp, BAR_FULL + stage), round & 1u);     // (asked before the instructions are queued)
                        // descriptor addresses count 16 bytes: a step of 16 is 2 along a K-major row, 128 down MN-major ones
                        auto issue = [&](auto ka, auto kb, uint64_t da, uint64_t db, uint32_t desc) {
                            constexpr int kA = decltype(ka)::value, kB = decltype(kb)::value;
                            if (left > 48) {
                                umma_four<PAIR, kA, kB>(elected, d, da, db, desc, acc);
                            } else {
                                for (int s = 0; 16 * s < left; ++s) umma_step<PAIR>(elected, d, da + kA * s, db + kB * s, desc, s ? 1u : acc);
                            }
                        };
                        using Row = std::integral_constant<int, 2>;
                        using Column = std::integral_constant<int, 128>;
                        if (MODE <= kGrad) issue(Row(), Row(), umma_desc_sw128(at), umma_desc_sw128(at + b_at), id_here);
                        else if (weight) issue(Column(), Column(), desc_mn(at, 8192), desc_mn(at + kATile, 8192), id | 1u << 15);
                        else issue(Row(), Column(), umma_desc_sw128(at), desc_mn(at + kATile, 8192), id);
                        acc = 1u;
                        umma_commit_e<PAIR>(elected, empty);
                    }
                umma_commit_e<PAIR>(elected, pipe_bar(pp, BAR_ACC + buf));
            }
            if (PAIR) umma_commit_first(elected, pipe_bar(pp, BAR_DRAIN));
            else umma_commit_e<false>(elected, pipe_bar(pp, BAR_DRAIN));
            mbar_wait_bounded(pipe_bar(pp, BAR_DRAIN), 0u, 1u << 20);
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------------------ epilogue
        // warp: 32 rows, and a quarter of a tile's hidden units (kForward, kGrad) or every fourth block of 32 columns
        const int q = warp & 3, quarter = warp >> 2;
        if constexpr (kScaled)
            if (MODE == kProducts || p.again) scale = gated_scale(p.largest, p.largest_parts, lane);
        const uint32_t patch = base + S::kOffPatch + warp * S::kPatch;
        const uint32_t read0 = PAIR ? in_block(pipe_bar(pp, BAR_READ), 0) : pipe_bar(pp, BAR_READ), elected = elect_lane();
        int ord = 0;
        auto release = [&](int buf) {
            tc_fence_before_sync();
            arrive_warp_e<PAIR>(elected, read0 + 8 * buf);
        };
        auto mine_too = [&](const Work& t) { return S::kParts == 1 || t.part == 0 || (quarter >> 1) == t.part - 1; };      // whether this warp has some of the tile
        auto column_at = [&](const Work& t) { return S::kParts > 1 && t.part ? 32 * (quarter & 1) : 32 * quarter; };       // of G in the accumulator (BN = 128)
        // accumulator of the next sum or piece, and the parity of its arrival
        auto accumulator = [&](const Work& t, int& parity) {
            if (!LONG || kHalfSums) {
                parity = kHalfSums ? ord : ord >> 1;
                return kHalfSums ? 0 : ord & 1;
            }
            const int buf = t.cut ? 0 : turn;
            parity = buf ? used1++ : used0++;
            if (!t.cut) turn ^= 1;
            return buf;
        };
        // a piece's columns of this warp are added to the sum
        auto add_piece = [&](const Work& t, int col, int n) {
#pragma unroll 1
            for (int c = col; c < col + n; c += 16) {
                const uint32_t at = pp.tmem + ((uint32_t)(32 * q) << 16) + c;
                float v[16];
                __syncwarp();
                tmem_ld16(at, v);
                tmem_ld_wait();
                if (!t.first) {
                    float w[16];
                    tmem_ld16(at + 256, w);
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[i] += w[i];
                }
                uint32_t o[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(v[i]);
                tmem_st16(at + 256, o);
                tmem_st_wait();
            }
        };
        // after a piece: whether the sum is there (in the second accumulator)
        auto summed = [&](const Work& t) {
            if (!kHalfSums || !t.last) release(0);                     // (fp32: what it reserves are both, until the sum has been read)
            return t.last;
        };
        auto await = [&](int bar, int parity) {
            if (!mbar_test(pipe_bar(pp, bar), parity & 1)) wait_par(pp, bar, parity, kTimeoutTile);
        };
        if constexpr (MODE <= kGrad && S::kStaged) {
            // Results leave through a patch of 32 rows of 64 bytes with their swizzle.  kGrad: dU has one patch, dG two in turn, in which dH arrives a
            // tile ahead and is overwritten.
            const uint32_t bias = base + S::kOffBias + warp * 256;
            const uint32_t matrix = 64 * (lane & 15), piece = lane >> 4, swz = (lane >> 1) & 3;      // this lane's row of four 8 x 8 values
            // An accumulator is read as 16 x 256 bits: a lane has rows lane / 4 and that plus 8, hidden units 8 j + 2 (lane % 4) and the next, so that it keeps
            // sums of its columns over all of a run's rows in registers, and the eight lanes that share them meet when the columns change.
            float2 column[2][4] = {};                                  // dG, dU
            int column_nt = -1;
            auto flush = [&] {
                const int first = (int)(((2ll * column_nt * p.tiles_m + 1) * count - 1) / (2ll * p.tiles_m * p.tiles_n));
                float* dst = p.column + (size_t)(8 * (who - first) + 4 * rank + q) * 2 * p.F;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    float2 v = column[k >> 2][k & 3];
                    column[k >> 2][k & 3] = both(0.f);
#pragma unroll
                    for (int o = 4; o < 32; o *= 2) v = fadd2(v, make_float2(__shfl_xor_sync(0xffffffffu, v.x, o), __shfl_xor_sync(0xffffffffu, v.y, o)));
                    const int f = BN * column_nt + 32 * quarter + 8 * (k & 3) + 2 * (lane & 3);
                    if (lane >> 2 == k && f < p.F) *reinterpret_cast<float2*>(dst + (size_t)(k >> 2) * p.F + f) = v;
                }
            };
            auto fetch = [&](const Work& t, int i) {                   // dH of tile i
                const uint32_t bar = pipe_bar(pp, BAR_DH + warp);
                mbar_arrive_expect_tx_e(elected, bar, kHalfPatch);
                tma_load_3d_e<false>(elected, patch + kHalfPatch * (i & 1), &p.g, BN * t.nt + 32 * quarter, 256 * t.mt + 128 * rank + 32 * q, 0, bar);
            };
            Work ahead;
            bool more = walk.next(ahead);
            int done = 0;                                              // tiles that this warp had some of
            if (MODE == kGrad && !LONG && more && mine_too(ahead)) fetch(ahead, 0);
            const bool biased = p.bg || p.bu;
            int bias_nt = -1;
            for (; more; ++ord) {
                t = ahead;
                more = walk.next(ahead);
                const int row0 = 256 * t.mt + 128 * rank + 32 * q, f0 = BN * t.nt + 32 * quarter, up = S::kParts > 1 && t.part ? BN / 2 : BN;
                int parity, buf = accumulator(t, parity);
                if (LONG && t.cut) {
                    await(BAR_ACC + buf, parity);
                    tc_fence_after_sync();
                    if (mine_too(t)) {
                        add_piece(t, column_at(t), 32);
                        add_piece(t, column_at(t) + up, 32);
                    }
                    if (!summed(t)) continue;
                    buf = 1;
                }
                const uint32_t acc = pp.tmem + 256 * buf + ((uint32_t)(32 * q) << 16) + column_at(t);
                if (MODE == kGrad && p.column && column_nt != t.nt) {
                    if (column_nt >= 0) flush();
                    column_nt = t.nt;
                }
                if (!mine_too(t)) {
                    if (!LONG || !t.cut) await(BAR_ACC + buf, parity);
                    release(buf);
                    if (MODE == kGrad && !LONG && more && mine_too(ahead)) fetch(ahead, done);
                    __syncwarp();
                    continue;
                }
                if (biased && bias_nt != t.nt) {                       // as fp32: [gate | up][32]
                    bias_nt = t.nt;
                    const int f = f0 + 2 * (lane & 15);
                    const void* src = lane < 16 ? p.bg : p.bu;
                    float2 b = both(0.f);
                    if (src && f < p.F) b = unpack2<T>(__ldg(reinterpret_cast<const uint32_t*>(static_cast<const T*>(src) + f)));
                    __syncwarp();
                    asm volatile("st.shared.v2.f32 [%0], {%1, %2};\n" ::"r"(bias + 8 * lane), "f"(b.x), "f"(b.y) : "memory");
                    __syncwarp();
                }
                if (!LONG || !t.cut) await(BAR_ACC + buf, parity);
                tc_fence_after_sync();
                store_wait_read<0>();                                  // the tile before has left the patches
                __syncwarp();
                const uint32_t mine = patch + (MODE == kGrad ? kHalfPatch * (done & 1) : 0), other = patch + 2 * kHalfPatch;
                if (MODE == kGrad) {
                    if (LONG) fetch(t, done);                          // (not ahead: pieces may come between)
                    await(BAR_DH + warp, done);
                    if (!LONG && more && mine_too(ahead)) fetch(ahead, done + 1);
                }
                ++done;
                by_activation(p.act, [&](auto act) {
#pragma unroll 1
                    for (int h = 0; h < 2; ++h) {                      // 16 rows
                        float g[16], v[16];
                        __syncwarp();
                        tmem_ld_16x256b_x4(acc + ((uint32_t)(16 * h) << 16), g);
                        tmem_ld_16x256b_x4(acc + ((uint32_t)(16 * h) << 16) + up, v);
                        tmem_ld_wait();
                        if (h == 1) release(buf);
#pragma unroll
                        for (int c = 0; c < 2; ++c) {                  // 16 hidden units
                            const uint32_t at = mine + matrix + 1024 * h + (((2 * c + piece) ^ swz) << 4);
                            float2 gg[4], vv[4];                       // [2 j + i]: hidden units 8 j + 2 (lane % 4), row lane / 4 + 8 i
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                gg[i] = make_float2(g[8 * c + 2 * i], g[8 * c + 2 * i + 1]);
                                vv[i] = make_float2(v[8 * c + 2 * i], v[8 * c + 2 * i + 1]);
                            }
                            if (biased) {
#pragma unroll
                                for (int j = 0; j < 2; ++j) {
                                    const uint32_t b = bias + 64 * c + 32 * j + 8 * (lane & 3);
                                    const float2 x = ld_shared_pair(b), y = ld_shared_pair(b + 128);
#pragma unroll
                                    for (int i = 0; i < 2; ++i) {
                                        gg[2 * j + i] = fadd2(gg[2 * j + i], x);
                                        vv[2 * j + i] = fadd2(vv[2 * j + i], y);
                                    }
                                }
                            }
                            uint32_t o0[4];
                            if constexpr (MODE == kForward) {
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    float2 a, da;
                                    activate<T, decltype(act)::value, false>(gg[i], a, da);
                                    a = fmul2(a, vv[i]);
                                    o0[i] = pack2<T>(a.x, a.y);
                                }
                            } else {
                                uint32_t d[4], o1[4];
                                [[maybe_unused]] float sizes[16];
                                ld_matrix4(d, at);
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    float2 a, da;
                                    activate<T, decltype(act)::value, true>(gg[i], a, da);
                                    const float2 dh = unpack2<T>(d[i]);
                                    da = fmul2(fmul2(dh, vv[i]), da);
                                    a = fmul2(dh, a);
                                    if constexpr (kScaled) {
                                        const float2 x = fmul2(da, both(scale)), y = fmul2(a, both(scale));
                                        o0[i] = pack2<T>(x.x, x.y);
                                        o1[i] = pack2<T>(y.x, y.y);
                                        sizes[4 * i] = da.x; sizes[4 * i + 1] = da.y; sizes[4 * i + 2] = a.x; sizes[4 * i + 3] = a.y;
                                    } else {
                                        o0[i] = pack2<T>(da.x, da.y);
                                        o1[i] = pack2<T>(a.x, a.y);
                                    }
                                    column[0][2 * c + i / 2] = fadd2(column[0][2 * c + i / 2], da);      // (before they are rounded)
                                    column[1][2 * c + i / 2] = fadd2(column[1][2 * c + i / 2], a);
                                }
                                if constexpr (kScaled) largest = largest_finite(largest, sizes);
                                __syncwarp();
                                st_matrix4(at - mine + other, o1);
                            }
                            st_matrix4(at, o0);
                        }
                    }
                });
                fence_proxy_async();
                __syncwarp();
                if (row0 < p.M && f0 < p.F) {
                    tma_store_3d_e(elected, &p.s[0], f0, row0, 0, mine);
                    if (MODE == kGrad) tma_store_3d_e(elected, &p.s[1], f0, row0, 0, other);
                }
                store_commit();
                __syncwarp();
            }
            if (MODE == kGrad && p.column && column_nt >= 0) flush();
            store_wait_read<0>();
            __syncwarp();
        } else if constexpr (MODE <= kGrad) {
            constexpr int kCols = BN / 4 > 16 ? BN / 4 : 16;           // of a warp (BN = 32: half of the warps have none)
            for (; walk.next(t); ++ord) {
                const int row = (PAIR ? 256 : 128) * t.mt + 128 * rank + 32 * q + lane, up = S::kParts > 1 && t.part ? BN / 2 : BN;
                const size_t plane = (size_t)p.M * p.F;
                const bool mine = quarter * kCols < BN && mine_too(t);
                int parity, buf = accumulator(t, parity);
                await(BAR_ACC + buf, parity);
                tc_fence_after_sync();
                if (LONG && t.cut) {
                    if (mine) {
                        add_piece(t, PAIR ? column_at(t) : quarter * kCols, kCols);
                        add_piece(t, (PAIR ? column_at(t) : quarter * kCols) + up, kCols);
                    }
                    if (!summed(t)) continue;
                    buf = 1;
                }
                const uint32_t acc = pp.tmem + 256 * buf + ((uint32_t)(32 * q) << 16);
                const int lent = kHalfSums ? 0 : buf;
                if (!mine) {
                    release(lent);
                    continue;
                }
                by_activation(p.act, [&](auto act) {
#pragma unroll 1
                    for (int s = 0; s < kCols / 16; ++s) {
                        const int col = quarter * kCols + 16 * s, f0 = BN * t.nt + col, at_col = PAIR ? column_at(t) + 16 * s : col;
                        float g[16], v[16];
                        __syncwarp();
                        tmem_ld16(acc + at_col, g);
                        tmem_ld16(acc + up + at_col, v);
                        tmem_ld_wait();
                        if (kHalfSums && p.chunks > 1 && !(LONG && t.cut)) {
                            float g2[16], v2[16];
                            tmem_ld16(acc + 256 + at_col, g2);
                            tmem_ld16(acc + 256 + up + at_col, v2);
                            tmem_ld_wait();
#pragma unroll
                            for (int i = 0; i < 16; ++i) { g[i] += g2[i]; v[i] += v2[i]; }
                        }
                        if (s == kCols / 16 - 1) release(lent);
#pragma unroll
                        for (int j = 0; j < 16; j += 8) {
                            const int f = f0 + j;
                            if (f >= p.F || row >= p.M) {
#pragma unroll
                                for (int i = j; i < j + 8; ++i) g[i] = v[i] = 0.f;
                                continue;
                            }
                            if (p.bg) {
                                float b[8];
                                load8<T>(static_cast<const T*>(p.bg) + f, b);
#pragma unroll
                                for (int i = 0; i < 8; ++i) g[j + i] += b[i];
                            }
                            if (p.bu) {
                                float b[8];
                                load8<T>(static_cast<const T*>(p.bu) + f, b);
#pragma unroll
                                for (int i = 0; i < 8; ++i) v[j + i] += b[i];
                            }
                            const size_t at = (size_t)row * p.F + f;
                            float dh[8];
                            if (MODE == kGrad) load8<T>(static_cast<const T*>(p.dh) + at, dh);
#pragma unroll
                            for (int i = j; i < j + 8; i += 2) {
                                float2 a, da;
                                activate<T, decltype(act)::value, MODE == kGrad>(make_float2(g[i], g[i + 1]), a, da);
                                if (MODE == kForward) {
                                    v[i] *= a.x; v[i + 1] *= a.y;
                                } else {
                                    g[i] = dh[i - j] * v[i] * da.x; g[i + 1] = dh[i + 1 - j] * v[i + 1] * da.y;
                                    v[i] = dh[i - j] * a.x; v[i + 1] = dh[i + 1 - j] * a.y;
                                }
                            }
                            if constexpr (MODE == kForward) {
                                store8<T>(static_cast<T*>(p.out0) + at, v + j);
                            } else if constexpr (kScaled) {
                                float x[8], y[8];
#pragma unroll
                                for (int i = 0; i < 8; ++i) { x[i] = g[j + i]; y[i] = v[j + i]; }
                                largest = largest_finite(largest_finite(largest, x), y);
#pragma unroll
                                for (int i = 0; i < 8; ++i) { x[i] *= scale; y[i] *= scale; }
                                store_operand8<T>(p.out0, plane, at, x, p.terms > 1);
                                store_operand8<T>(p.out1, plane, at, y, p.terms > 1);
                            } else {
                                store_operand8<T>(p.out0, plane, at, g + j, p.terms > 1);
                                store_operand8<T>(p.out1, plane, at, v + j, p.terms > 1);
                            }
                        }
                        if (MODE == kGrad && p.column) {               // sums of the warp's rows, a slot for every 32
                            __syncwarp();
                            const float sg = sum_lanes16(g, lane), su = sum_lanes16(v, lane);
                            const int f = f0 + (lane >> 1);
                            if (!(lane & 1) && f < p.F && row - lane < p.M) {
                                float* dst = p.column + (size_t)(row >> 5) * 2 * p.F + f;
                                dst[0] = sg;
                                dst[p.F] = su;
                            }
                        }
                    }
                });
                __syncwarp();
            }
        } else {
            // boxes of 32 columns and 32 rows, those of a tile in turn by the four warps that share its rows
            [[maybe_unused]] const float back = 1.f / scale;
            for (; walk.next(t); ++ord) {
                const int blocks = p.line.n / 32, limit = t.weight ? p.F : p.M;
                const int in_tile = 128 * rank + 32 * q, row0 = t.weight ? 128 * t.mt + 32 * q : 256 * t.mt + in_tile;
                const CUtensorMap* map = !t.whole ? &p.share : t.weight ? &p.s[1 + rank] : &p.s[0];
                const bool wide = sizeof(T) == 4 || !t.whole;
                int parity, buf = accumulator(t, parity);
                await(BAR_ACC + buf, parity);
                tc_fence_after_sync();
                if (LONG && t.cut) {
                    for (int b = quarter; b < blocks; b += 4) add_piece(t, 32 * b, 32);
                    if (!summed(t)) continue;
                    buf = 1;
                }
                const uint32_t acc = pp.tmem + 256 * buf + ((uint32_t)(32 * q) << 16);
                const int lent = kHalfSums ? 0 : buf;
#pragma unroll 1
                for (int b = quarter; b < blocks; b += 4) {
                    float v[32];
                    __syncwarp();
                    tmem_ld32(acc + 32 * b, reinterpret_cast<uint32_t(&)[32]>(v));
                    tmem_ld_wait();
                    if (kHalfSums && t.k1 - t.k0 > 1 && !(LONG && t.cut)) {
#pragma unroll
                        for (int i = 0; i < 32; i += 16) {
                            float w[16];
                            tmem_ld16(acc + 256 + 32 * b + i, w);
                            tmem_ld_wait();
#pragma unroll
                            for (int j = 0; j < 16; ++j) v[i + j] += w[j];
                        }
                    }
                    if (b + 4 >= blocks) release(lent);
                    if constexpr (kScaled) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] *= back;
                    }
                    store_wait_read<0>();
                    __syncwarp();
                    if (wide) {                                        // rows of 128 bytes
#pragma unroll
                        for (int c = 0; c < 8; ++c) st_shared4(patch + 128 * lane + ((c ^ (lane & 7)) << 4), pack16<float>(v + 4 * c));
                    } else if constexpr (sizeof(T) == 2) {             // rows of 64 bytes
#pragma unroll
                        for (int c = 0; c < 4; ++c) st_shared4(patch + 64 * lane + ((c ^ ((lane >> 1) & 3)) << 4), pack16<T>(v + 8 * c));
                    }
                    fence_proxy_async();
                    __syncwarp();
                    const int c0 = p.line.n * t.nt + 32 * b;
                    if (row0 < limit && c0 < p.C) tma_store_3d_e(elected, map, t.whole ? c0 : 32 * b, t.whole ? row0 : in_tile, t.whole ? 0 : t.slot, patch);
                    store_commit();
                }
                if (quarter >= blocks) release(lent);
                __syncwarp();
            }
            store_wait_read<0>();
            __syncwarp();
        }
    }
    if constexpr (MODE == kGrad && kScaled) {
#pragma unroll
        for (int o = 16; o; o >>= 1) largest = fmaxf(largest, __shfl_xor_sync(0xffffffffu, largest, o));
        if (lane == 0) atomicMax(&s_largest, __float_as_int(largest));         // (of numbers that are not negative the order is that of their bits)
    }
    tc_fence_before_sync();
    __syncthreads();
    if constexpr (MODE == kGrad && kScaled)
        if (tid == 0 && !p.again) p.largest[blockIdx.x] = __int_as_float(s_largest);
    if (PAIR) {
        cluster_sync();                                               // the other block's instructions read this one's memory
        if (warp == kEpiWarps) tmem_dealloc_pair<512>(pp.tmem);
    } else if (warp == kEpiWarps) {
        tmem_dealloc<512>(pp.tmem);
    }
}

// Forward pass of small fp32 problems on the CUDA cores, in one launch: a block has 32 rows and 32 hidden units of G and U, a thread four rows and two
// units of both.  Against terms and tensor cores (rows x channels x hidden units, us): 196 x 192 x 512 6.6 and 9.8, 512 x 192 x 512 9.0 and 10.0, 4096 x 64 x 256
// 11.2 and 9.2, 196 x 320 x 1280 13.7 and 13.4, 1024 x 192 x 512 15.2 and 11.3; it saves a launch and a workspace besides.
constexpr long long kSmallProducts = 50000000;
constexpr int kSmallThreads = 128, kSmallTile = 32, kSmallK = 32, kSmallPitch = kSmallK + 4, kSmallStages = 4;      // (pitch: eight rows in different banks)
constexpr int kSmallSmem = kSmallStages * 3 * kSmallTile * kSmallPitch * 4;
__global__ void __launch_bounds__(kSmallThreads) gated_small_kernel(const float* x, const float* wg, const float* wu, const float* bg, const float* bu, int M, int C, int F, int act, float* out) {
    extern __shared__ __align__(16) float s_small[];      // [stage][X, Wg, Wu][row or unit][channel]
    pdl_wait_prior();
    pdl_release_next();
    const int tid = threadIdx.x, m0 = kSmallTile * blockIdx.y, f0 = kSmallTile * blockIdx.x;
    const int chunks = (C + kSmallK - 1) / kSmallK, lr = tid >> 3, lc = 4 * (tid & 7);
    auto fetch = [&](int chunk) {
        if (chunk < chunks) {
            float* to = s_small + (chunk % kSmallStages) * 3 * kSmallTile * kSmallPitch;
            const int c = kSmallK * chunk + lc;
#pragma unroll
            for (int i = 0; i < 3 * kSmallTile / 16; ++i) {
                const int which = i / 2, row = 16 * (i % 2) + lr, at = (which ? f0 : m0) + row;
                const bool there = c < C && at < (which ? F : M);
                const float* src = which == 0 ? x : which == 1 ? wg : wu;
                cp_async16(to + (which * kSmallTile + row) * kSmallPitch + lc, there ? src + (size_t)at * C + c : src, there ? 16 : 0);
            }
        }
        cp_async_commit();
    };
#pragma unroll
    for (int i = 0; i < kSmallStages - 1; ++i) fetch(i);
    const int row = tid & 7, unit = tid >> 3;             // rows row + 8 i, units unit + 16 j
    float g[4][2] = {}, u[4][2] = {}, gs[4][2] = {}, us[4][2] = {};      // sums of 256 channels, and of these
    for (int chunk = 0; chunk < chunks; ++chunk) {
        cp_async_wait<kSmallStages - 2>();
        __syncthreads();
        fetch(chunk + kSmallStages - 1);                  // into the stage that all have read before the barrier
        const float* at = s_small + (chunk % kSmallStages) * 3 * kSmallTile * kSmallPitch;
#pragma unroll
        for (int k = 0; k < kSmallK; k += 4) {
            float4 a[4], p[2], q[2];
#pragma unroll
            for (int i = 0; i < 4; ++i) a[i] = *reinterpret_cast<const float4*>(at + (row + 8 * i) * kSmallPitch + k);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                p[j] = *reinterpret_cast<const float4*>(at + (kSmallTile + unit + 16 * j) * kSmallPitch + k);
                q[j] = *reinterpret_cast<const float4*>(at + (2 * kSmallTile + unit + 16 * j) * kSmallPitch + k);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    g[i][j] = fmaf(a[i].w, p[j].w, fmaf(a[i].z, p[j].z, fmaf(a[i].y, p[j].y, fmaf(a[i].x, p[j].x, g[i][j]))));
                    u[i][j] = fmaf(a[i].w, q[j].w, fmaf(a[i].z, q[j].z, fmaf(a[i].y, q[j].y, fmaf(a[i].x, q[j].x, u[i][j]))));
                }
        }
        if (chunk % 8 == 7 || chunk == chunks - 1) {      // (one sum of 8192 channels is off by 2.1e-6)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    gs[i][j] += g[i][j];
                    us[i][j] += u[i][j];
                    g[i][j] = u[i][j] = 0.f;
                }
        }
    }
    cp_async_wait<0>();
    by_activation(act, [&](auto a) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int f = f0 + unit + 16 * j;
            if (f >= F) continue;
            const float b = bg ? bg[f] : 0.f, d = bu ? bu[f] : 0.f;
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
                float2 v, unused;
                activate<float, decltype(a)::value, false>(make_float2(gs[i][j] + b, gs[i + 1][j] + b), v, unused);
                const int m = m0 + row + 8 * i;
                if (m < M) out[(size_t)m * F + f] = v.x * (us[i][j] + d);
                if (m + 8 < M) out[(size_t)(m + 8) * F + f] = v.y * (us[i + 1][j] + d);
            }
        }
    });
}

// Forward pass of few rows (single tokens): bound by the weights' bytes.  A warp has two hidden units and all rows, its lanes 16 bytes of channels at
// a time; the weights are read once, the rows come from L1.  1024 channels, 4096 hidden units, bf16: one row 2.7 us (6.2 TB/s of weights that L2 holds; 10.6 on the
// tensor cores, whose tiles of 128 rows are one row full), four 5.4 (10.8), eight 8.6 (9.8); 320 channels, 1280 units: 1.7, 2.9 (4.3), 4.5 (4.5), sixteen
// rows 7.0 (4.3).  fp32, one row: 4.0 (70, the weights' terms).
constexpr int kFewThreads = 128, kFewUnits = 2;
template <typename T, int ROWS> __global__ void __launch_bounds__(kFewThreads) gated_few_kernel(const T* x, const T* wg, const T* wu, const T* bg, const T* bu, int M, int C, int F, int act, T* out) {
    constexpr int V = Elem<T>::kVec;
    pdl_wait_prior();
    pdl_release_next();
    const int lane = threadIdx.x & 31, f0 = kFewUnits * (blockIdx.x * (kFewThreads / 32) + (threadIdx.x >> 5)), m0 = ROWS * blockIdx.y;
    if (f0 >= F) return;                                  // (F is a multiple of eight)
    float2 sum[ROWS][2 * kFewUnits] = {};                 // [row][gate, up of each unit], two halves
#pragma unroll 2
    for (int c = V * lane; c < C; c += 32 * V) {
        float w[2 * kFewUnits][V];
#pragma unroll
        for (int i = 0; i < kFewUnits; ++i) {
            unpack16<T>(__ldg(reinterpret_cast<const uint4*>(wg + (size_t)(f0 + i) * C + c)), w[2 * i]);
            unpack16<T>(__ldg(reinterpret_cast<const uint4*>(wu + (size_t)(f0 + i) * C + c)), w[2 * i + 1]);
        }
#pragma unroll
        for (int m = 0; m < ROWS; ++m) {
            float a[V] = {};
            if (m0 + m < M) unpack16<T>(__ldg(reinterpret_cast<const uint4*>(x + (size_t)(m0 + m) * C + c)), a);
#pragma unroll
            for (int i = 0; i < 2 * kFewUnits; ++i)
#pragma unroll
                for (int j = 0; j < V; j += 2) sum[m][i] = ffma2(make_float2(a[j], a[j + 1]), make_float2(w[i][j], w[i][j + 1]), sum[m][i]);
        }
    }
    float g = 0.f, u = 0.f;                               // of row lane / kFewUnits, unit lane % kFewUnits
#pragma unroll
    for (int m = 0; m < ROWS; ++m)
#pragma unroll
        for (int i = 0; i < 2 * kFewUnits; ++i) {
            float v = sum[m][i].x + sum[m][i].y;
#pragma unroll
            for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
            if (lane == kFewUnits * m + i / 2) (i % 2 ? u : g) = v;
        }
    const int m = m0 + lane / kFewUnits, f = f0 + lane % kFewUnits;
    if (lane >= ROWS * kFewUnits || m >= M) return;
    if (bg) g += Elem<T>::to_f32(bg[f]);
    if (bu) u += Elem<T>::to_f32(bu[f]);
    by_activation(act, [&](auto a) {
        float2 v, unused;
        activate<T, decltype(a)::value, false>(both(g), v, unused);
        out[(size_t)m * F + f] = Elem<T>::from_f32(v.x * u);
    });
}
constexpr int kFewRows = 8;
bool few_forward(int M) { return M <= kFewRows; }
bool small_forward(int dtype, int M, int C, int F) { return dtype == kF32 && (long long)M * C * F <= kSmallProducts; }

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

// What is left after kProducts, always in the same order.  The first blocks: sums of the columns of dG and dU (32 of the 2 F each) over the shares
// that kGrad left: one for every 32 rows (`runs`), or those of the pairs that had the column range.  The others: 1024 values of a tile that no pair
// had whole, as the sum of its shares, whose list the host makes (found by the blocks themselves: 7.0 and 8.4 us instead of 5.8 and 6.1).
constexpr int kMostPairs = 128, kShares = 12;            // shares in flight
struct FinishArgs {
    const float *share, *column;
    void *dx, *dwg, *dwu, *dbg, *dbu;
    GatedLine line;
    int M, C, F;
    int column_blocks, runs, tiles_m, units, count;      // column sums; kGrad's halves of tiles: in a column range, in all
    int tiles;                                           // with shares: which ones, and their slots in their order
    int tile[kMostPairs];
    unsigned short first[kMostPairs + 1];
    unsigned char slot[2 * kMostPairs];
};
// A pair has at most two tiles in part: the first and the last of its run
void list_shares(FinishArgs* f) {
    const GatedLine& l = f->line;
    const long long rest = (long long)(l.tiles_x - l.whole) * l.chunks_x;
    int entries = 0;
    for (int q = 0; q < l.pairs; ++q) {
        const long long first = l.begin(q), end = l.begin(q + 1);
        for (long long at = first; at < end;) {
            const bool weight = at >= rest;
            const int chunks = weight ? l.chunks_w : l.chunks_x, own = (int)((weight ? at - rest : at) / chunks);
            const long long begin = (weight ? rest : 0) + (long long)own * chunks, limit = weight || end < rest ? end : rest;
            if (at == begin && limit - at >= chunks) {                // whole tiles
                at += (limit - at) / chunks * chunks;
                continue;
            }
            if (weight ? l.dw : l.dx) {
                const int tile = weight ? l.tiles_x + own : l.whole + own;
                if (!f->tiles || f->tile[f->tiles - 1] != tile) {
                    f->first[f->tiles] = (unsigned short)entries;
                    f->tile[f->tiles++] = tile;
                }
                f->slot[entries++] = (unsigned char)(2 * q + (at == first ? 0 : 1));
            }
            at = begin + chunks < end ? begin + chunks : end;
        }
    }
    f->first[f->tiles] = (unsigned short)entries;
}
template <typename T> __global__ void __launch_bounds__(256) gated_finish_kernel(const __grid_constant__ FinishArgs p) {
    __shared__ float s_sum[8][32];
    pdl_wait_prior();
    pdl_release_next();
    const int r = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if ((int)blockIdx.x < p.column_blocks) {
        const int i = 32 * blockIdx.x + lane, op = i >= p.F, f = i - op * p.F;
        float v = 0.f;
        if (i < 2 * p.F) {
            int slots = p.runs;
            if (!slots) {
                const int nt = f / 128;
                const int first = (int)((((long long)nt * p.tiles_m + 1) * p.count - 1) / p.units), last = (int)(((long long)(nt + 1) * p.tiles_m * p.count - 1) / p.units);
                slots = 8 * (last - first + 1);
            }
            for (int s = r; s < slots; s += 8 * kShares) {
                float w[kShares];
#pragma unroll
                for (int u = 0; u < kShares; ++u) w[u] = s + 8 * u < slots ? p.column[(size_t)(s + 8 * u) * 2 * p.F + i] : 0.f;
#pragma unroll
                for (int u = 0; u < kShares; ++u) v += w[u];
            }
        }
        s_sum[r][lane] = v;
        __syncthreads();
        if (r == 0 && i < 2 * p.F) {
#pragma unroll
            for (int k = 1; k < 8; ++k) v += s_sum[k][lane];
            static_cast<T*>(op ? p.dbu : p.dbg)[f] = Elem<T>::from_f32(v);
        }
        return;
    }
    const GatedLine& l = p.line;
    const int per = l.n / 4, block = blockIdx.x - p.column_blocks, which = block / per, tile = p.tile[which], e = 1024 * (block - which * per) + 4 * threadIdx.x;
    const bool weight = tile >= l.tiles_x;
    const int own = weight ? tile - l.tiles_x : tile, mt = own / l.tiles_n, nt = own - mt * l.tiles_n;
    const int row = e / l.n, c0 = l.n * nt + e - row * l.n, in_tile = weight ? row & 127 : row;
    if (in_tile >= (weight ? p.F - 128 * mt : p.M - 256 * mt) || c0 >= p.C) return;
    const float* src = p.share + e;
    const size_t slot_size = (size_t)256 * l.n;
    const int last = p.first[which + 1];
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int k = p.first[which]; k < last; k += kShares) {
        float4 w[kShares];
#pragma unroll
        for (int u = 0; u < kShares; ++u) w[u] = k + u < last ? *reinterpret_cast<const float4*>(src + p.slot[k + u] * slot_size) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int u = 0; u < kShares; ++u) { v.x += w[u].x; v.y += w[u].y; v.z += w[u].z; v.w += w[u].w; }
    }
    T* out = static_cast<T*>(!weight ? p.dx : row < 128 ? p.dwg : p.dwu) + (size_t)(weight ? 128 * mt + in_tile : 256 * mt + row) * p.C + c0;
    if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(out) = v;
    else *reinterpret_cast<uint2*>(out) = make_uint2(pack2<T>(v.x, v.y), pack2<T>(v.z, v.w));
}

// Tiles of at most 256 columns; at least six chunks a pair, so that shares stay few: backward of 512 x 320 x 1280 bf16 with 3, 6 and 12 26.3, 22.7 and 24.2 us,
// 1568 x 192 x 512 25.4, 21.5 and 22.1 (64 x 192 x 512 16.9, 19.3 and 20.3).
GatedLine plan_line(int M, int C, int F, int sm_count) {
    GatedLine l;
    l.dx = l.dw = 1;
    l.tiles_n = (C + 255) / 256;
    l.n = ((C + l.tiles_n - 1) / l.tiles_n + 31) / 32 * 32;
    l.tiles_x = (M + 255) / 256 * l.tiles_n;
    l.chunks_x = 2 * ((F + 63) / 64);
    l.tiles_w = (F + 127) / 128 * l.tiles_n;
    l.chunks_w = (M + 63) / 64;
    const long long most = (l.total() + 5) / 6;
    const int pairs = sm_count / 2 < kMostPairs ? sm_count / 2 : kMostPairs;
    l.pairs = (int)(most < pairs ? most : pairs);
    const long long all = l.total() / l.pairs / l.chunks_x * l.pairs;        // no more whole tiles a pair than it has chunks
    l.whole = (int)(all < l.tiles_x ? all : l.tiles_x);
    return l;
}

// At least as many chunks as a pair has of any tile
long long longest_sum(const GatedLine& l) {
    const long long own = l.whole ? l.chunks_x : 0, run = l.total() / l.pairs + 1 - (long long)(l.whole / l.pairs) * l.chunks_x;
    const long long tile = l.tiles_x > l.whole && l.chunks_x > l.chunks_w ? l.chunks_x : l.chunks_w, part = tile < run ? tile : run;
    return own > part ? own : part;
}

// G and U: 128 hidden units a tile of 256 rows for a pair of blocks; where that leaves half of the SMs without work, tiles of 128 rows and 64 units, or 32
// where those still do.  Forward, bf16 (us with 128, 64, 32 units): 512 x 192 x 512 5.8, 4.4, 3.9; 768 x 320 x 1280 6.5, 5.0, 6.0; 1536 x 320 x 1280 7.2, 7.0, 9.2;
// 512 x 1024 x 4096 10.7, 12.2, 18.8.  fp32: 256 x 320 x 1280 18.0, 14.5, 13.3; 768 18.9, 16.4, 21.5; 1024 19.8, 24.7, 29.5.
// `lone`: tiles of a pair are out (their epilogue writes one term of dG and dU).
struct GatedTiles { int bn, tiles_m, tiles_n, blocks; };
GatedTiles plan_tiles(int M, int F, bool lone, int sm_count) {
    GatedTiles t;
    t.bn = 128;
    t.tiles_m = (M + 255) / 256;
    t.tiles_n = (F + 127) / 128;
    const long long pairs = (long long)t.tiles_m * t.tiles_n;
    if (lone || 4 * pairs <= sm_count) {
        t.bn = (long long)((M + 127) / 128) * ((F + 63) / 64) * 2 <= sm_count ? 32 : 64;
        t.tiles_m = (M + 127) / 128;
        t.tiles_n = (F + t.bn - 1) / t.bn;
    }
    const long long units = (long long)t.tiles_m * t.tiles_n, most = t.bn == 128 ? sm_count / 2 : sm_count;
    t.blocks = (int)(units < most ? units : most) * (t.bn == 128 ? 2 : 1);
    return t;
}
int column_slots(const GatedTiles& t) {
    const int pairs = t.blocks / 2, runs = (pairs + t.tiles_n - 1) / t.tiles_n + 1;
    return 8 * (runs < t.tiles_m + 1 ? runs : t.tiles_m + 1);
}

// 16-bit elements: dG and dU as one term, rounded to the element type, which makes the error of dX and the weights' gradients 1.4 times that of their own
// rounding; over few rows it is more by chance (up to 2.1 times with one row, 1.6 with 32, 1.5 with 128), and there two terms keep it at 1.  (64 x 320 x 1280
// bf16 17.7 and 19.3 us, 128 x 1024 x 8192 46.6 and 50.5, 128 x 2048 x 11008 f16 107 and 116; 256 x 640 x 2560 25.6 and 30.4, which one term has.)
// A caller may ask for two over any number of rows, whose G and U then come in tiles of 64: 8192 x 320 x 1280 f16 59 and
// 132 us, 25088 x 192 x 512 bf16 53 and 132.
int gradient_terms(int M, bool two) { return two || M <= 128 ? 2 : 1; }
// Tiles of the projections of a call
GatedTiles call_tiles(int dtype, int M, int F, bool backward, bool two, int sm_count) { return plan_tiles(M, F, backward && dtype != kF32 && gradient_terms(M, two) > 1, sm_count); }

// Workspace: terms of X, Wg, Wu (fp32) | dG | dU | shares of tiles of dX and the weights' gradients, of the column sums | largest of dG and dU (f16)
struct GatedWs { size_t x, wg, wu, dg, du, share, db, largest, total; };
GatedWs gated_layout(int dtype, int M, int C, int F, bool backward, bool two, int sm_count) {
    GatedWs w;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at += (bytes + 255) / 256 * 256; return o; };
    const size_t terms = dtype == kF32 && (backward || !(few_forward(M) || small_forward(dtype, M, C, F))) ? 3 : 0;
    w.x = take(terms * M * C * 2);
    w.wg = take(terms * F * C * 2);
    w.wu = take(terms * F * C * 2);
    w.dg = w.du = w.share = w.db = w.largest = at;
    if (backward) {
        const GatedTiles t = call_tiles(dtype, M, F, true, two, sm_count);
        const size_t planes = (dtype == kF32 ? 3 : gradient_terms(M, two)) * (size_t)M * F * 2;
        w.dg = take(planes);
        w.du = take(planes);
        w.share = take((size_t)(sm_count / 2) * 2 * 256 * plan_line(M, C, F, sm_count).n * 4);
        const size_t slots = dtype != kF32 && t.bn == 128 ? column_slots(t) : (M + 31) / 32;
        w.db = take(slots * 2 * F * 4);
        w.largest = take(dtype == kF16 ? t.blocks * 4 : 0);
    }
    w.total = at;
    return w;
}

// Map of [z][rows][cols] elements of `unit` bytes (rows a multiple of 16 bytes) in boxes of 32 x 32; the swizzle spans a row of the box
bool make_box_map(CUtensorMap* out, const void* base, int unit, uint64_t zs, uint64_t rows, uint64_t cols) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t dims[3] = {cols, rows, zs};
    const cuuint64_t strides[2] = {unit * cols, rows * unit * cols};
    const cuuint32_t box[3] = {32, 32, 1};
    const cuuint32_t estr[3] = {1, 1, 1};
    return fn(out, unit == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16, 3, const_cast<void*>(base), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, unit == 4 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, GatedMode MODE, int BN, bool LONG> cudaError_t launch_kernel(const GatedArgs& a, int blocks, cudaStream_t st) {
    using S = GatedShape<T, MODE, BN>;
    static_assert(S::kSmem <= 232448, "shared memory");
    static std::atomic<unsigned long long> done{0};
    const cudaError_t e = allow_smem(gated_kernel<T, MODE, BN, LONG>, done, S::kSmem);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = S::kSmem;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = 2; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = S::kPair ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, gated_kernel<T, MODE, BN, LONG>, a);
}
// `longest`: chunks of the longest sum
template <typename T, GatedMode MODE, int BN> cudaError_t launch_mode(const GatedArgs& a, int blocks, long long longest, cudaStream_t st) {
    return longest > GatedTerms<T>::kMost ? launch_kernel<T, MODE, BN, true>(a, blocks, st) : launch_kernel<T, MODE, BN, false>(a, blocks, st);
}
template <typename T, GatedMode MODE> cudaError_t launch_projections(const GatedArgs& a, const GatedTiles& t, cudaStream_t st) {
    if (t.bn == 128) return launch_mode<T, MODE, 128>(a, t.blocks, a.chunks, st);
    return t.bn == 64 ? launch_mode<T, MODE, 64>(a, t.blocks, a.chunks, st) : launch_mode<T, MODE, 32>(a, t.blocks, a.chunks, st);
}

template <typename T> cudaError_t run_gated(const GatedCall& c, cudaStream_t st, int* launches) {
    constexpr int kTerms = GatedTerms<T>::kTerms;
    constexpr bool kWide = sizeof(T) == 4;
    constexpr int kType = kWide ? kF32 : Elem<T>::kIsBf16 ? kBF16 : kF16;
    const GatedWs w = gated_layout(kType, c.M, c.C, c.F, c.dh != nullptr, c.two_terms, c.sm_count);
    char* ws = static_cast<char*>(c.ws);
    const void *x = c.x, *wg = c.wg, *wu = c.wu;
    cudaError_t e;
    if (!c.dh && few_forward(c.M)) {
        ++*launches;
        auto few = [&](auto kern, int rows) {
            return launch_dependent(kern, dim3((c.F + 4 * kFewUnits - 1) / (4 * kFewUnits), (c.M + rows - 1) / rows), kFewThreads, 0, st, static_cast<const T*>(x), static_cast<const T*>(wg),
                                    static_cast<const T*>(wu), static_cast<const T*>(c.bg), static_cast<const T*>(c.bu), c.M, c.C, c.F, c.act, static_cast<T*>(c.h));
        };
        return c.M == 1 ? few(gated_few_kernel<T, 1>, 1) : c.M <= 4 ? few(gated_few_kernel<T, 4>, 4) : few(gated_few_kernel<T, 8>, 8);
    }
    if (!c.dh && small_forward(kType, c.M, c.C, c.F)) {
        static std::atomic<unsigned long long> done{0};
        if ((e = allow_smem(gated_small_kernel, done, kSmallSmem)) != cudaSuccess) return e;
        ++*launches;
        return launch_dependent(gated_small_kernel, dim3((c.F + kSmallTile - 1) / kSmallTile, (c.M + kSmallTile - 1) / kSmallTile), kSmallThreads, kSmallSmem, st, static_cast<const float*>(x),
                                static_cast<const float*>(wg), static_cast<const float*>(wu), static_cast<const float*>(c.bg), static_cast<const float*>(c.bu), c.M, c.C, c.F, c.act, static_cast<float*>(c.h));
    }
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
    const GatedTiles t = call_tiles(kType, c.M, c.F, c.dh != nullptr, c.two_terms, c.sm_count);
    a.tiles_m = t.tiles_m; a.tiles_n = t.tiles_n; a.chunks = (c.C + 63) / 64;
    a.out0 = c.dh ? ws + w.dg : static_cast<char*>(c.h);
    a.out1 = ws + w.du;
    a.terms = kWide ? kTerms : gradient_terms(c.M, c.two_terms);
    float* column = reinterpret_cast<float*>(ws + w.db);
    a.column = c.dbg ? column : nullptr;
    a.largest = reinterpret_cast<float*>(ws + w.largest);
    a.largest_parts = t.blocks;
    if (!make_map_3d_u16(&a.a[0], x, kTerms, c.M, c.C, 128) || !make_map_3d_u16(&a.b[0], wg, kTerms, c.F, c.C, t.bn) || !make_map_3d_u16(&a.b[1], wu, kTerms, c.F, c.C, t.bn)) return cudaErrorInvalidValue;
    if (!kWide && t.bn == 128) {
        if (!make_box_map(&a.s[0], a.out0, 2, 1, c.M, c.F)) return cudaErrorInvalidValue;
        if (c.dh && (!make_box_map(&a.s[1], a.out1, 2, 1, c.M, c.F) || !make_box_map(&a.g, c.dh, 2, 1, c.M, c.F))) return cudaErrorInvalidValue;
    }
    e = c.dh ? launch_projections<T, kGrad>(a, t, st) : launch_projections<T, kForward>(a, t, st);
    if (e != cudaSuccess) return e;
    ++*launches;
    if (!c.dh) return cudaSuccess;
    if (kType == kF16 && (c.dx || c.dwg)) {                // (biases sum numbers that are not rounded)
        a.again = 1;
        if ((e = launch_projections<T, kGrad>(a, t, st)) != cudaSuccess) return e;
        ++*launches;
    }

    const void *dg = ws + w.dg, *du = ws + w.du;
    FinishArgs f;
    memset(&f, 0, sizeof(f));
    f.dx = c.dx; f.dwg = c.dwg; f.dwu = c.dwu; f.dbg = c.dbg; f.dbu = c.dbu;
    f.M = c.M; f.C = c.C; f.F = c.F;
    f.column = column;
    if (c.dbg) {
        f.column_blocks = (2 * c.F + 31) / 32;
        f.tiles_m = 2 * t.tiles_m; f.units = 2 * t.tiles_m * t.tiles_n; f.count = t.blocks / 2;            // in halves
        if (kWide || t.bn < 128) f.runs = (c.M + 31) / 32;
    }
    a.line = plan_line(c.M, c.C, c.F, c.sm_count);
    a.line.dx = c.dx != nullptr;
    a.line.dw = c.dwg != nullptr;
    f.line = a.line;
    float* share = reinterpret_cast<float*>(ws + w.share);
    f.share = share;
    if (c.dx || c.dwg) {
        const GatedLine& l = a.line;
        const int unit = kWide ? 4 : 2;
        if (!make_map_3d_u16(&a.a[0], dg, a.terms, c.M, c.F, 128) || !make_map_3d_u16(&a.a[1], du, a.terms, c.M, c.F, 128) ||
            !make_map_3d_u16(&a.w[0], dg, a.terms, c.M, c.F, 64) || !make_map_3d_u16(&a.w[1], du, a.terms, c.M, c.F, 64) ||
            !make_map_3d_u16(&a.b[0], wg, kTerms, c.F, c.C, 64) || !make_map_3d_u16(&a.b[1], wu, kTerms, c.F, c.C, 64) || !make_map_3d_u16(&a.x, x, kTerms, c.M, c.C, 64) ||
            (c.dx && !make_box_map(&a.s[0], c.dx, unit, 1, c.M, c.C)) ||
            (c.dwg && (!make_box_map(&a.s[1], c.dwg, unit, 1, c.F, c.C) || !make_box_map(&a.s[2], c.dwu, unit, 1, c.F, c.C))) ||
            !make_box_map(&a.share, share, 4, 2 * l.pairs, 256, l.n)) return cudaErrorInvalidValue;
        if ((e = launch_mode<T, kProducts, 128>(a, 2 * l.pairs, longest_sum(l), st)) != cudaSuccess) return e;
        ++*launches;
        list_shares(&f);
    }
    const int blocks = f.column_blocks + f.tiles * (a.line.n / 4);
    if (!blocks) return cudaSuccess;                       // (no biases, every tile a pair's own)
    if ((e = launch_dependent(gated_finish_kernel<T>, dim3(blocks), 256, 0, st, f)) != cudaSuccess) return e;
    ++*launches;
    return cudaSuccess;
}

}  // namespace

size_t gated_bytes(int dtype, int M, int C, int F, bool backward, bool two_terms, int sm_count) { return gated_layout(dtype, M, C, F, backward, two_terms, sm_count).total; }

cudaError_t launch_gated(int dtype, const GatedCall& c, cudaStream_t st, int* launches) {
    switch (dtype) {
        case kF32: return run_gated<float>(c, st, launches);
        case kBF16: return run_gated<__nv_bfloat16>(c, st, launches);
        case kF16: return run_gated<__half>(c, st, launches);
        default: return cudaErrorInvalidValue;
    }
}

}  // namespace aa
