// Layer norm over the channels of a row, and its gradient.
//
//     y = (x - m) r w + b,  m = mean(x),  r = 1 / sqrt(mean((x - m)^2) + eps)
//     xh = (x - m) r,  g = dy w:   dx = r (g - mean(g) - xh mean(g xh)),  dw = sum over rows of dy xh,  db = sum over rows of dy
//
// Bound by HBM: every row is read once (x; x and dy) and stays in registers for its sums, which are fp32 and taken about the mean.  TPR threads share a
// row, so that a thread holds at most four vectors of 16 bytes: 4 to 32 lanes of a warp, which meet by shuffles, or a block of 128 or 512 threads.
// Blocks walk rows with the gains in registers; the gains' gradients are summed there too, leave as one row of sums a block and are added in a
// fixed order by a second launch.  Rows that are no whole vectors (channel counts, or addresses) go element by element, up to 8192 of them; rows that no
// such share holds (more than that, or more than 16384 channels in whole vectors, 8192 in fp32) are read from memory, in practice from L2, for each of their sums.
// 131072 x 512 bf16 48 us (5.6 TB/s), gradient of 200704 x 64 with its join 21.5.
#include "common.cuh"
#include "kernels.h"

#include <algorithm>
#include <climits>

namespace aa {

namespace {

// V elements of a row as they are in memory, and as fp32
template <typename T, int V> struct Raw { using R = uint4; };
template <typename T> struct Raw<T, 1> { using R = T; };
template <typename T, int V> using RawT = typename Raw<T, V>::R;
template <typename T, int V> __device__ __forceinline__ RawT<T, V> read_raw(const T* p) { return __ldg(reinterpret_cast<const RawT<T, V>*>(p)); }
template <typename T, int V> __device__ __forceinline__ void unpack_raw(const RawT<T, V>& r, float* f) {
    if constexpr (V == 1) f[0] = Elem<T>::to_f32(r);
    else unpack16<T>(r, f);
}
template <typename T, int V> __device__ __forceinline__ void write_vec(T* p, const float* f) {
    if constexpr (V == 1) *p = Elem<T>::from_f32(f[0]);
    else *reinterpret_cast<uint4*>(p) = pack16<T>(f);
}

// Sums over the TPR threads of a row; `part`: two rounds of shared memory for rows of several warps, taken in turns
template <int TPR, int N> __device__ __forceinline__ void row_sums(float (&s)[N], float* part, int& turn) {
#pragma unroll
    for (int o = (TPR < 32 ? TPR : 32) / 2; o; o >>= 1)
#pragma unroll
        for (int n = 0; n < N; ++n) s[n] += __shfl_xor_sync(0xffffffffu, s[n], o);
    if constexpr (TPR > 32) {
        constexpr int W = TPR / 32;
        float* p = part + turn * 2 * W;
        turn ^= 1;
        if ((threadIdx.x & 31) == 0)
#pragma unroll
            for (int n = 0; n < N; ++n) p[n * W + (threadIdx.x >> 5)] = s[n];
        __syncthreads();
#pragma unroll
        for (int n = 0; n < N; ++n) {
            s[n] = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) s[n] += p[n * W + w];
        }
    }
}

// Rows that a thread adds up before the sum joins others: equal numbers on a growing sum are rounded the same way each time, up to 2^-25 of it (2^21 rows of 2048 channels in
// 592 blocks: 5e-5).
constexpr int kMostRows = 256;

// How a block's threads share rows
template <int TPR> constexpr int kBlock = TPR > 32 ? TPR : 256;

// Blocks of an SM: what registers leave (a thread holds F values of a row, backward four times that, and the next row as it is in memory)
template <int TPR, int F, bool BACK> constexpr int kPerSm = TPR == 512 ? (F <= 8 ? 2 : 1) : (F <= 8 ? (BACK ? 4 : 6) : F <= 16 ? (BACK ? 2 : 4) : BACK ? 1 : 2) * (TPR == 128 ? 2 : 1);
// FULL: the threads' vectors are just the row's
template <typename T, int TPR, int NV, int V, bool BACK, bool FULL>
__global__ void __launch_bounds__(kBlock<TPR>, kPerSm<TPR, NV * V, BACK>) norm_kernel(const __grid_constant__ NormArgs a) {
    constexpr int THREADS = kBlock<TPR>, RPB = THREADS / TPR, F = NV * V, P = F / 2;
    extern __shared__ float sums[];                        // backward: [warps][C]
    __shared__ float part[TPR > 32 ? 4 * (TPR / 32) : 1];
    const int tid = threadIdx.x, lane = tid % TPR, C = a.C;
    const float inv = 1.f / (float)C;
    int turn = 0;
    float2 dw[BACK ? P : 1], db[BACK ? P : 1], w[P], b[BACK ? 1 : P];      // pairs of neighbouring values: half the instructions, which bound these kernels
    RawT<T, V> x[NV], dy[BACK ? NV : 1];
    auto in = [&](int v) { return FULL || (v * TPR + lane) * V < C; };
    auto fetch = [&](bool some, long long at) {            // (this lane's first element of the row)
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            x[v] = RawT<T, V>{};                           // (what is none counts as zero)
            if constexpr (BACK) dy[v] = RawT<T, V>{};
            if (some && in(v)) {
                x[v] = read_raw<T, V>(static_cast<const T*>(a.x) + at + v * TPR * V);
                if constexpr (BACK) dy[v] = read_raw<T, V>(static_cast<const T*>(a.dy) + at + v * TPR * V);
            }
        }
    };
    auto unpack = [&](const RawT<T, V>* raw, float2* f) {
        float t[F];
#pragma unroll
        for (int v = 0; v < NV; ++v) unpack_raw<T, V>(raw[v], t + v * V);
#pragma unroll
        for (int i = 0; i < P; ++i) f[i] = make_float2(t[2 * i], t[2 * i + 1]);
    };
    auto both = [](float v) { return make_float2(v, v); };
    if (BACK) pdl_release_next();
    const unsigned rows = (unsigned)a.rows, stride = gridDim.x * RPB, own = tid / TPR;
    const long long step = (long long)stride * C;
    long long at = (long long)(blockIdx.x * RPB + own) * C + lane * V;
    fetch(blockIdx.x * RPB + own < rows, at);
#pragma unroll
    for (int i = 0; i < P; ++i) {
        w[i] = both(1.f);
        if (!BACK) b[i] = both(0.f);
        if (BACK) dw[i] = db[i] = both(0.f);
    }
    {
        RawT<T, V> t[NV];
        if (a.w) {
#pragma unroll
            for (int v = 0; v < NV; ++v) t[v] = in(v) ? read_raw<T, V>(static_cast<const T*>(a.w) + (v * TPR + lane) * V) : RawT<T, V>{};
            unpack(t, w);
        }
        if constexpr (!BACK)
            if (a.b) {
#pragma unroll
                for (int v = 0; v < NV; ++v) t[v] = in(v) ? read_raw<T, V>(static_cast<const T*>(a.b) + (v * TPR + lane) * V) : RawT<T, V>{};
                unpack(t, b);
            }
    }
    // (every thread of a block takes the same number of turns: shuffles and barriers are met by all)
    for (unsigned r0 = blockIdx.x * RPB; r0 < rows; r0 += stride, at += step) {
        const bool live = r0 + own < rows;
        float2 f[P], g[BACK ? P : 1];
        unpack(x, f);
        if constexpr (BACK) unpack(dy, g);
        fetch(r0 + own + stride < rows, at + step);
        float2 q = f[0];
#pragma unroll
        for (int i = 1; i < P; ++i) q = fadd2(q, f[i]);
        float s[1] = {q.x + q.y};
        row_sums<TPR, 1>(s, part, turn);
        const float mean = s[0] * inv;
        q = both(0.f);
#pragma unroll
        for (int i = 0; i < P; ++i) {
            f[i] = fadd2(f[i], both(-mean));
            if (!FULL) {
                if (!in(2 * i / V)) f[i].x = 0.f;
                if (!in((2 * i + 1) / V)) f[i].y = 0.f;
            }
            q = ffma2(f[i], f[i], q);
        }
        s[0] = q.x + q.y;
        row_sums<TPR, 1>(s, part, turn);
        const float root = rsqrtf(s[0] * inv + a.eps), rs = live ? root : 0.f;      // (of a row that is none it may be infinite)
        if constexpr (!BACK) {
#pragma unroll
            for (int i = 0; i < P; ++i) f[i] = ffma2(fmul2(f[i], both(rs)), w[i], b[i]);
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                float y[V];
#pragma unroll
                for (int e = 0; e < V; ++e) y[e] = (v * V + e) & 1 ? f[(v * V + e) / 2].y : f[(v * V + e) / 2].x;
                if (live && in(v)) write_vec<T, V>(static_cast<T*>(a.y) + at + v * TPR * V, y);
            }
        } else {
            float2 t0 = both(0.f), t1 = t0;
#pragma unroll
            for (int i = 0; i < P; ++i) {
                f[i] = fmul2(f[i], both(rs));
                dw[i] = ffma2(g[i], f[i], dw[i]);
                db[i] = fadd2(db[i], g[i]);
                g[i] = fmul2(g[i], w[i]);
                t0 = fadd2(t0, g[i]);
                t1 = ffma2(g[i], f[i], t1);
            }
            if (a.dx) {
                float t[2] = {t0.x + t0.y, t1.x + t1.y};
                row_sums<TPR, 2>(t, part, turn);
                const float2 m0 = both(-t[0] * inv), m1 = both(-t[1] * inv);
#pragma unroll
                for (int i = 0; i < P; ++i) g[i] = fmul2(fadd2(ffma2(f[i], m1, g[i]), m0), both(rs));
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    float y[V];
#pragma unroll
                    for (int e = 0; e < V; ++e) y[e] = (v * V + e) & 1 ? g[(v * V + e) / 2].y : g[(v * V + e) / 2].x;
                    if (live && in(v)) write_vec<T, V>(static_cast<T*>(a.dx) + at + v * TPR * V, y);
                }
            }
        }
    }
    if constexpr (BACK) {
        if (!a.ws) return;
        // one row of sums a block
        if constexpr (TPR < 32) {
#pragma unroll
            for (int o = TPR; o < 32; o <<= 1)
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    dw[i] = fadd2(dw[i], make_float2(__shfl_xor_sync(0xffffffffu, dw[i].x, o), __shfl_xor_sync(0xffffffffu, dw[i].y, o)));
                    db[i] = fadd2(db[i], make_float2(__shfl_xor_sync(0xffffffffu, db[i].x, o), __shfl_xor_sync(0xffffffffu, db[i].y, o)));
                }
        }
        float* out = a.ws + (long long)blockIdx.x * 2 * C;
        constexpr int WARPS = TPR > 32 ? 1 : THREADS / 32;         // whose sums of the same columns meet in shared memory, in order
        const bool first = TPR >= 32 || (tid & 31) < TPR;
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            if (WARPS > 1 && side) __syncthreads();
#pragma unroll
            for (int i = 0; i < F; ++i) {
                const int c = (i / V * TPR + lane) * V + i % V;
                const float2 t = side ? db[i / 2] : dw[i / 2];
                if (first && in(i / V)) (WARPS > 1 ? sums + (tid >> 5) * C : out + side * C)[c] = i & 1 ? t.y : t.x;
            }
            if (WARPS > 1) {
                __syncthreads();
                for (int c = tid; c < C; c += THREADS) {
                    float t = sums[c];
#pragma unroll
                    for (int k = 1; k < WARPS; ++k) t += sums[k * C + c];
                    out[side * C + c] = t;
                }
            }
        }
    }
}

// Rows of any length, a block each, read again for each sum.  Backward: dx, and (mean, r) of every row for the gains' gradients.
template <typename T, bool BACK> __global__ void __launch_bounds__(512) norm_wide_kernel(const __grid_constant__ NormArgs a, float2* stats) {
    __shared__ float part[4 * 16];
    int turn = 0;
    const int C = a.C;
    const float inv = 1.f / (float)C;
    for (long long r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + r * C;
        float s[1] = {0.f};
        for (int c = threadIdx.x; c < C; c += 512) s[0] += Elem<T>::to_f32(x[c]);
        row_sums<512, 1>(s, part, turn);
        const float mean = s[0] * inv;
        s[0] = 0.f;
        for (int c = threadIdx.x; c < C; c += 512) {
            const float z = Elem<T>::to_f32(x[c]) - mean;
            s[0] = fmaf(z, z, s[0]);
        }
        row_sums<512, 1>(s, part, turn);
        const float rs = 1.f / sqrtf(s[0] * inv + a.eps);
        auto gain = [&](int c) { return a.w ? Elem<T>::to_f32(static_cast<const T*>(a.w)[c]) : 1.f; };
        if constexpr (!BACK) {
            for (int c = threadIdx.x; c < C; c += 512)
                static_cast<T*>(a.y)[r * C + c] = Elem<T>::from_f32(fmaf((Elem<T>::to_f32(x[c]) - mean) * rs, gain(c), a.b ? Elem<T>::to_f32(static_cast<const T*>(a.b)[c]) : 0.f));
        } else {
            if (stats && threadIdx.x == 0) stats[r] = make_float2(mean, rs);
            if (!a.dx) continue;
            const T* dy = static_cast<const T*>(a.dy) + r * C;
            float t[2] = {0.f, 0.f};
            for (int c = threadIdx.x; c < C; c += 512) {
                const float g = Elem<T>::to_f32(dy[c]) * gain(c);
                t[0] += g;
                t[1] = fmaf(g, (Elem<T>::to_f32(x[c]) - mean) * rs, t[1]);
            }
            row_sums<512, 2>(t, part, turn);
            for (int c = threadIdx.x; c < C; c += 512)
                static_cast<T*>(a.dx)[r * C + c] = Elem<T>::from_f32(rs * (Elem<T>::to_f32(dy[c]) * gain(c) - t[0] * inv - (Elem<T>::to_f32(x[c]) - mean) * rs * t[1] * inv));
        }
    }
}
// Sums of a run of rows for 256 columns
template <typename T> __global__ void __launch_bounds__(256) norm_columns_kernel(const __grid_constant__ NormArgs a, const float2* stats, float* out) {
    const int c = blockIdx.x * 256 + threadIdx.x, C = a.C;
    const long long first = a.rows * blockIdx.y / gridDim.y, last = a.rows * (blockIdx.y + 1) / gridDim.y;
    if (c >= C) return;
    float p = 0.f, q = 0.f;
    for (long long r0 = first; r0 < last; r0 += kMostRows) {
        float u = 0.f, v = 0.f;
        for (long long r = r0; r < min(last, r0 + kMostRows); ++r) {
            const float2 s = __ldg(stats + r);
            const float g = Elem<T>::to_f32(static_cast<const T*>(a.dy)[r * C + c]);
            u = fmaf(g, (Elem<T>::to_f32(static_cast<const T*>(a.x)[r * C + c]) - s.x) * s.y, u);
            v += g;
        }
        p += u;
        q += v;
    }
    out[(long long)blockIdx.y * 2 * C + c] = p;
    out[(long long)blockIdx.y * 2 * C + C + c] = q;
}
// Rows of sums [shares][2][C] -> dw, db: 32 columns a block, every warp a run of shares, joined in order
__global__ void __launch_bounds__(1024) norm_join_kernel(const float* in, int shares, int C, float* dw, float* db) {
    __shared__ float part[32][33];
    pdl_wait_prior();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c = blockIdx.x * 32 + lane;
    float s = 0.f;
    const int first = (int)((long long)shares * warp / 32), last = (int)((long long)shares * (warp + 1) / 32);
    if (c < 2 * C) {
        const int most = min(last, first + kMostRows);
#pragma unroll 16
        for (int k = first; k < most; ++k) s += in[(long long)k * 2 * C + c];
        for (int k0 = most; k0 < last; k0 += kMostRows) {
            float t = 0.f;
            for (int k = k0; k < min(last, k0 + kMostRows); ++k) t += in[(long long)k * 2 * C + c];
            s += t;
        }
    }
    part[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && c < 2 * C) {
        s = 0.f;
#pragma unroll
        for (int k = 0; k < 32; ++k) s += part[k][lane];
        float* out = c < C ? dw : db;
        if (out) out[c < C ? c : c - C] = s;
    }
}

constexpr int kColumnShares = 64;

bool aligned16(const NormArgs& a) {
    const void* const p[] = {a.x, a.w, a.b, a.y, a.dy, a.dx};
    uintptr_t bits = 0;
    for (const void* q : p) bits |= reinterpret_cast<uintptr_t>(q);
    return bits % 16 == 0;
}
// How rows of C channels are shared: threads a row, vectors a thread, elements a vector; 0: norm_wide_kernel
struct NormPlan {
    int tpr, nv, v;
};
NormPlan plan_of(int dtype, int C, bool aligned, bool back) {
    const int vec = dtype == 0 ? 4 : 8;
    NormPlan p{0, 0, 0};
    if (C % vec == 0 && aligned) {
        const int n = C / vec;
        p.v = vec;
        // up to a warp a row: the fewest idle lanes, then the fewest vectors a lane; backward, where a thread holds four times as much, three vectors only for a third less
        // (8192 x 320 f16: three vectors in 16 lanes 19.7 us, two in 32 8.6 us)
        int least = INT_MAX;
        for (int v = 1; v <= 4; ++v)
            for (int t : {4, 8, 16, 32})
                if (const int cost = t * v * (back && v > 2 ? 3 : 2); n <= t * v && cost < least && (v < 4 || t == 32)) {
                    least = cost;
                    p.tpr = t;
                    p.nv = v;
                }
        if (p.tpr) return p;
        for (int t : {128, 512})
            if (n <= 4 * t) { p.tpr = t; p.nv = (n + t - 1) / t; return p; }
    } else {
        p.v = 1;
        for (int t : {8, 32, 128, 512})
            if (C <= 16 * t) { p.tpr = t; p.nv = C <= 4 * t ? 4 : 16; return p; }
    }
    p.tpr = 0;
    return p;
}
// Blocks that walk the rows: as many as run at once; where the gains' gradients are sums of too many rows (kMostRows), a multiple of that
long long blocks_of(const NormPlan& p, long long rows, int sm_count, bool back) {
    const int rpb = p.tpr > 32 ? 1 : 256 / p.tpr, f = p.nv * p.v;
    const int per = p.tpr == 512 ? (f <= 8 ? 2 : 1) : (f <= 8 ? (back ? 4 : 6) : f <= 16 ? (back ? 2 : 4) : back ? 1 : 2) * (p.tpr == 128 ? 2 : 1);       // kPerSm
    const long long turns = (rows + rpb - 1) / rpb, wave = (long long)sm_count * per;
    return turns <= wave ? turns : back ? wave * ((turns + wave * kMostRows - 1) / (wave * kMostRows)) : wave;
}

template <typename T, int TPR, int NV, int V, bool BACK> cudaError_t run_norm(const NormArgs& a, const NormPlan& p, int sm_count, cudaStream_t st) {
    const int smem = BACK && a.ws && TPR <= 32 ? kBlock<TPR> / 32 * a.C * 4 : 0;       // (32 KB at most: 1024 channels)
    const unsigned blocks = (unsigned)blocks_of(p, a.rows, sm_count, BACK);
    if (V > 1 && a.C == TPR * NV * V) norm_kernel<T, TPR, NV, V, BACK, true><<<blocks, kBlock<TPR>, smem, st>>>(a);
    else norm_kernel<T, TPR, NV, V, BACK, false><<<blocks, kBlock<TPR>, smem, st>>>(a);
    return cudaGetLastError();
}
template <typename T, bool BACK> cudaError_t norm_of(const NormArgs& a, int sm_count, cudaStream_t st) {
    constexpr int V = Elem<T>::kVec;
    const NormPlan p = plan_of(sizeof(T) == 4 ? 0 : 1, a.C, aligned16(a), BACK);
#define AA_NORM(TPR, NV, VEC) if (p.tpr == TPR && p.nv == NV && p.v == VEC) return run_norm<T, TPR, NV, VEC, BACK>(a, p, sm_count, st);
    AA_NORM(4, 1, V) AA_NORM(4, 2, V) AA_NORM(4, 3, V)
    AA_NORM(8, 1, V) AA_NORM(8, 2, V) AA_NORM(8, 3, V)
    AA_NORM(16, 1, V) AA_NORM(16, 2, V) AA_NORM(16, 3, V)
    AA_NORM(32, 1, V) AA_NORM(32, 2, V) AA_NORM(32, 3, V) AA_NORM(32, 4, V)
    AA_NORM(128, 1, V) AA_NORM(128, 2, V) AA_NORM(128, 3, V) AA_NORM(128, 4, V)
    AA_NORM(512, 1, V) AA_NORM(512, 2, V) AA_NORM(512, 3, V) AA_NORM(512, 4, V)
    AA_NORM(8, 4, 1) AA_NORM(8, 16, 1) AA_NORM(32, 4, 1) AA_NORM(32, 16, 1)
    AA_NORM(128, 4, 1) AA_NORM(128, 16, 1) AA_NORM(512, 4, 1) AA_NORM(512, 16, 1)
#undef AA_NORM
    const unsigned blocks = (unsigned)std::min<long long>(a.rows, (long long)sm_count * 4);
    float2* stats = BACK && a.ws ? reinterpret_cast<float2*>(a.ws + (long long)kColumnShares * 2 * a.C) : nullptr;
    const bool place = BACK && stats && a.dx == a.dy;      // dx takes the place of dy: after the gains' gradients have read it
    NormArgs first = a;
    if (place) first.dx = nullptr;
    norm_wide_kernel<T, BACK><<<blocks, 512, 0, st>>>(first, stats);
    if (cudaError_t e = cudaGetLastError()) return e;
    if (stats) norm_columns_kernel<T><<<dim3((a.C + 255) / 256, kColumnShares), 256, 0, st>>>(a, stats, a.ws);
    if (cudaError_t e = cudaGetLastError()) return e;
    if (place) norm_wide_kernel<T, BACK><<<blocks, 512, 0, st>>>(a, nullptr);
    return cudaGetLastError();
}

}  // namespace

size_t norm_backward_bytes(int dtype, long long rows, int C, int sm_count) {
    size_t most = 0;                               // (the size does not depend on the pointers)
    for (bool aligned : {false, true}) {
        const NormPlan p = plan_of(dtype, C, aligned, true);
        const size_t shares = p.tpr ? (size_t)blocks_of(p, rows, sm_count, true) : (size_t)kColumnShares;
        most = std::max(most, shares * 2 * C * sizeof(float) + (p.tpr ? 0 : (size_t)rows * sizeof(float2)));
    }
    return most;
}
cudaError_t launch_norm(int dtype, const NormArgs& a, int sm_count, cudaStream_t st) {
    return dtype == 0 ? norm_of<float, false>(a, sm_count, st) : dtype == 1 ? norm_of<__nv_bfloat16, false>(a, sm_count, st) : norm_of<__half, false>(a, sm_count, st);
}
cudaError_t launch_norm_backward(int dtype, const NormArgs& a, int sm_count, cudaStream_t st, int* launches) {
    NormArgs b = a;
    if (!a.dw && !a.db) b.ws = nullptr;
    const cudaError_t e = dtype == 0 ? norm_of<float, true>(b, sm_count, st) : dtype == 1 ? norm_of<__nv_bfloat16, true>(b, sm_count, st) : norm_of<__half, true>(b, sm_count, st);
    const NormPlan p = plan_of(dtype, a.C, aligned16(a), true);
    *launches = (p.tpr || !b.ws ? 1 : a.dx == a.dy ? 3 : 2) + (b.ws ? 1 : 0);
    if (e != cudaSuccess || !b.ws) return e;
    const int shares = p.tpr ? (int)blocks_of(p, a.rows, sm_count, true) : kColumnShares;
    return launch_dependent(norm_join_kernel, dim3((2 * a.C + 31) / 32), 1024, 0, st, b.ws, shares, a.C, a.dw, a.db);
}

}  // namespace aa
