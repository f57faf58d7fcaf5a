// Queries and keys before the attention: an optional RMS norm of each head and rotary positions with up to three axes, in one pass; and its
// gradient.
//
// Forward, per token with position p and per head row x of d channels: y = gain x / sqrt(mean(x^2) + eps) (or y = x), then for every pair
// (u, v) of channels of axis a with angle t = p_a f:  (y_u cos t - y_v sin t, y_u sin t + y_v cos t).  Backward, with g the gradient of the
// result and R the rotation: g' = R^T g, xh = x r, r = 1 / sqrt(mean(x^2) + eps):  dx = r (g' gain - xh mean(g' gain xh)),
// dgain = sum of g' xh over batch, heads and tokens.
//
// A group of lanes owns a token: a lane has 16 bytes of channels and keeps their cosines and sines (with the gains folded in) for all
// heads, batch entries and both tensors that the block visits, so that an angle is computed once for many rows.  The angle is taken in
// turns: p f / (2 pi) with its rounding error by fma, less its nearest integer, so that large positions cost no accuracy; the partner of a
// channel comes from the lane itself (neighbouring channels as pairs), from another lane by a shuffle (halves of a segment, of whole
// 16-byte pieces) or through shared memory (halves of any other size).
#include "common.cuh"
#include "kernels.h"

namespace aa {

namespace {

constexpr int kRotThreads = 256, kRotWarps = kRotThreads / 32;
enum PairKind { kNeighbours, kHalvesShuffle, kHalvesShared };

// What a lane knows of its C channels: frequency in turns (two terms), axis and partner of each.
template <int C, bool NEIGHBOURS> struct LaneAngles {
    static constexpr int kAngles = NEIGHBOURS ? C / 2 : C;
    float hi[kAngles], lo[kAngles];
    unsigned axis;                        // two bits an angle
    unsigned rotated;                     // a bit a channel: it has a partner
    unsigned second;                      // a bit a channel: it is the second of its pair
    unsigned char partner[C];             // its partner's channel
};

template <int C, bool NEIGHBOURS> __device__ __forceinline__ void lane_angles(const RotateArgs& p, int c0, LaneAngles<C, NEIGHBOURS>& la) {
    la.axis = la.rotated = la.second = 0;
#pragma unroll
    for (int j = 0; j < C; ++j) {
        const int c = c0 + j;
        int at = 0, fr = 0, f = -1, axis = 0, partner = c;
        bool second = false;
#pragma unroll
        for (int a = 0; a < 3; ++a) {
            const int seg = p.channels[a], half = seg >> 1, o = c - at;
            if (o >= 0 && o < seg) {
                axis = a;
                if (NEIGHBOURS) { f = fr + (o >> 1); second = o & 1; partner = c ^ 1; }
                else { second = o >= half; f = fr + (second ? o - half : o); partner = second ? c - half : c + half; }
            }
            at += seg;
            fr += half;
        }
        la.partner[j] = (unsigned char)partner;
        if (f >= 0) la.rotated |= 1u << j;
        if (second) la.second |= 1u << j;
        if (!NEIGHBOURS || j % 2 == 0) {
            constexpr float kInv = 0.15915494309189535f, kInvLo = 6.420638243e-09f;     // 1 / (2 pi) as a sum of two fp32 numbers
            const int i = NEIGHBOURS ? j / 2 : j;
            const float w = f >= 0 ? __ldg(p.freq + f) : 0.f;
            la.hi[i] = w * kInv;
            la.lo[i] = fmaf(w, kInv, -la.hi[i]) + w * kInvLo;
            la.axis |= (unsigned)axis << (2 * i);
        }
    }
}

// cos and sin of position * frequency
__device__ __forceinline__ void turn(float pos, float hi, float lo, float& c, float& s) {
    const float t = pos * hi, e = fmaf(pos, lo, fmaf(pos, hi, -t));
    const float r = (t - rintf(t)) + e;
    sincospif(2.f * r, &s, &c);
}

// Position of a token in a batch entry
__device__ __forceinline__ void token_position(const RotateArgs& p, int b, int tok, float (&pos)[3]) {
    pos[0] = pos[1] = pos[2] = 0.f;
    if (p.positions) {
        const float* q = p.positions + (long long)b * p.pos_batch + (long long)tok * p.axes;
#pragma unroll
        for (int a = 0; a < 3; ++a)
            if (a < p.axes) pos[a] = __ldg(q + a);
    } else {
        int rest = tok;
#pragma unroll
        for (int a = 2; a >= 0; --a)
            if (a < p.axes) {
                const int n = p.extent[a], hi = rest / n;
                pos[a] = (float)(rest - hi * n);
                rest = hi;
            }
    }
}

// Factors of a channel's own value and of its partner's
template <int C, bool NEIGHBOURS> __device__ __forceinline__ void token_turns(const RotateArgs& p, const LaneAngles<C, NEIGHBOURS>& la, int b, int tok, bool inverse, float (&cs)[C], float (&sn)[C]) {
    float pos[3];
    token_position(p, b, tok, pos);
#pragma unroll
    for (int j = 0; j < C; ++j) {
        const int i = NEIGHBOURS ? j / 2 : j;
        if (NEIGHBOURS && j % 2) { cs[j] = cs[j - 1]; sn[j] = -sn[j - 1]; continue; }
        const unsigned a = la.axis >> (2 * i) & 3u;
        float c, s;
        turn(a == 0 ? pos[0] : a == 1 ? pos[1] : pos[2], la.hi[i], la.lo[i], c, s);
        cs[j] = c;
        sn[j] = ((la.second >> j & 1u) != 0) != inverse ? s : -s;
    }
}

// Values of the partners of this lane's channels
template <int C, PairKind KIND> __device__ __forceinline__ void partners(const float (&x)[C], const LaneAngles<C, KIND == kNeighbours>& la, int c0, int first_lane, float* patch, float (&y)[C]) {
    if constexpr (KIND == kNeighbours) {
#pragma unroll
        for (int j = 0; j < C; ++j) y[j] = x[j ^ 1];
    } else if constexpr (KIND == kHalvesShuffle) {
        const int src = first_lane + la.partner[0] / C;
#pragma unroll
        for (int j = 0; j < C; ++j) y[j] = __shfl_sync(0xffffffffu, x[j], src);
    } else {
        const int row = first_lane * C;
        __syncwarp();
#pragma unroll
        for (int j = 0; j < C; ++j) patch[row + c0 + j] = x[j];
        __syncwarp();
#pragma unroll
        for (int j = 0; j < C; ++j) y[j] = patch[row + la.partner[j]];
    }
}

template <typename T> __device__ __forceinline__ void load_vec(const T* src, bool live, float (&f)[Elem<T>::kVec]) {
    uint4 raw = make_uint4(0u, 0u, 0u, 0u);
    if (live) raw = *reinterpret_cast<const uint4*>(src);
    unpack16<T>(raw, f);
}

__device__ __forceinline__ float group_sum(float v, int lanes) {
    for (int o = lanes >> 1; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

template <typename T, PairKind KIND, bool NORM> __global__ void __launch_bounds__(kRotThreads) rotate_kernel(const __grid_constant__ RotateArgs p) {
    constexpr int C = Elem<T>::kVec;
    __shared__ float s_patch[KIND == kHalvesShared ? kRotWarps : 1][KIND == kHalvesShared ? 32 * C : 1];
    pdl_wait_prior();
    pdl_release_next();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gl = lane & (p.lanes - 1), c0 = gl * C, first_lane = lane - gl;
    const int tok = blockIdx.x * (kRotThreads / p.lanes) + threadIdx.x / p.lanes;
    const bool live = tok < p.N && c0 < p.d;
    const int unit = blockIdx.y / p.chunks, s0 = unit * p.unit_slabs + (blockIdx.y % p.chunks) * p.share, s1 = min(s0 + p.share, (unit + 1) * p.unit_slabs);
    LaneAngles<C, KIND == kNeighbours> la;
    lane_angles<C, KIND == kNeighbours>(p, c0, la);
    float cs[2][C], sn[2][C];
    token_turns<C, KIND == kNeighbours>(p, la, s0 / p.heads, min(tok, p.N - 1), p.inverse, cs[0], sn[0]);
#pragma unroll
    for (int j = 0; j < C; ++j) { cs[1][j] = cs[0][j]; sn[1][j] = sn[0][j]; }
    if (NORM) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (p.gain[i]) {
                const T* g = static_cast<const T*>(p.gain[i]);
#pragma unroll
                for (int j = 0; j < C; ++j)
                    if (c0 + j < p.d) { cs[i][j] *= Elem<T>::to_f32(g[c0 + j]); sn[i][j] *= Elem<T>::to_f32(g[la.partner[j]]); }
            }
    }
    float* patch = s_patch[KIND == kHalvesShared ? warp : 0];
    for (int s = s0; s < s1; ++s) {
        const long long in = tok_offset(p.lin, s, p.heads, tok) + c0, out = tok_offset(p.lout, s, p.heads, tok) + c0;
        float x[2][C];
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (p.x[i]) load_vec<T>(static_cast<const T*>(p.x[i]) + in, live, x[i]);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (!p.x[i]) continue;
            float r = 1.f;
            if (NORM) {
                float sq = 0.f;
#pragma unroll
                for (int j = 0; j < C; ++j) sq = fmaf(x[i][j], x[i][j], sq);
                r = rsqrtf(group_sum(sq, p.lanes) * p.inv_d + p.eps);
            }
            float y[C];
            partners<C, KIND>(x[i], la, c0, first_lane, patch, y);
#pragma unroll
            for (int j = 0; j < C; ++j) {
                const float own = x[i][j] * cs[i][j];
                y[j] = la.rotated >> j & 1u ? fmaf(y[j], sn[i][j], own) : own;
                if (NORM) y[j] *= r;
            }
            if (live) *reinterpret_cast<uint4*>(static_cast<T*>(p.y[i]) + out) = pack16<T>(y);
        }
    }
}

// Gradient through norm and rotation.  Blocks loop over (tile of tokens, run of slabs); gain gradients stay in registers until the block's end
// and leave as one row of partial sums a block, which gain_sum_kernel adds up in a fixed order.
template <typename T, PairKind KIND> __global__ void __launch_bounds__(kRotThreads) rotate_backward_kernel(const __grid_constant__ RotateBwdArgs p) {
    constexpr int C = Elem<T>::kVec;
    __shared__ float s_patch[KIND == kHalvesShared ? kRotWarps : 1][KIND == kHalvesShared ? 32 * C : 1];
    __shared__ float s_sum[kRotThreads * C];
    pdl_wait_prior();
    pdl_release_next();
    const RotateArgs& f = p.fwd;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gl = lane & (f.lanes - 1), c0 = gl * C, first_lane = lane - gl;
    const int groups = kRotThreads / f.lanes, tiles = (f.N + groups - 1) / groups;
    LaneAngles<C, KIND == kNeighbours> la;
    lane_angles<C, KIND == kNeighbours>(f, c0, la);
    float gain[2][C], sum[2][C];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < C; ++j) {
            gain[i][j] = f.gain[i] && c0 + j < f.d ? Elem<T>::to_f32(static_cast<const T*>(f.gain[i])[c0 + j]) : 1.f;
            sum[i][j] = 0.f;
        }
    float* patch = s_patch[KIND == kHalvesShared ? warp : 0];
    const int runs = f.chunks * (f.slabs / f.unit_slabs);
    for (long long item = blockIdx.x; item < (long long)tiles * runs; item += gridDim.x) {
        const int run = (int)(item / tiles), tok = (int)(item - (long long)run * tiles) * groups + threadIdx.x / f.lanes;
        const bool live = tok < f.N && c0 < f.d;
        const int unit = run / f.chunks, s0 = unit * f.unit_slabs + (run % f.chunks) * f.share, s1 = min(s0 + f.share, (unit + 1) * f.unit_slabs);
        float cs[C], sn[C];
        token_turns<C, KIND == kNeighbours>(f, la, s0 / f.heads, min(tok, f.N - 1), true, cs, sn);
        for (int s = s0; s < s1; ++s) {
            const long long at = tok_offset(f.lin, s, f.heads, tok) + c0, ga = tok_offset(p.lgrad, s, f.heads, tok) + c0, out = tok_offset(f.lout, s, f.heads, tok) + c0;
            float x[2][C], g[2][C];
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (f.x[i]) {
                    load_vec<T>(static_cast<const T*>(f.x[i]) + at, live, x[i]);
#pragma unroll
                    for (int j = 0; j < C; j += 4) {
                        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
                        if (live) v = *reinterpret_cast<const float4*>(p.grad[i] + ga + j);
                        g[i][j] = v.x; g[i][j + 1] = v.y; g[i][j + 2] = v.z; g[i][j + 3] = v.w;
                    }
                }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (!f.x[i]) continue;
                float y[C], sq = 0.f, dot = 0.f;
                partners<C, KIND>(g[i], la, c0, first_lane, patch, y);
#pragma unroll
                for (int j = 0; j < C; ++j) {
                    y[j] = la.rotated >> j & 1u ? fmaf(y[j], sn[j], g[i][j] * cs[j]) : g[i][j];
                    sq = fmaf(x[i][j], x[i][j], sq);
                    dot = fmaf(y[j] * gain[i][j], x[i][j], dot);
                }
                const float r = rsqrtf(group_sum(sq, f.lanes) * f.inv_d + f.eps);
                const float m = group_sum(dot, f.lanes) * f.inv_d * r * r * r;
#pragma unroll
                for (int j = 0; j < C; ++j) {
                    sum[i][j] = fmaf(y[j], x[i][j] * r, sum[i][j]);
                    y[j] = fmaf(r * gain[i][j], y[j], -m * x[i][j]);
                }
                if (live) {
#pragma unroll
                    for (int j = 0; j < C; j += 4) *reinterpret_cast<float4*>(static_cast<float*>(f.y[i]) + out + j) = make_float4(y[j], y[j + 1], y[j + 2], y[j + 3]);
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < C; ++j) s_sum[threadIdx.x * C + j] = sum[i][j];
        __syncthreads();
        const int width = f.lanes * C;
        for (int c = threadIdx.x; c < f.d; c += kRotThreads) {
            float v = 0.f;
            for (int k = 0; k < groups; ++k) v += s_sum[k * width + c];
            p.part[((long long)blockIdx.x * 2 + i) * f.d + c] = v;
        }
    }
}

// Sum of the blocks' rows: a warp per eight columns of the 2 d, four rows at a time
__global__ void __launch_bounds__(kRotThreads) gain_sum_kernel(const float* part, int rows, int d, float* dq, float* dk) {
    pdl_wait_prior();
    pdl_release_next();
    const int lane = threadIdx.x & 31, c = (blockIdx.x * kRotWarps + (threadIdx.x >> 5)) * 8 + (lane & 7);
    float v = 0.f;
    if (c < 2 * d)
        for (int r = lane >> 3; r < rows; r += 4) v += part[(long long)r * 2 * d + c];
    v += __shfl_xor_sync(0xffffffffu, v, 8);
    v += __shfl_xor_sync(0xffffffffu, v, 16);
    if (lane < 8 && c < 2 * d) {
        if (c < d) { if (dq) dq[c] = v; }
        else if (dk) dk[c - d] = v;
    }
}

PairKind pair_kind(const RotateArgs& a, int c) {
    if (a.neighbours) return kNeighbours;
    int at = 0;
    bool whole = true;
    for (int s : a.channels) {
        if (s % (2 * c) || at % c) whole = whole && s == 0;
        at += s;
    }
    return whole && at % c == 0 ? kHalvesShuffle : kHalvesShared;
}

// Lanes of a token, and how many slabs a block visits with one set of angles: as many as leave about two waves of blocks.
void plan_rotate(RotateArgs* a, int vec, int sm_count, int* tiles) {
    a->lanes = 1;
    while (a->lanes * vec < a->d) a->lanes *= 2;
    const int groups = kRotThreads / a->lanes;
    *tiles = (a->N + groups - 1) / groups;
    a->unit_slabs = a->positions && a->pos_batch ? a->heads : a->slabs;
    const long long rows = (long long)*tiles * a->slabs;
    long long share = rows / (16ll * sm_count);
    if (share < 1) share = 1;
    if (share > a->unit_slabs) share = a->unit_slabs;
    a->share = (int)share;
    a->chunks = (a->unit_slabs + a->share - 1) / a->share;
    a->inv_d = 1.f / (float)a->d;
}

template <typename T, PairKind KIND> cudaError_t launch_rotate_kind(const RotateArgs& a, dim3 grid, cudaStream_t st) {
    if (a.norm) return launch_dependent(rotate_kernel<T, KIND, true>, grid, kRotThreads, 0, st, a);
    return launch_dependent(rotate_kernel<T, KIND, false>, grid, kRotThreads, 0, st, a);
}
template <typename T> cudaError_t launch_rotate_type(RotateArgs a, int sm_count, cudaStream_t st) {
    int tiles;
    plan_rotate(&a, Elem<T>::kVec, sm_count, &tiles);
    const dim3 grid(tiles, a.chunks * (a.slabs / a.unit_slabs));
    switch (pair_kind(a, Elem<T>::kVec)) {
        case kNeighbours: return launch_rotate_kind<T, kNeighbours>(a, grid, st);
        case kHalvesShuffle: return launch_rotate_kind<T, kHalvesShuffle>(a, grid, st);
        default: return launch_rotate_kind<T, kHalvesShared>(a, grid, st);
    }
}
int backward_blocks(int sm_count) { return 4 * sm_count; }
template <typename T> cudaError_t launch_rotate_bwd_type(RotateBwdArgs a, int sm_count, cudaStream_t st) {
    int tiles;
    plan_rotate(&a.fwd, Elem<T>::kVec, sm_count, &tiles);
    const long long items = (long long)tiles * a.fwd.chunks * (a.fwd.slabs / a.fwd.unit_slabs);
    const int blocks = (int)(items < backward_blocks(sm_count) ? items : backward_blocks(sm_count));
    cudaError_t e;
    switch (pair_kind(a.fwd, Elem<T>::kVec)) {
        case kNeighbours: e = launch_dependent(rotate_backward_kernel<T, kNeighbours>, dim3(blocks), kRotThreads, 0, st, a); break;
        case kHalvesShuffle: e = launch_dependent(rotate_backward_kernel<T, kHalvesShuffle>, dim3(blocks), kRotThreads, 0, st, a); break;
        default: e = launch_dependent(rotate_backward_kernel<T, kHalvesShared>, dim3(blocks), kRotThreads, 0, st, a); break;
    }
    if (e != cudaSuccess || (!a.dgain[0] && !a.dgain[1])) return e;
    return launch_dependent(gain_sum_kernel, dim3((2 * a.fwd.d + 8 * kRotWarps - 1) / (8 * kRotWarps)), kRotThreads, 0, st, a.part, blocks, a.fwd.d, a.dgain[0], a.dgain[1]);
}

}  // namespace

size_t rotate_backward_bytes(int d, int sm_count) { return (size_t)backward_blocks(sm_count) * 2 * d * sizeof(float); }

cudaError_t launch_rotate(int dtype, const RotateArgs& a, int sm_count, cudaStream_t st) {
    switch (dtype) {
        case kF32: return launch_rotate_type<float>(a, sm_count, st);
        case kBF16: return launch_rotate_type<__nv_bfloat16>(a, sm_count, st);
        case kF16: return launch_rotate_type<__half>(a, sm_count, st);
        default: return cudaErrorInvalidValue;
    }
}

cudaError_t launch_rotate_backward(int dtype, const RotateBwdArgs& a, int sm_count, cudaStream_t st) {
    switch (dtype) {
        case kF32: return launch_rotate_bwd_type<float>(a, sm_count, st);
        case kBF16: return launch_rotate_bwd_type<__nv_bfloat16>(a, sm_count, st);
        case kF16: return launch_rotate_bwd_type<__half>(a, sm_count, st);
        default: return cudaErrorInvalidValue;
    }
}

}  // namespace aa
