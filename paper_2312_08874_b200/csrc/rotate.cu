// Queries and keys before the attention: an optional RMS norm of each head and rotary positions with up to three axes, in one pass; and its
// gradient.
//
// Forward, per token with position p and per head row x of d channels: y = gain x / sqrt(mean(x^2) + eps) (or y = x), then for every pair
// (u, v) of channels of axis a with angle t = p_a f:  (y_u cos t - y_v sin t, y_u sin t + y_v cos t).  Backward, with g the gradient of the
// result and R the rotation: g' = R^T g, xh = x r, r = 1 / sqrt(mean(x^2) + eps):  dx = r (g' gain - xh mean(g' gain xh)),
// dgain = sum of g' xh over batch, heads and tokens.
//
// A group of lanes owns a token and keeps the cosines and sines of its channels (forward: with the gains folded in) for all heads and batch entries
// that the block visits, so that an angle is computed once for many rows.  The angle is taken in turns: p f / (2 pi) with its rounding error by fma,
// less its nearest integer, so that large positions cost no accuracy.  Where the channels of a pair lie, in the order of preference:
//   forward, rotate_pairs_kernel: a lane has two pieces of 16 bytes that hold whole pairs: a piece of a segment's first half and the one half a segment
//     on, or two pieces with neighbouring channels as pairs.  Nothing crosses lanes but the norm's sum.
//   forward, rotate_patch_kernel: halves that are no whole pieces, and 16 bits without a norm: a lane has one piece, its partners come through shared
//     memory.  Whole pieces both ways (us, pairs and patch): bf16 with a norm 64 slabs of 56 x 56 18.8 and 32.0, 16 of 128 x 128 25.6 and 39.3; without
//     a norm 19.6 and 18.0, 25.4 and 23.7 (four blocks an SM instead of three); fp32 8 slabs of 128 x 128 x 32 channels 15.2 and 19.6, 10.9 and 11.7.
//   backward: a lane has one piece; partners are whole pieces of the row in shared memory, or single channels (48 and 66 us on 64 slabs of 56 x 56).
// Rows arrive by asynchronous copies, three ahead.  Bound by HBM, forward 4 bytes an element of 16 bits, backward 10, with the issue of instructions close
// behind it (57 % to 73 % of the slots).  A pass among others, inputs that L2 does not hold, 64 channels: norm and rotation on a 256 x 256 grid, 16 slabs,
// 537 MB in 100 us (5.4 TB/s); 64 slabs of 56 x 56, 103 MB in 23 us (4.4 TB/s, starts and angles 5 us of it); rotation of a video grid, 236 MB in 45 us
// (5.2 TB/s); gradient on a 128 x 128 grid, 336 MB in 64 us (5.3 TB/s).
#include "common.cuh"
#include "kernels.h"

namespace aa {

namespace {

constexpr int kRotThreads = 256;
enum PairKind { kNeighbours, kHalvesShuffle, kHalvesShared };      // how partners meet

// What a lane knows of its C channels: frequency in turns (two terms) and axis of the angles that it computes, partners.
template <int C, PairKind KIND> struct LaneAngles {
    static constexpr int kAngles = KIND == kHalvesShared ? C : C / 2;      // (shuffle: the partner lane computes the other half)
    float hi[kAngles], lo[kAngles];
    unsigned axis;                        // two bits an angle
    unsigned rotated;                     // a bit a channel: it has a partner
    unsigned second;                      // a bit a channel: it is the second of its pair
    unsigned char partner[C];             // its partner's channel
};

template <int C, PairKind KIND> __device__ __forceinline__ void lane_angles(const RotateArgs& p, int c0, LaneAngles<C, KIND>& la) {
    la.axis = la.rotated = la.second = 0;
    int freq[C], axes[C];
#pragma unroll
    for (int j = 0; j < C; ++j) {
        const int c = c0 + j;
        int at = 0, fr = 0, partner = c;
        bool second = false;
        freq[j] = -1;
        axes[j] = 3;                      // none: it keeps its value whatever the position, an infinite one too
#pragma unroll
        for (int a = 0; a < 3; ++a) {
            const int seg = p.channels[a], half = seg >> 1, o = c - at;
            if (o >= 0 && o < seg) {
                axes[j] = a;
                if (KIND == kNeighbours) { freq[j] = fr + (o >> 1); second = o & 1; partner = c ^ 1; }
                else { second = o >= half; freq[j] = fr + (second ? o - half : o); partner = second ? c - half : c + half; }
            }
            at += seg;
            fr += half;
        }
        la.partner[j] = (unsigned char)partner;
        if (freq[j] >= 0) la.rotated |= 1u << j;
        if (second) la.second |= 1u << j;
    }
#pragma unroll
    for (int i = 0; i < LaneAngles<C, KIND>::kAngles; ++i) {
        constexpr float kInv = 0.15915494309189535f, kInvLo = 6.420638243e-09f;     // 1 / (2 pi) as a sum of two fp32 numbers
        int f = freq[KIND == kNeighbours ? 2 * i : i], a = axes[KIND == kNeighbours ? 2 * i : i];
        if (KIND == kHalvesShuffle && la.second) { f = freq[i + C / 2]; a = axes[i + C / 2]; }
        const float w = f >= 0 ? __ldg(p.freq + f) : 0.f;
        la.hi[i] = w * kInv;
        la.lo[i] = fmaf(w, kInv, -la.hi[i]) + w * kInvLo;
        la.axis |= (unsigned)a << (2 * i);
    }
}

// cos and sin of position * frequency.  FAST (16-bit results): the special-function unit's, within 5e-7 on half a turn.
template <bool FAST> __device__ __forceinline__ void turn(float pos, float hi, float lo, float& c, float& s) {
    const float t = pos * hi, e = fmaf(pos, lo, fmaf(pos, hi, -t));
    const float r = (t - rintf(t)) + e;
    if (FAST) {
        c = __cosf(6.2831853f * r);
        s = __sinf(6.2831853f * r);
    } else {
        sincospif(2.f * r, &s, &c);
    }
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

__device__ __forceinline__ float on_axis(const float (&pos)[3], unsigned a) { return a == 0 ? pos[0] : a == 1 ? pos[1] : a == 2 ? pos[2] : 0.f; }

// Factors of a channel's own value and of its partner's, in pairs
template <int C, PairKind KIND, bool FAST> __device__ __forceinline__ void token_turns(const RotateArgs& p, const LaneAngles<C, KIND>& la, int b, int tok, int partner_lane, bool inverse, float2 (&cs)[C / 2], float2 (&sn)[C / 2]) {
    constexpr int A = LaneAngles<C, KIND>::kAngles;
    float pos[3], c[C], s[C];
    token_position(p, b, tok, pos);
#pragma unroll
    for (int i = 0; i < A; ++i) {
        const unsigned a = la.axis >> (2 * i) & 3u;
        turn<FAST>(on_axis(pos, a), la.hi[i], la.lo[i], c[i], s[i]);
    }
    if constexpr (KIND == kNeighbours) {
#pragma unroll
        for (int i = C / 2 - 1; i >= 0; --i) { c[2 * i + 1] = c[2 * i] = c[i]; s[2 * i + 1] = s[2 * i] = s[i]; }
    } else if constexpr (KIND == kHalvesShuffle) {
        const bool second = la.second != 0;
#pragma unroll
        for (int i = 0; i < A; ++i) {
            const float oc = __shfl_sync(0xffffffffu, c[i], partner_lane), os = __shfl_sync(0xffffffffu, s[i], partner_lane);
            c[i + A] = second ? c[i] : oc;
            s[i + A] = second ? s[i] : os;
            c[i] = second ? oc : c[i];
            s[i] = second ? os : s[i];
        }
    }
#pragma unroll
    for (int j = 0; j < C; ++j)
        s[j] = __uint_as_float(__float_as_uint(s[j]) ^ ((~la.second >> j & 1u) ^ (inverse ? 1u : 0u)) << 31);      // minus in a pair's first channel
#pragma unroll
    for (int i = 0; i < C / 2; ++i) { cs[i] = make_float2(c[2 * i], c[2 * i + 1]); sn[i] = make_float2(s[2 * i], s[2 * i + 1]); }
}

__device__ __forceinline__ uint4 load_raw(const void* src, bool live) {
    uint4 raw = make_uint4(0u, 0u, 0u, 0u);
    if (live) raw = *static_cast<const uint4*>(src);
    return raw;
}
template <typename T> __device__ __forceinline__ void unpack_pairs(const uint4& raw, float2 (&f)[Elem<T>::kVec / 2]) {
    float v[Elem<T>::kVec];
    unpack16<T>(raw, v);
#pragma unroll
    for (int i = 0; i < Elem<T>::kVec / 2; ++i) f[i] = make_float2(v[2 * i], v[2 * i + 1]);
}

// Sum over the lanes of a token.  Forward kernels: any number of lanes, in one order for all of them.
__device__ __forceinline__ float token_sum(float v, int lanes, int first_lane) {
    if (lanes == 4) {
        v += __shfl_xor_sync(0xffffffffu, v, 1);
        return v + __shfl_xor_sync(0xffffffffu, v, 2);
    }
    float sum = __shfl_sync(0xffffffffu, v, first_lane);
    for (int k = 1; k < lanes; ++k) sum += __shfl_sync(0xffffffffu, v, first_lane + k);
    return sum;
}
__device__ __forceinline__ float group_sum(float v, int lanes) {
    if (lanes >= 4) {                     // (heads of 40 to 64 channels have 4 or 8)
        v += __shfl_xor_sync(0xffffffffu, v, 1);
        v += __shfl_xor_sync(0xffffffffu, v, 2);
        for (int o = 4; o < lanes; o *= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
    } else if (lanes == 2) {
        v += __shfl_xor_sync(0xffffffffu, v, 1);
    }
    return v;
}
__device__ __forceinline__ float2 pair_of(float x) { return make_float2(x, x); }
// a where bit i is set, else b (by a mask: a predicate for each channel is more than there are)
__device__ __forceinline__ float pick(unsigned bits, int i, float a, float b) {
    const unsigned m = 0u - (bits >> i & 1u);
    return __uint_as_float((__float_as_uint(a) & m) | (__float_as_uint(b) & ~m));
}
// (x turned): own values times cs, partners' times sn; a channel without a partner keeps its own
template <int C> __device__ __forceinline__ void turned(const float2 (&x)[C / 2], float2 (&y)[C / 2], const float2 (&cs)[C / 2], const float2 (&sn)[C / 2], unsigned rotated) {
#pragma unroll
    for (int i = 0; i < C / 2; ++i) y[i] = ffma2(y[i], sn[i], fmul2(x[i], cs[i]));
    if (rotated != (1u << C) - 1u) {
#pragma unroll
        for (int i = 0; i < C / 2; ++i) {
            y[i].x = pick(rotated, 2 * i, y[i].x, x[i].x * cs[i].x);
            y[i].y = pick(rotated, 2 * i + 1, y[i].y, x[i].y * cs[i].y);
        }
    }
}
// Where a row lies, slab after slab
template <typename T> struct RowWalk {
    T* at;
    long long step, wrap;                 // from head to head; from the last head to the next batch entry
    __device__ RowWalk(T* base, const TokLayout& l, int slab, int heads, int tok, int c) : at(base + tok_offset(l, slab, heads, tok) + c), step(l.sh), wrap(l.sb - (heads - 1) * l.sh) {}
    __device__ void next(bool last_head) { at += last_head ? wrap : step; }
};

// Position of the block's unit (batch entry, or all of them) and its run of slabs
struct SlabRun { int begin, end; };
__device__ __forceinline__ SlabRun slab_run(const RotateArgs& p) {
    const int unit = blockIdx.y / p.chunks, s0 = unit * p.unit_slabs + (blockIdx.y % p.chunks) * p.share;
    return {s0, min(s0 + p.share, (unit + 1) * p.unit_slabs)};
}
template <int C> __device__ __forceinline__ void square_sum(const float2 (&x)[C / 2], float2& sq) {
#pragma unroll
    for (int i = 0; i < C / 2; ++i) sq = ffma2(x[i], x[i], sq);
}
template <typename T> __device__ __forceinline__ void store_pairs(T* dst, const float2 (&y)[Elem<T>::kVec / 2]) {
    float v[Elem<T>::kVec];
#pragma unroll
    for (int i = 0; i < Elem<T>::kVec / 2; ++i) { v[2 * i] = y[i].x; v[2 * i + 1] = y[i].y; }
    *reinterpret_cast<uint4*>(dst) = pack16<T>(v);
}

// A thread's place in the forward kernels: the warp's lanes make up as many whole groups as there are
struct Place {
    int gl, first, tok;                   // lane of the group, the group's first lane, token (past the last: none)
    int row;                              // thread that has the first piece of the group's row; lanes that make up no whole group look at the warp's first row
    __device__ explicit Place(const RotateArgs& p) {
        const int lane = threadIdx.x & 31, in_warp = 32 / p.lanes, group = lane / p.lanes;
        gl = lane - group * p.lanes;
        first = lane - gl;
        tok = group < in_warp ? (blockIdx.x * (kRotThreads / 32) + (threadIdx.x >> 5)) * in_warp + group : p.N;
        row = group < in_warp ? threadIdx.x - gl : threadIdx.x & ~31;
    }
};

// Rows of a block's run, tensor after tensor, slab after slab: where the next one lies
template <typename T> struct RowCursor {
    const T* at;
    long long step, wrap;
    int head, heads, left, tensor;
    const RotateArgs& p;
    long long start;
    int run, first_head;
    bool output;
    __device__ RowCursor(const RotateArgs& args, const SlabRun& r, int tok, int c, bool out, int first)
        : heads(args.heads), tensor(first), p(args), run(r.end - r.begin), first_head(r.begin % args.heads), output(out) {
        const TokLayout& l = out ? args.lout : args.lin;
        start = tok_offset(l, r.begin, heads, tok) + c;
        step = l.sh;
        wrap = l.sb - (heads - 1) * l.sh;
        begin();
    }
    __device__ void begin() {
        left = run;
        head = first_head;
        at = static_cast<const T*>(output ? p.y[tensor] : p.x[tensor]) + start;
    }
    __device__ void next() {              // (past the last row it stays somewhere that nobody reads)
        if (--left == 0) {
            tensor = 1;
            begin();
            return;
        }
        if (++head == heads) { head = 0; at += wrap; }
        else at += step;
    }
};

// A lane has two pieces u and v of its token's row.  Rows arrive by asynchronous copies, kDepth - 1 ahead: in registers one row ahead is all there is
// room for, which leaves the 256 x 256 grid at 118 us.
constexpr int kDepth = 4;
template <typename T, bool HALVES, bool NORM> __global__ void __launch_bounds__(kRotThreads, 3) rotate_pairs_kernel(const __grid_constant__ RotateArgs p) {
    constexpr int C = Elem<T>::kVec;
    __shared__ uint4 s_ring[kDepth][2][kRotThreads];
    __shared__ float2 s_turn[NORM ? C : 1][NORM ? kRotThreads : 1];          // (cos, sin): the gains are folded into them tensor by tensor
    pdl_wait_prior();
    pdl_release_next();
    const Place at(p);
    const int gl = at.gl, tok = at.tok, first = p.x[0] ? 0 : 1, tensors = p.x[0] && p.x[1] ? 2 : 1;
    const SlabRun run = slab_run(p);
    // channels of the pieces, and the number of the first angle: with HALVES that of u's first channel, which is v's too
    int cu = 2 * gl * C, cv = cu + C, angle = 0, axis = 0;
    bool turns = !HALVES;
    if (HALVES) {
        int start = 0, fr = 0, left = gl;
#pragma unroll
        for (int a = 0; a < 3; ++a) {
            const int half = p.channels[a] >> 1;
            if (!turns && left >= 0) {
                if (left * C < half) {
                    turns = true;
                    cu = start + left * C; cv = cu + half;
                    angle = fr + left * C;
                    axis = a;
                }
                left -= half / C;
            }
            start += 2 * half;
            fr += half;
        }
        if (!turns) { cu = start + 2 * left * C; cv = cu + C; }         // past the segments
    }
    const int dv = cv - cu, size_u = tok < p.N && cu < p.d ? 16 : 0, size_v = tok < p.N && cv < p.d ? 16 : 0;
    const int n = run.end - run.begin, rows = n * tensors;
    RowCursor<T> in(p, run, min(tok, p.N - 1), cu < p.d ? cu : 0, false, first);
    auto fetch = [&](int i, int stage) {
        if (i < rows) {
            cp_async16(&s_ring[stage][0][threadIdx.x], in.at, size_u);
            cp_async16(&s_ring[stage][1][threadIdx.x], in.at + (size_v ? dv : 0), size_v);
            in.next();
        }
        cp_async_commit();
    };
#pragma unroll
    for (int i = 0; i < kDepth - 1; ++i) fetch(i, i);

    float2 own_u[C / 2], par_u[C / 2], own_v[C / 2], par_v[C / 2];
    unsigned apart = 0;                                              // neighbours: a bit for each pair (of u, then of v) that does not turn
    float c[C], s[C];
    {
        float pos[3];
        token_position(p, run.begin / p.heads, min(tok, p.N - 1), pos);
#pragma unroll
        for (int j = 0; j < C; ++j) {
            int f = angle + j, ax = axis;
            bool on = turns;
            if (!HALVES) {                                           // pair j of the 16 bytes u, v: channels 2 gl C + 2 j and the next
                const int ch = cu + 2 * j;
                f = ch >> 1;
                ax = ch < p.channels[0] ? 0 : ch < p.channels[0] + p.channels[1] ? 1 : 2;
                on = ch < p.channels[0] + p.channels[1] + p.channels[2];
                if (!on && ch < p.d) apart |= 1u << j;
            }
            const float w = on ? __ldg(p.freq + f) : 0.f;
            constexpr float kInv = 0.15915494309189535f, kInvLo = 6.420638243e-09f;     // 1 / (2 pi) as a sum of two fp32 numbers
            const float hi = w * kInv, lo = fmaf(w, kInv, -hi) + w * kInvLo;
            turn<sizeof(T) == 2>(on_axis(pos, on ? ax : 3), hi, lo, c[j], s[j]);
            if (p.inverse) s[j] = -s[j];
            if (NORM) s_turn[j][threadIdx.x] = make_float2(c[j], s[j]);
        }
    }
    auto factors = [&](int t) {
        if (HALVES) {
#pragma unroll
            for (int i = 0; i < C / 2; ++i) {
                own_u[i] = own_v[i] = make_float2(c[2 * i], c[2 * i + 1]);
                par_u[i] = make_float2(-s[2 * i], -s[2 * i + 1]);
                par_v[i] = make_float2(s[2 * i], s[2 * i + 1]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < C / 2; ++i) {
                own_u[i] = pair_of(c[i]);
                own_v[i] = pair_of(c[C / 2 + i]);
                par_u[i] = make_float2(-s[i], s[i]);
                par_v[i] = make_float2(-s[C / 2 + i], s[C / 2 + i]);
            }
        }
        if (NORM && p.gain[t]) {
            const T* g = static_cast<const T*>(p.gain[t]);
            float2 gu[C / 2], gv[C / 2];
            unpack_pairs<T>(load_raw(g + cu, cu < p.d), gu);
            unpack_pairs<T>(load_raw(g + cv, cv < p.d), gv);
#pragma unroll
            for (int i = 0; i < C / 2; ++i) {
                own_u[i] = fmul2(own_u[i], gu[i]);
                own_v[i] = fmul2(own_v[i], gv[i]);
                par_u[i] = fmul2(par_u[i], HALVES ? gv[i] : make_float2(gu[i].y, gu[i].x));
                par_v[i] = fmul2(par_v[i], HALVES ? gu[i] : make_float2(gv[i].y, gv[i].x));
            }
        }
    };
    factors(first);
    RowCursor<T> out(p, run, min(tok, p.N - 1), cu, true, first);
    auto row = [&](int i, int stage) {
        if (NORM && i == n) {                                        // the keys: other gains
#pragma unroll
            for (int j = 0; j < C; ++j) { c[j] = s_turn[j][threadIdx.x].x; s[j] = s_turn[j][threadIdx.x].y; }
            factors(1);
        }
        fetch(i + kDepth - 1, (stage + kDepth - 1) % kDepth);
        cp_async_wait<kDepth - 1>();
        float2 u[C / 2], v[C / 2], yu[C / 2], yv[C / 2];
        unpack_pairs<T>(s_ring[stage][0][threadIdx.x], u);
        unpack_pairs<T>(s_ring[stage][1][threadIdx.x], v);
        float r = 1.f;
        if (NORM) {
            float2 sq = pair_of(0.f);
            square_sum<C>(u, sq);
            square_sum<C>(v, sq);
            r = rsqrtf(token_sum(sq.x + sq.y, p.lanes, at.first) * p.inv_d + p.eps);
        }
#pragma unroll
        for (int k = 0; k < C / 2; ++k) {
            yu[k] = fmul2(u[k], own_u[k]);
            yv[k] = fmul2(v[k], own_v[k]);
        }
        if (turns) {
#pragma unroll
            for (int k = 0; k < C / 2; ++k) {
                const float2 tu = ffma2(HALVES ? v[k] : make_float2(u[k].y, u[k].x), par_u[k], yu[k]), tv = ffma2(HALVES ? u[k] : make_float2(v[k].y, v[k].x), par_v[k], yv[k]);
                if (HALVES || !apart) {
                    yu[k] = tu;
                    yv[k] = tv;
                } else {
                    yu[k] = make_float2(pick(apart, k, yu[k].x, tu.x), pick(apart, k, yu[k].y, tu.y));
                    yv[k] = make_float2(pick(apart, C / 2 + k, yv[k].x, tv.x), pick(apart, C / 2 + k, yv[k].y, tv.y));
                }
            }
        }
        if (NORM) {
#pragma unroll
            for (int k = 0; k < C / 2; ++k) {
                yu[k] = fmul2(yu[k], pair_of(r));
                yv[k] = fmul2(yv[k], pair_of(r));
            }
        }
        T* dst = const_cast<T*>(out.at);
        if (size_u) store_pairs<T>(dst, yu);
        if (size_v) store_pairs<T>(dst + dv, yv);
        out.next();
    };
#pragma unroll 1
    for (int i = 0; i < rows; i += kDepth) {
#pragma unroll
        for (int k = 0; k < kDepth; ++k)
            if (i + k < rows) row(i + k, k);
    }
}

// A lane has one piece; partners through shared memory, where the row lies as it is in memory: 32-bit words (WORDS: fp32, or 16-bit segments of a
// multiple of four channels, whose pairs' partners are pairs), else element by element.
template <typename T, bool WORDS, bool NORM> __global__ void __launch_bounds__(kRotThreads, NORM ? 3 : 4) rotate_patch_kernel(const __grid_constant__ RotateArgs p) {
    constexpr int C = Elem<T>::kVec, kPer = sizeof(T) == 4 ? 1 : 2;  // elements of a word
    __shared__ uint4 s_ring[kDepth][kRotThreads];
    pdl_wait_prior();
    pdl_release_next();
    const Place at(p);
    const int gl = at.gl, c0 = gl * C, tok = at.tok;
    const int first = p.x[0] ? 0 : 1, tensors = p.x[0] && p.x[1] ? 2 : 1;
    const SlabRun run = slab_run(p);
    const int size = tok < p.N && c0 < p.d ? 16 : 0, n = run.end - run.begin, rows = n * tensors;
    RowCursor<T> in(p, run, min(tok, p.N - 1), c0 < p.d ? c0 : 0, false, first);
    auto fetch = [&](int i, int stage) {
        if (i < rows) {
            cp_async16(&s_ring[stage][threadIdx.x], in.at, size);
            in.next();
        }
        cp_async_commit();
    };
#pragma unroll
    for (int i = 0; i < kDepth - 1; ++i) fetch(i, i);
    LaneAngles<C, kHalvesShared> la;
    lane_angles<C, kHalvesShared>(p, c0, la);
    float2 cs[C / 2], sn[C / 2], own[C / 2], par[C / 2];
    token_turns<C, kHalvesShared, sizeof(T) == 2>(p, la, run.begin / p.heads, min(tok, p.N - 1), at.first, p.inverse, cs, sn);
    auto factors = [&](int t) {
#pragma unroll
        for (int i = 0; i < C / 2; ++i) { own[i] = cs[i]; par[i] = sn[i]; }
        if (NORM && p.gain[t] && c0 < p.d) {
            const T* g = static_cast<const T*>(p.gain[t]);
#pragma unroll
            for (int i = 0; i < C / 2; ++i) {
                own[i] = fmul2(own[i], make_float2(Elem<T>::to_f32(g[c0 + 2 * i]), Elem<T>::to_f32(g[c0 + 2 * i + 1])));
                par[i] = fmul2(par[i], make_float2(Elem<T>::to_f32(g[la.partner[2 * i]]), Elem<T>::to_f32(g[la.partner[2 * i + 1]])));
            }
        }
    };
    factors(first);
    const bool whole = la.rotated == (1u << C) - 1u;
    RowCursor<T> out(p, run, min(tok, p.N - 1), c0, true, first);
    auto row_of = [&](int i, int stage) {
        if (NORM && i == n) factors(1);
        __syncwarp();                                                // (the stage that is filled next has been read by the whole warp)
        fetch(i + kDepth - 1, (stage + kDepth - 1) % kDepth);
        cp_async_wait<kDepth - 1>();
        __syncwarp();
        const T* row = reinterpret_cast<const T*>(&s_ring[stage][at.row]);
        float2 x[C / 2], y[C / 2];
        unpack_pairs<T>(s_ring[stage][threadIdx.x], x);
        if (WORDS) {
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = *reinterpret_cast<const uint32_t*>(row + la.partner[kPer * k]);
            unpack_pairs<T>(make_uint4(w[0], w[1], w[2], w[3]), y);
        } else {
#pragma unroll
            for (int k = 0; k < C / 2; ++k) y[k] = make_float2(Elem<T>::to_f32(row[la.partner[2 * k]]), Elem<T>::to_f32(row[la.partner[2 * k + 1]]));
        }
        float r = 1.f;
        if (NORM) {
            float2 sq = pair_of(0.f);
            square_sum<C>(x, sq);
            r = rsqrtf(token_sum(sq.x + sq.y, p.lanes, at.first) * p.inv_d + p.eps);
        }
#pragma unroll
        for (int k = 0; k < C / 2; ++k) {
            const float2 o = fmul2(x[k], own[k]);
            y[k] = ffma2(y[k], par[k], o);
            if (!whole) {
                y[k].x = pick(la.rotated, 2 * k, y[k].x, o.x);
                y[k].y = pick(la.rotated, 2 * k + 1, y[k].y, o.y);
            }
            if (NORM) y[k] = fmul2(y[k], pair_of(r));
        }
        if (size) store_pairs<T>(const_cast<T*>(out.at), y);
        out.next();
    };
#pragma unroll 1
    for (int i = 0; i < rows; i += kDepth) {
#pragma unroll
        for (int k = 0; k < kDepth; ++k)
            if (i + k < rows) row_of(i + k, k);
    }
}

// The gradient's work: a line of slabs, in which those of a tile of tokens (and of a batch entry, where positions differ) lie side by side.  A block has an
// even part of it: runs of a few tiles, angles once for each.  Runs of one length, dealt out block by block, left the last round of them emptier: 384
// slabs of 196 tokens took 27.5 us instead of 24.1, 16 of 128 x 128 66 instead of 63.6.  (Not the forward kernels': blocks that come and go keep to one region of
// memory at a time; as a line the 256 x 256 grid takes 110 us instead of 100.)
struct SlabLine {
    long long at, end;
    __device__ explicit SlabLine(const RotateArgs& p) {
        const long long total = (long long)p.tiles * p.slabs;
        at = total * blockIdx.x / gridDim.x;
        end = total * (blockIdx.x + 1) / gridDim.x;
    }
    __device__ bool next(const RotateArgs& p, int& tile, SlabRun& r) {
        if (at >= end) return false;
        const long long column = at / p.unit_slabs;
        const int first = (int)(at - column * p.unit_slabs), unit = (int)(column / p.tiles);
        tile = (int)(column - (long long)unit * p.tiles);
        r.begin = unit * p.unit_slabs + first;
        r.end = r.begin + (int)min((long long)(p.unit_slabs - first), end - at);
        at += r.end - r.begin;
        return true;
    }
};
// Gradient through norm and rotation.  A block has one of the tensors (blockIdx.y); the gain's gradient stays in registers until the block's end and
// leaves as one row of sums a block, which gain_sum_kernel adds up in a fixed order.  A lane has 16 bytes of x; the gradient's row (fp32) is copied by
// the group's lanes in whole sectors and lies in shared memory as it is in memory, from where a lane reads its channels and their partners.  Results
// change hands between two lanes so that they leave in whole sectors.
template <typename T, PairKind KIND> __global__ void __launch_bounds__(kRotThreads, 3) rotate_backward_kernel(const __grid_constant__ RotateBwdArgs p) {
    constexpr int C = Elem<T>::kVec, kPieces = C / 4, kAhead = 3;            // 16-byte pieces of a lane's fp32 channels
    extern __shared__ __align__(16) unsigned char s_dyn[];                   // [kAhead][1 + kPieces][threads] uint4; at the end sums
    uint4* ring = reinterpret_cast<uint4*>(s_dyn);
    constexpr int kStage = (1 + kPieces) * kRotThreads;
    pdl_wait_prior();
    pdl_release_next();
    const RotateArgs& f = p.fwd;
    const int lane = threadIdx.x & 31, gl = lane & (f.lanes - 1), c0 = gl * C, first_lane = lane - gl;
    const int groups = kRotThreads / f.lanes, t = f.x[0] ? blockIdx.y : 1;
    LaneAngles<C, KIND> la;
    lane_angles<C, KIND>(f, c0, la);
    const int partner_lane = first_lane + la.partner[0] / C;
    const T *xs = static_cast<const T*>(f.x[t]), *gs = static_cast<const T*>(f.gain[t]);
    const float* grad = p.grad[t];
    float* dst = static_cast<float*>(f.y[t]);
    float2 gain[C / 2], sum[C / 2];
#pragma unroll
    for (int i = 0; i < C / 2; ++i) {
        gain[i] = gs && c0 < f.d ? make_float2(Elem<T>::to_f32(gs[c0 + 2 * i]), Elem<T>::to_f32(gs[c0 + 2 * i + 1])) : pair_of(1.f);
        sum[i] = pair_of(0.f);
    }
    const int row_at = kRotThreads + (threadIdx.x - gl) * kPieces;       // of the group's gradient row in a stage
    SlabLine line(f);
    SlabRun run;
    int tile;
#pragma unroll 1
    while (line.next(f, tile, run)) {
        const int tok = tile * groups + threadIdx.x / f.lanes;
        const bool token = tok < f.N, live = token && c0 < f.d;
        const int here = min(tok, f.N - 1), ch = c0 < f.d ? c0 : 0;
        const int s0 = run.begin, n = run.end - run.begin;
        RowWalk<const T> in(xs, f.lin, s0, f.heads, here, ch);
        RowWalk<const float> gin(grad, p.lgrad, s0, f.heads, here, 0);
        RowWalk<float> out(dst, f.lout, s0, f.heads, here, 0);
        int head = s0 % f.heads, fhead = head;
        int piece_at[kPieces], piece_size[kPieces];
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {
            const int at = 4 * (gl + k * f.lanes);
            piece_size[k] = token && at < f.d ? 16 : 0;
            piece_at[k] = at < f.d ? at : 0;
        }
        auto fetch = [&](int i, int stage) {
            if (i < n) {
                uint4* to = ring + stage * kStage;
                cp_async16(to + threadIdx.x, in.at, live ? 16 : 0);
#pragma unroll
                for (int k = 0; k < kPieces; ++k) cp_async16(to + row_at + gl + k * f.lanes, gin.at + piece_at[k], piece_size[k]);
                const bool wrap = ++fhead == f.heads;
                if (wrap) fhead = 0;
                in.next(wrap);
                gin.next(wrap);
            }
            cp_async_commit();
        };
        __syncwarp();
#pragma unroll
        for (int i = 0; i < kAhead - 1; ++i) fetch(i, i);
        float2 cs[C / 2], sn[C / 2];
        token_turns<C, KIND, false>(f, la, s0 / f.heads, here, partner_lane, true, cs, sn);
        auto row_of = [&](int i, int stage) {
            __syncwarp();                                                    // (the stage that is filled next has been read by the whole warp)
            fetch(i + kAhead - 1, (stage + kAhead - 1) % kAhead);
            cp_async_wait<kAhead - 1>();
            __syncwarp();
            const uint4* from = ring + stage * kStage;
            const float* row = reinterpret_cast<const float*>(from + row_at);
            float2 x[C / 2], g[C / 2], y[C / 2];
            unpack_pairs<T>(from[threadIdx.x], x);
#pragma unroll
            for (int k = 0; k < kPieces; ++k) {
                const float4 w = *reinterpret_cast<const float4*>(row + c0 + 4 * k);
                g[2 * k] = make_float2(w.x, w.y);
                g[2 * k + 1] = make_float2(w.z, w.w);
            }
            if constexpr (KIND == kNeighbours) {
#pragma unroll
                for (int k = 0; k < C / 2; ++k) y[k] = make_float2(g[k].y, g[k].x);
            } else if constexpr (KIND == kHalvesShuffle) {
#pragma unroll
                for (int k = 0; k < kPieces; ++k) {
                    const float4 w = *reinterpret_cast<const float4*>(row + la.partner[0] + 4 * k);
                    y[2 * k] = make_float2(w.x, w.y);
                    y[2 * k + 1] = make_float2(w.z, w.w);
                }
            } else {
#pragma unroll
                for (int k = 0; k < C / 2; ++k) y[k] = make_float2(row[la.partner[2 * k]], row[la.partner[2 * k + 1]]);
            }
            turned<C>(g, y, cs, sn, la.rotated);
            float2 sq = pair_of(0.f), dot = pair_of(0.f);
#pragma unroll
            for (int k = 0; k < C / 2; ++k) {
                sq = ffma2(x[k], x[k], sq);
                dot = ffma2(fmul2(y[k], gain[k]), x[k], dot);
            }
            const float ms = group_sum(sq.x + sq.y, f.lanes) * f.inv_d;
            const float r = token ? rsqrtf(ms + f.eps) : 0.f;                // (past the last token nothing is added to the gains' sums, not 0 / sqrt(0) for eps = 0)
            const float m = -group_sum(dot.x + dot.y, f.lanes) * f.inv_d * r * r * r;
            float v[C];
#pragma unroll
            for (int k = 0; k < C / 2; ++k) {
                sum[k] = ffma2(y[k], fmul2(x[k], pair_of(r)), sum[k]);
                y[k] = ffma2(fmul2(gain[k], pair_of(r)), y[k], fmul2(pair_of(m), x[k]));
                v[2 * k] = y[k].x;
                v[2 * k + 1] = y[k].y;
            }
            float* to = out.at;
            if (kPieces == 1) {
                if (live) *reinterpret_cast<float4*>(to + c0) = make_float4(v[0], v[1], v[2], v[3]);
            } else if (f.lanes == 1) {
                if (live) {
#pragma unroll
                    for (int k = 0; k < kPieces; ++k) *reinterpret_cast<float4*>(to + c0 + 4 * k) = make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
                }
            } else {
                // the even lane of two gets its first piece and the odd one's first, the odd lane the second ones: 32 bytes side by side a store
                const bool odd = gl & 1;
                float w[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    w[k] = __shfl_xor_sync(0xffffffffu, odd ? v[k] : v[(4 + k) % C], 1);
                    if (odd) { v[k] = w[k]; w[k] = v[(4 + k) % C]; }
                }
                const int pair = (gl & ~1) * C + (odd ? 4 : 0);
                if (token && pair < f.d) *reinterpret_cast<float4*>(to + pair) = make_float4(v[0], v[1], v[2], v[3]);
                if (token && pair + C < f.d) *reinterpret_cast<float4*>(to + pair + C) = make_float4(w[0], w[1], w[2], w[3]);
            }
            const bool wrap = ++head == f.heads;
            if (wrap) head = 0;
            out.next(wrap);
        };
#pragma unroll 1
        for (int i = 0; i < n; i += kAhead) {
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                if (i + k < n) row_of(i + k, k);
        }
    }
    float* s_sum = reinterpret_cast<float*>(s_dyn);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < C / 2; ++i) *reinterpret_cast<float2*>(s_sum + threadIdx.x * C + 2 * i) = sum[i];
    __syncthreads();
    const int width = f.lanes * C;
    if (threadIdx.x < f.d) {
        float v = 0.f;
        for (int k = 0; k < groups; ++k) v += s_sum[k * width + threadIdx.x];
        p.part[((long long)t * gridDim.x + blockIdx.x) * f.d + threadIdx.x] = v;
    }
}

// Sum of the blocks' rows: 32 columns of a tensor's d, each row's in turn by 32 warps
__global__ void __launch_bounds__(1024) gain_sum_kernel(const float* part, int rows, int d, float* dq, float* dk) {
    __shared__ float s_sum[32][33];
    pdl_wait_prior();
    pdl_release_next();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = 32 * blockIdx.x + lane;
    float* out = blockIdx.y ? dk : dq;
    if (!out) return;
    float v = 0.f;
    if (c < d) {
#pragma unroll 8
        for (int r = warp; r < rows; r += 32) v += part[((long long)blockIdx.y * rows + r) * d + c];
    }
    s_sum[warp][lane] = v;
    __syncthreads();
    v = s_sum[lane][warp];
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (lane == 0 && 32 * blockIdx.x + warp < d) out[32 * blockIdx.x + warp] = v;
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

// Tiles of `tokens`, and slabs whose positions are the same
int units_of(RotateArgs* a, int tokens) {
    a->unit_slabs = a->positions && a->pos_batch ? a->heads : a->slabs;
    a->inv_d = 1.f / (float)a->d;
    return a->tiles = (a->N + tokens - 1) / tokens;
}
// How many slabs a block visits with one set of angles; `tokens` of a block.  Fewer: the angles cost more, as much as
// four rows; more: the last of the waves of `resident` blocks is emptier.  `rows`: of a slab (the tensors of a block).  With angles at 0, 1, 2, 4, 8 and 16
// rows (us): norm and rotation of 16 slabs of 128 x 128, bf16, in whole pairs 30.2, 30.3, 26.5, 26.5, 31.7 and 31.6, through shared memory 101, 49, 48, 42, 42 and
// 46; rotation of the video grid 130, 52, 42, 42, 42 and 42; fp32, 16 slabs of 128 x 128 x 64 channels 69, 43, 43, 46, 46 and 52 (two rows would do there).
int plan_rotate(RotateArgs* a, int tokens, int rows, int resident) {
    const int tiles = units_of(a, tokens);
    const long long alone = (long long)tiles * (a->slabs / a->unit_slabs);          // blocks if each visits all slabs of its unit
    long long best = 0;
    for (int chunks = 1; chunks <= a->unit_slabs; ++chunks) {
        const int share = (a->unit_slabs + chunks - 1) / chunks;
        const long long blocks = alone * ((a->unit_slabs + share - 1) / share), cost = (blocks + resident - 1) / resident * (4 + rows * share);
        if (chunks == 1 || cost < best) {
            best = cost;
            a->share = share;
        }
        if (blocks > 16ll * resident) break;
    }
    a->chunks = (a->unit_slabs + a->share - 1) / a->share;
    return tiles;
}

template <typename T> cudaError_t launch_rotate_type(RotateArgs a, int sm_count, cudaStream_t st) {
    constexpr int C = Elem<T>::kVec;
    const int tensors = (a.x[0] != nullptr) + (a.x[1] != nullptr);
    PairKind kind = pair_kind(a, C);
    if (C == 8 && !a.norm && kind == kHalvesShuffle) kind = kHalvesShared;
    int lanes = (a.d + C - 1) / C;
    if (kind == kNeighbours) lanes = (a.d + 2 * C - 1) / (2 * C);
    if (kind == kHalvesShuffle) {
        const int turning = a.channels[0] + a.channels[1] + a.channels[2];
        lanes = turning / (2 * C) + (a.d - turning + 2 * C - 1) / (2 * C);
    }
    a.lanes = lanes;
    const int tiles = plan_rotate(&a, kRotThreads / 32 * (32 / lanes), tensors, (kind == kHalvesShared && !a.norm ? 4 : 3) * sm_count);
    const dim3 grid(tiles, a.chunks * (a.slabs / a.unit_slabs));
    auto launch = [&](auto plain, auto norm) { return launch_dependent(a.norm ? norm : plain, grid, kRotThreads, 0, st, a); };
    if (kind == kNeighbours) return launch(rotate_pairs_kernel<T, false, false>, rotate_pairs_kernel<T, false, true>);
    if (kind == kHalvesShuffle) return launch(rotate_pairs_kernel<T, true, C == 8>, rotate_pairs_kernel<T, true, true>);
    // 32-bit words, or element by element: the video grid of 8 x 45 x 80, bf16, 44.8 and 51.2 us
    const bool words = C == 4 || (a.channels[0] % 4 == 0 && a.channels[1] % 4 == 0 && a.channels[2] % 4 == 0);
    if (words) return launch(rotate_patch_kernel<T, true, false>, rotate_patch_kernel<T, true, true>);
    return launch(rotate_patch_kernel<T, C == 4, false>, rotate_patch_kernel<T, C == 4, true>);
}

int backward_blocks(int sm_count) { return 3 * sm_count; }           // of a tensor
template <typename T, PairKind KIND> cudaError_t launch_backward_kind(const RotateBwdArgs& a, dim3 grid, cudaStream_t st) {
    constexpr int kBytes = 3 * (1 + Elem<T>::kVec / 4) * kRotThreads * 16;
    return launch_dependent(rotate_backward_kernel<T, KIND>, grid, kRotThreads, kBytes, st, a);
}
template <typename T> cudaError_t launch_rotate_bwd_type(RotateBwdArgs a, int sm_count, cudaStream_t st) {
    const int tensors = (a.fwd.x[0] != nullptr) + (a.fwd.x[1] != nullptr), most = backward_blocks(sm_count) / tensors;
    a.fwd.lanes = 1;
    while (a.fwd.lanes * Elem<T>::kVec < a.fwd.d) a.fwd.lanes *= 2;
    const long long all = (long long)units_of(&a.fwd, kRotThreads / a.fwd.lanes) * a.fwd.slabs;
    const int blocks = (int)(all < most ? all : most);
    const dim3 grid(blocks, tensors);
    cudaError_t e;
    switch (pair_kind(a.fwd, Elem<T>::kVec)) {
        case kNeighbours: e = launch_backward_kind<T, kNeighbours>(a, grid, st); break;
        case kHalvesShuffle: e = launch_backward_kind<T, kHalvesShuffle>(a, grid, st); break;
        default: e = launch_backward_kind<T, kHalvesShared>(a, grid, st); break;
    }
    if (e != cudaSuccess || (!a.dgain[0] && !a.dgain[1])) return e;
    return launch_dependent(gain_sum_kernel, dim3((a.fwd.d + 31) / 32, 2), 1024, 0, st, a.part, blocks, a.fwd.d, a.dgain[0], a.dgain[1]);
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
