// Softmax attention over whole sequences: what its kernels share.
//
//     P = softmax over the visible keys of scale Q K^T,  O = P V        dV = P^T dO,  dP = dO V^T,  dS = P (dP - D),  D = rowsum(dO O)
//     dQ = scale dS K,  dK = scale dS^T Q
//
// A sequence is a run of queries and a run of keys: a batch entry (its first `length` rows, or all of them), or rows offsets[s] .. offsets[s + 1] of the
// only batch entry.  Lengths and offsets are device numbers, so the host plans for the most that can be; every kernel clamps them to the tensors and
// blocks without work end at once.  Causal: query i of nq sees the keys j <= i + nk - nq of nk.
#pragma once
#include "common.cuh"
#include "kernels.h"

namespace aa {

struct Span {
    int batch, first, count;
};
// Rows of sequence s: `most` rows a batch entry
__device__ __forceinline__ Span span_of(const int* offsets, const int* lengths, int most, int s) {
    Span r;
    if (offsets) {
        const int a = min(max(__ldg(offsets + s), 0), most);
        r.batch = 0;
        r.first = a;
        r.count = min(max(__ldg(offsets + s + 1), a), most) - a;
    } else {
        r.batch = s;
        r.first = 0;
        r.count = lengths ? min(max(__ldg(lengths + s), 0), most) : most;
    }
    return r;
}

// Tiles of `rows` rows (of `unit` rows a token: the heads that share keys) of all sequences.  Of packed sequences the first slot of s is
// floor(offset unit / rows) + s: at least as many slots as tiles, and the sequence of a slot is found by bisection, without a sum over the others.
__host__ __device__ inline long long slots_of(bool packed, int sequences, int most, int unit, int rows) {
    return packed ? (long long)most * unit / rows + sequences : (((long long)most * unit + rows - 1) / rows) * sequences;
}
__device__ __forceinline__ bool find_slot(const int* offsets, int sequences, int most, int unit, int rows, unsigned slot, int* seq, int* tile) {
    if (!offsets) {
        const unsigned per = (unsigned)(((long long)most * unit + rows - 1) / rows);
        *seq = (int)(slot / per);
        *tile = (int)(slot % per);
        return true;
    }
    auto base = [&](int s) { return (unsigned)((long long)min(max(__ldg(offsets + s), 0), most) * unit / rows) + (unsigned)s; };
    int lo = 0, hi = sequences;                    // base(lo) <= slot < base(hi), or there is none
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (base(mid) <= slot) lo = mid;
        else hi = mid;
    }
    const unsigned b = base(lo);
    *seq = lo;
    *tile = (int)(slot - b);
    return slot >= b;
}
// Keys that query i of a sequence sees: 0 .. result - 1
__device__ __forceinline__ int visible_keys(int causal, int i, int nq, int nk) { return causal ? max(0, min(nk, i + nk - nq + 1)) : nk; }

// How long a sum in a tensor core's accumulator gets.  It cuts off what lies below the last bit at every step of 16, always towards zero: 3e-8 of the sum a step, half of
// that on the average of a sum that grows, so 2^20 rows would be off by 1e-3 (2 f16 roundings; 2^25 by 18 %).  Pieces of 1024 steps are off by 3e-5 at most and join in fp32.
constexpr int kPieceKeys = 16384;

constexpr float kLn2 = 0.6931471805599453f;

// The exponents' reference of a row moves only when a logit exceeds it by more than kSlack (log2 units), so P is at most 2^kSlack.  f16, whose normal numbers end at
// 2^-14 and whose last one is 2^-24, holds P times 2^kHeld, as much as its range leaves: keys far below a row's largest lose no bits before 2^-25 of it, and half a
// step of the last number is 2^-36 (the sum counts what P V would lose: 65536 keys 17.5 below one, 1.6e-3 of the result).  The factor leaves with the row's sum.
// (The smaller slack: 8 heads of 8192 x 8192 x 128 281 us with logits that vary by 1, bf16 280; 313 where they vary by 3, bf16 291; 324 by 10, bf16 318.)
template <typename T> constexpr bool is_f16 = sizeof(T) == 2 && !Elem<T>::kIsBf16;
template <typename T> constexpr float kSlack = is_f16<T> ? 4.f : 8.f;
template <typename T> constexpr float kHeld = is_f16<T> ? 11.f : 0.f;

// f16 gradients.  P and dS are operands of products and have to be f16, whose normal numbers end at 2^-14: P is held times 2^15 (it is at most one), dS times the
// power of two that brings the bound 2 |dO_i| max |v_j| of |dP - D| into [2^14, 2^15): of the row where rows are queries, of the sequence's largest row
// where the sum goes over them.  The results are brought back in fp32.
constexpr float kHeldP = 15.f, kHeldBack = 1.f / 32768.f;
constexpr int kDotRows = 64;
__host__ __device__ inline float* grad_norms(const AttendArgs& a) { return a.ws + 2 * (long long)a.batch * a.heads * a.N; }
__host__ __device__ inline unsigned* grad_most(const AttendArgs& a, int seq, int hk) {
    return reinterpret_cast<unsigned*>(a.ws + 3 * (long long)a.batch * a.heads * a.N) + 2 * ((long long)seq * a.kv_heads + hk);
}
// The power of two for dP - D where P is held times 2^15 already
__device__ __forceinline__ float grad_factor(float dout, float value) {
    const float bound = 2.f * dout * value;
    if (!(bound > 1e-30f) || !(bound < 1e30f)) return kHeldBack;               // (nothing to hold, or nothing that could be)
    const int e = (int)((__float_as_uint(bound) >> 23) & 0xffu) - 127;         // bound in [2^e, 2^(e + 1))
    return __uint_as_float((unsigned)(127 + 14 - e - 15) << 23);               // e in [-100, 100]
}

}  // namespace aa
