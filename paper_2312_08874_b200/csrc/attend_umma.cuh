// Softmax attention over whole sequences on the 5th-generation tensor cores: what the forward kernel and the gradients' share.
#pragma once
#include "attend.cuh"
#include "pair.cuh"
#include "stream_common.cuh"

namespace aa {

// Map of a [batch][heads][rows][d] tensor of 16-bit elements with any strides: boxes of 64 channels x `box_rows` rows of one head, 128-byte swizzle; channels past
// d and rows past the tensor read zero.  Dimensions 1 to 3 are rows (0), head (1) and batch (2) in the order of their strides.
struct RowMap {
    alignas(64) CUtensorMap map;
    int order[3];
};
__device__ __forceinline__ void load_rows(uint32_t dst, const RowMap& m, int channel, int row, int head, int batch, uint32_t bar) {
    auto at = [&](int i) { return m.order[i] == 0 ? row : m.order[i] == 1 ? head : batch; };
    tma_load_4d(dst, &m.map, channel, at(0), at(1), at(2), bar);
}
inline bool make_row_map(RowMap* out, const void* base, const TokLayout& l, int batch, int heads, int rows, int d, int box_rows = 128) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t n[3] = {(cuuint64_t)rows, (cuuint64_t)heads, (cuuint64_t)batch};
    const cuuint64_t s[3] = {(cuuint64_t)l.st * 2, (cuuint64_t)l.sh * 2, (cuuint64_t)l.sb * 2};
    int o[3] = {0, 1, 2};                          // single entries last (their strides are never used), the others by stride
    auto before = [&](int a, int b) { return (n[a] > 1) != (n[b] > 1) ? n[a] > 1 : n[a] > 1 && s[a] < s[b]; };
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2 - i; ++j)
            if (before(o[j + 1], o[j])) { const int t = o[j]; o[j] = o[j + 1]; o[j + 1] = t; }
    cuuint64_t dims[4] = {(cuuint64_t)d, 0, 0, 0}, strides[3], last = (cuuint64_t)(d + 7) / 8 * 16;
    cuuint32_t box[4] = {64, 1, 1, 1}, one[4] = {1, 1, 1, 1};
    for (int i = 0; i < 3; ++i) {
        dims[i + 1] = n[o[i]];
        strides[i] = n[o[i]] > 1 ? s[o[i]] : last;
        if (strides[i] % 16 || strides[i] >= (1ull << 40)) return false;
        last = strides[i];
        if (o[i] == 0) box[i + 1] = (cuuint32_t)box_rows;
        out->order[i] = o[i];
    }
    return fn(&out->map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 4, const_cast<void*>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

constexpr int kTileRows = 128, kTileBytes = kTileRows * 128;     // a box: 128 rows of 64 channels
constexpr int kAttendTimeout = 9;

// Wait of a warp for work that is due soon: the hardware's own suspension, no sleep on top of it.
__device__ __forceinline__ void wait_soon(Pipe& pp, int i, uint32_t parity) {
    const uint32_t bar = pipe_bar(pp, i);
    for (unsigned tries = 0; tries < (1u << 22); ++tries) {
        if (mbar_try_wait(bar, parity & 1u)) return;
        if ((tries & 63u) == 63u && pipe_dead(pp)) return;
    }
    *reinterpret_cast<volatile int*>(pp.dead) = 1;
    if (pp.status) atomicCAS(pp.status, 0, kAttendTimeout);
}
// Maxima that keep a NaN
__device__ __forceinline__ float max_nan(float a, float b) {
    float d;
    asm("max.NaN.f32 %0, %1, %2;\n" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;\n" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// Rows from `from` on of a tile of ROWS rows in shared memory (`boxes` of 64 channels) become zero: what lies behind a sequence must not meet a probability of zero.
template <int ROWS> __device__ __forceinline__ void clear_rows(uint32_t tile, int boxes, int from, int lane) {
    for (int b = 0; b < boxes; ++b)
        for (uint32_t at = from * 128 + lane * 16; at < (uint32_t)ROWS * 128; at += 512)
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};\n" ::"r"(tile + b * ROWS * 128 + at), "r"(0) : "memory");
}
// Four steps of 16 of a sum with A in tensor memory (8 columns a step, MID from the second to the third) and B's rows the sum's, by the elected lane
template <int MID> __device__ __forceinline__ void umma_four_ts(uint32_t elected, uint32_t d, uint32_t a, uint64_t b, uint32_t id, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q, t;\n\t.reg .b32 a;\n\t.reg .b64 b;\n\tsetp.ne.b32 q, %5, 0;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.eq.b32 t, 0, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t"
        "add.s32 a, %1, 8;\n\tadd.s64 b, %2, 128;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, t;\n\t"
        "add.s32 a, a, %6;\n\tadd.s64 b, b, 128;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, t;\n\t"
        "add.s32 a, a, 8;\n\tadd.s64 b, b, 128;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, t;\n\t}\n"
        ::"r"(d), "r"(a), "l"(b), "r"(id), "r"(accumulate), "r"(elected), "n"(MID) : "memory");
}
// D = A B with A (128 rows) and B (ROWS) in shared memory, both K-major: `steps` of 16 channels
template <int BOXES, int ROWS> __device__ __forceinline__ void mma_rows(uint32_t elected, uint32_t d, uint32_t a, uint32_t b, uint32_t id, int steps) {
#pragma unroll
    for (int x = 0; x < BOXES; ++x) {
        const uint64_t da = umma_desc_sw128(a + x * kTileBytes), db = umma_desc_sw128(b + x * ROWS * 128);
        if (steps >= 4 * x + 4) umma_four<false, 2, 2>(elected, d, da, db, id, x);
        else
            for (int k = 0; k < steps - 4 * x; ++k) umma_step<false>(elected, d, da + 2 * k, db + 2 * k, id, x | k);
    }
}
// D (+)= P B: P (128 rows, KEYS columns of 16 bits) in tensor memory, EACH of them together every EACH columns; B's KEYS rows are the sum's
template <int BOXES, int KEYS, int EACH> __device__ __forceinline__ void mma_sum(uint32_t elected, uint32_t d, uint32_t p, uint32_t b, uint32_t id, bool add) {
    const uint64_t db = BOXES == 1 ? umma_desc_sw128(b) : desc_mn(b, KEYS * 128);
#pragma unroll
    for (int k = 0; k < KEYS / 64; ++k) umma_four_ts<EACH == 32 ? 24 : 8>(elected, d, p + (EACH == 32 || EACH == 64 ? 64 : 32) * k, db + 512 * k, id, add || k > 0);
}

}  // namespace aa
