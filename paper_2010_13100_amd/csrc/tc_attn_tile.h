// Matrix products of the attention kernels on 32x32 blocks, and the LDS tiles
// they read.
//
// Scores are formed transposed: a block S^T has keys as rows and queries as
// columns, so that a lane holds 16 keys of one query (the result layout of
// the 32x32 matrix instructions: register r of lane l is row 8*(r/4) +
// 4*(l/32) + r%4, column l%32). Row statistics are then sums within a lane
// and one exchange between the wavefront's halves, and the probabilities are
// already the right operand of the next product (out^T = V^T P^T): its sum
// runs over keys in any order, so the left operand is read with the keys in
// the order in which the lane holds them. Probabilities never pass through
// LDS.
//
// An operand of a product over 16 values is 8 values a lane: row (or column)
// l%32, values 8*(l/32) .. +7 of the 16. fp32 uses the same operands with
// eight 32x32x2 instructions.
//
// A tile in LDS has rows of DH elements in chunks of 8; chunk c of row r is at
// place c ^ (r & 7), so that reads of one chunk from 32 rows and transposed
// reads of 32 columns from 8 rows spread over the banks.
#pragma once

#include "tc_attn.h"

namespace tc {
namespace attn {

template <class T>
using V8 = typename El<T>::v8;

__device__ __forceinline__ f32x16 mma(bf16x8 a, bf16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(f32x8 a, f32x8 b, f32x16 c) {
#pragma unroll
    for (int i = 0; i < 8; i++) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
    return c;
}

__device__ __forceinline__ f32x16 zero16() {
    f32x16 z;
#pragma unroll
    for (int r = 0; r < 16; r++) z[r] = 0.0f;
    return z;
}

// Row of register r in a half's share of a block (add 4*half).
__device__ __forceinline__ constexpr int reg_row(int r) { return 8 * (r >> 2) + (r & 3); }

// Registers 8*s .. 8*s + 7 of a block as an operand.
__device__ __forceinline__ void pack(const f32x16 &x, int s, bf16x8 &f) {
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const f32x2 y = {x[8 * s + 2 * i], x[8 * s + 2 * i + 1]};
        const bf16x2 p = __builtin_convertvector(y, bf16x2);
        f[2 * i] = p[0];
        f[2 * i + 1] = p[1];
    }
}
__device__ __forceinline__ void pack(const f32x16 &x, int s, f32x8 &f) {
#pragma unroll
    for (int i = 0; i < 8; i++) f[i] = x[8 * s + i];
}

// --- 8 elements from memory ---------------------------------------------------

template <class CT>
struct Raw;  // 8 elements as they lie in memory
template <>
struct Raw<float> {
    f32x8 x;
};
template <>
struct Raw<bf16> {
    bf16x8 x;
};
template <>
struct Raw<fp8> {
    u32x2 x;
    uint32_t e;
};

__device__ __forceinline__ Raw<float> load_raw(const float *p, uint32_t) {
    const f32x4 a = *reinterpret_cast<const f32x4 *>(p), b = *reinterpret_cast<const f32x4 *>(p + 4);
    return {__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7)};
}
__device__ __forceinline__ Raw<bf16> load_raw(const bf16 *p, uint32_t) {
    return {*reinterpret_cast<const bf16x8 *>(p)};
}
__device__ __forceinline__ Raw<fp8> load_raw(const fp8 *p, uint32_t e) {
    return {*reinterpret_cast<const u32x2 *>(p), e};
}
template <class CT>
__device__ __forceinline__ Raw<CT> zero_raw();
template <>
__device__ __forceinline__ Raw<float> zero_raw<float>() {
    return {f32x8{0, 0, 0, 0, 0, 0, 0, 0}};
}
template <>
__device__ __forceinline__ Raw<bf16> zero_raw<bf16>() {
    return {__builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0})};
}
template <>
__device__ __forceinline__ Raw<fp8> zero_raw<fp8>() {
    return {u32x2{0, 0}, 127};
}

// As elements of the products. 8-bit values times a power of two are exact.
__device__ __forceinline__ void expand(const Raw<float> &r, f32x8 &x) { x = r.x; }
__device__ __forceinline__ void expand(const Raw<bf16> &r, bf16x8 &x) { x = r.x; }
__device__ __forceinline__ void expand(const Raw<fp8> &r, f32x8 &x) {
    const float s = exp_scale(r.e);
#pragma unroll
    for (int w = 0; w < 2; w++) {
        const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(int(r.x[w]), false);
        const f32x2 b = __builtin_amdgcn_cvt_pk_f32_fp8(int(r.x[w]), true);
        x[4 * w] = a[0] * s;
        x[4 * w + 1] = a[1] * s;
        x[4 * w + 2] = b[0] * s;
        x[4 * w + 3] = b[1] * s;
    }
}
__device__ __forceinline__ void expand(const Raw<fp8> &r, bf16x8 &x) {
    const float s = exp_scale(r.e);
#pragma unroll
    for (int w = 0; w < 2; w++) {
        const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(r.x[w], s, false);
        const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(r.x[w], s, true);
        x[4 * w] = a[0];
        x[4 * w + 1] = a[1];
        x[4 * w + 2] = b[0];
        x[4 * w + 3] = b[1];
    }
}

// Sets NaN and infinities among the 8 elements to zero; true if there were any.
//
// A tile that some rows of a block see and others do not is cleaned by this
// before it enters a product: 0 * NaN would reach the rows that do not see the
// value. Rows that do see it are then computed again, one by one, from memory.
__device__ __forceinline__ bool clean(f32x8 &x) {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const bool b = (__builtin_bit_cast(uint32_t, float(x[i])) & 0x7f800000u) == 0x7f800000u;
        x[i] = b ? 0.0f : x[i];
        bad |= b;
    }
    return bad;
}
__device__ __forceinline__ bool clean(bf16x8 &x) {
    u32x4 w = __builtin_bit_cast(u32x4, x);
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const bool lo = (w[i] & 0x7f80u) == 0x7f80u, hi = (w[i] & 0x7f800000u) == 0x7f800000u;
        w[i] = (lo ? 0u : w[i] & 0xffffu) | (hi ? 0u : w[i] & 0xffff0000u);
        bad |= lo | hi;
    }
    x = __builtin_bit_cast(bf16x8, w);
    return bad;
}

// --- tiles -------------------------------------------------------------------

template <class T, int DH>
struct Tile {
    static __device__ __forceinline__ int at(int row, int chunk) {
        return row * DH + ((chunk ^ (row & 7)) << 3);
    }
    static __device__ __forceinline__ void put(T *t, int row, int chunk, const V8<T> &x) {
        *reinterpret_cast<V8<T> *>(t + at(row, chunk)) = x;
    }
    // Left operand: rows r0 .. r0+31, values 16*ks .. +15 of each.
    static __device__ __forceinline__ V8<T> rows(const T *t, int r0, int ks) {
        const int l = threadIdx.x & 63;
        return *reinterpret_cast<const V8<T> *>(t + at(r0 + (l & 31), 2 * ks + (l >> 5)));
    }
    // Left operand of the transposed tile: columns 32*db .. +31 as rows; its 16
    // values are the tile's rows r0 .. r0+15 in the order of a block's
    // registers. r0 is a multiple of 16.
    static __device__ __forceinline__ V8<T> cols(const T *t, int r0, int db) {
        const int l = threadIdx.x & 63, half = l >> 5;
        V8<T> x;
        if constexpr (sizeof(T) == 2) {
            // 16 lanes read a 4 x 16 block of 16-bit values transposed: lane j
            // gives the address of row j/4, values 4*(j%4) .. +3, and gets column j
            const int j = l & 15, row = 4 * half + (j >> 2);
            const int d = db * 32 + ((l >> 4) & 1) * 16 + (j & 3) * 4;
            const T *p = t + r0 * DH + at(row, d >> 3) + (d & 7);
            typedef __attribute__((address_space(3))) s16x4 lds4;
            const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(p));
            const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(p + 8 * DH));
            x = __builtin_bit_cast(V8<T>, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            const int d = db * 32 + (l & 31);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const int row = 4 * half + (i < 4 ? i : i + 4);
                x[i] = t[r0 * DH + at(row, d >> 3) + (d & 7)];
            }
        }
        return x;
    }
};

// Right operand from a row in memory: columns are rows of 8-element chunks.
template <class T>
__device__ __forceinline__ V8<T> chunk_of(const T *row, int chunk, int dim) {
    V8<T> x;
    expand(chunk * 8 < dim ? load_raw(row + chunk * 8, 0) : zero_raw<T>(), x);
    return x;
}

// Writes a transposed block (rows are elements 32*db .. +31 of this lane's
// row) times f.
__device__ __forceinline__ void store4(float *p, const float *x) {
    *reinterpret_cast<f32x4 *>(p) = f32x4{x[0], x[1], x[2], x[3]};
}
__device__ __forceinline__ void store4(bf16 *p, const float *x) {
    bf16x4 y;
#pragma unroll
    for (int i = 0; i < 4; i++) y[i] = bf16(x[i]);
    *reinterpret_cast<bf16x4 *>(p) = y;
}
template <class T>
__device__ __forceinline__ void store_block(T *row, const f32x16 &x, float f, int db, int dim) {
    const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int g = 0; g < 4; g++) {
        const int d = db * 32 + 8 * g + 4 * half;
        const float y[4] = {x[4 * g] * f, x[4 * g + 1] * f, x[4 * g + 2] * f, x[4 * g + 3] * f};
        if (d < dim) store4(row + d, y);
    }
}

// --- tiles of sequences -------------------------------------------------------

// Tiles of `bm` rows are numbered without a count of them: sequence b's first
// tile has number offsets[b]/bm + b, which leaves room for ceil(rows/bm) of
// them before the next one's. total/bm + num_seqs numbers cover all; a number
// between a sequence's last tile and the next one's first has no rows.
inline int64_t tile_slots(int64_t total, int64_t num_seqs, int bm) { return total / bm + num_seqs; }

// The last b with first(b) <= x, for a non-decreasing `first` with first(0) <=
// x: a search of 64 probes a step by the whole wavefront (uniform result).
template <class F>
__device__ __forceinline__ int last_at_most(int n, int64_t x, F first) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int step = (hi - lo + kWave - 1) / kWave;
        const int i = lo + int(threadIdx.x & 63) * step;
        const int k = __popcll(__ballot(i < hi && first(i) <= x));
        lo += (max(k, 1) - 1) * step;
        hi = min(hi, lo + step);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

// The sequence of tile number `slot`; `tile` is its tile within the sequence.
__device__ __forceinline__ int seq_of_slot(const int32_t *off, int num_seqs, int slot, int bm,
                                           int &tile) {
    auto first = [&](int b) { return int64_t(uint32_t(off[b]) / uint32_t(bm)) + b; };
    const int b = last_at_most(num_seqs, slot, first);
    tile = slot - int(first(b));
    return b;
}

// --- the distance bias in LDS ---------------------------------------------------
//
// Entry i is the bias (times log2 e) of distance i - reach - 63, cut to the
// reach: a 32x32 block that is not wholly past the reach on one side has
// distances within reach + 62, and is looked up without a cut.
constexpr int kBiasPad = 63;
inline int bias_entries(int reach) { return 2 * (reach + kBiasPad) + 1; }

__device__ __forceinline__ void load_bias(const Args &a, int h, float *lds) {
    const int n = 2 * (a.reach + kBiasPad) + 1;
    for (int i = threadIdx.x; i < n; i += blockDim.x)
        lds[i] = log2_bias(a, h, i - a.reach - kBiasPad);
}

// Adds the bias to a block of scores whose distance at (row 0, column 0) is
// `rel`: this lane's registers are keys 4*half + reg_row(r), query col.
__device__ __forceinline__ void add_bias(const Args &a, const float *lds, int rel, f32x16 &x) {
    const int l = threadIdx.x & 63;
    if (rel + 31 <= -a.reach || rel - 31 >= a.reach) {
        const float c = lds[rel < 0 ? 0 : 2 * (a.reach + kBiasPad)];
#pragma unroll
        for (int r = 0; r < 16; r++) x[r] += c;
        return;
    }
    const float *p = lds + (rel + 4 * (l >> 5) - (l & 31) + a.reach + kBiasPad);
#pragma unroll
    for (int r = 0; r < 16; r++) x[r] += p[reg_row(r)];
}

// The same for a block whose rows are queries: this lane's registers are
// queries 4*half + reg_row(r), key col.
__device__ __forceinline__ void add_bias_queries(const Args &a, const float *lds, int rel,
                                                 f32x16 &x) {
    const int l = threadIdx.x & 63;
    if (rel + 31 <= -a.reach || rel - 31 >= a.reach) {
        const float c = lds[rel < 0 ? 0 : 2 * (a.reach + kBiasPad)];
#pragma unroll
        for (int r = 0; r < 16; r++) x[r] += c;
        return;
    }
    const float *p = lds + (rel - 4 * (l >> 5) + (l & 31) + a.reach + kBiasPad);
#pragma unroll
    for (int r = 0; r < 16; r++) x[r] += p[-reg_row(r)];
}

}  // namespace attn
}  // namespace tc
