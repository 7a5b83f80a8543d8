// The paged cache of keys and values: rows appended (tc_cache_write) and read
// back (tc_cache_read), in the rows' own type or in 8 bits (e4m3 values with a
// power-of-two scale per row of one position and key head).
//
// A power of two as scale makes x * 2^-e and stored * 2^e exact, so the one
// rounding is the one to e4m3, and costs no accuracy: e4m3 values carry
// their own exponent, and a scale between two powers would only move the
// row's largest value within the top binade.
//
// Both calls move every element once and compute almost nothing: bound by
// memory (16 x 4096 tokens, 8 heads of 128, from and to bf16: written in 8 bits in
// 109 us, 3.7 TB/s, in bf16 in 109 us, 4.9 TB/s; read in 103 us, 3.9 TB/s, and 113 us,
// 4.7 TB/s). A lane group of dim/8 lanes (a power of two, up to 16) has a row, 8
// elements a lane, so that loads and stores are 16 or 32 bytes and a row's
// maximum is a few shuffles. A workgroup has a run of tokens, kTokens of them at
// a time in each lane group, so that many loads are under way; the sequence of
// the run's first token is found by a search, that of the others by walking on.
#include "tc_attn.h"

namespace tc {
namespace {

using namespace attn;

// Sequence of token t: the last b with offsets[b] <= t (empty sequences
// before it share its offset, and are passed over).
__device__ __forceinline__ int seq_of_token(const int32_t *offsets, int n, int64_t t) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (offsets[mid] <= t)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

__device__ __forceinline__ void load8(const float *p, float *x) {
    const f32x4 a = *reinterpret_cast<const f32x4 *>(p), b = *reinterpret_cast<const f32x4 *>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; i++) x[i] = a[i], x[i + 4] = b[i];
}
__device__ __forceinline__ void load8(const bf16 *p, float *x) {
    const bf16x8 a = *reinterpret_cast<const bf16x8 *>(p);
#pragma unroll
    for (int i = 0; i < 8; i++) x[i] = float(a[i]);
}
__device__ __forceinline__ void store8(float *p, const float *x) {
    *reinterpret_cast<f32x4 *>(p) = f32x4{x[0], x[1], x[2], x[3]};
    *reinterpret_cast<f32x4 *>(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
}
__device__ __forceinline__ void store8(bf16 *p, const float *x) {
    bf16x8 a;
#pragma unroll
    for (int i = 0; i < 8; i++) a[i] = bf16(x[i]);
    *reinterpret_cast<bf16x8 *>(p) = a;
}

// 8-bit form of one row's 8 elements in this lane: LANES lanes have the row.
template <int LANES>
__device__ __forceinline__ u32x2 quantise(const float *x, uint32_t &e_out) {
    // the largest magnitude by its bits: integers order as the floats do,
    // with infinities and NaN above all finite values
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; i++)
        top = max(top, __builtin_bit_cast(uint32_t, x[i]) & 0x7fffffffu);
    // over the row's lanes, without LDS: neighbours, pairs, then mirrored halves
    // and rows of 16
    if (LANES > 1) top = max(top, uint32_t(__builtin_amdgcn_mov_dpp(int(top), 0xb1, 0xf, 0xf, true)));
    if (LANES > 2) top = max(top, uint32_t(__builtin_amdgcn_mov_dpp(int(top), 0x4e, 0xf, 0xf, true)));
    if (LANES > 4) top = max(top, uint32_t(__builtin_amdgcn_mov_dpp(int(top), 0x141, 0xf, 0xf, true)));
    if (LANES > 8) top = max(top, uint32_t(__builtin_amdgcn_mov_dpp(int(top), 0x140, 0xf, 0xf, true)));
    if (top >= 0x7f800000u) {
        e_out = 255;
        return u32x2{0x7f7f7f7fu, 0x7f7f7f7fu};
    }
    // amax = (1.f) * 2^E <= 448 * 2^e = 1.75 * 2^(e+8): e = E - 8, one more
    // if the fraction passes 0.75. Subnormals count as E = -127: e is -126.
    int e = int(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
    e = top == 0 ? 0 : max(e, -126);
    e_out = uint32_t(e + 127);
    // x * 2^-e in two exact factors (2^-e itself may pass the range)
    const float s = exp_scale(uint32_t(127 - e / 2)), s2 = exp_scale(uint32_t(127 - (e - e / 2)));
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; i++) y[i] = x[i] * s * s2;
    u32x2 r;
    r[0] = uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false));
    r[0] = uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], int(r[0]), true));
    r[1] = uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], 0, false));
    r[1] = uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], int(r[1]), true));
    return r;
}

__device__ __forceinline__ void dequantise(u32x2 r, uint32_t e, float *x) {
    const float s = exp_scale(e < 1 ? 1 : e > 254 ? 254 : e);
#pragma unroll
    for (int w = 0; w < 2; w++) {
        const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(int(r[w]), false);
        const f32x2 b = __builtin_amdgcn_cvt_pk_f32_fp8(int(r[w]), true);
        x[4 * w] = a[0] * s;
        x[4 * w + 1] = a[1] * s;
        x[4 * w + 2] = b[0] * s;
        x[4 * w + 3] = b[1] * s;
    }
}

constexpr int kTokens = 4;

// Read in place of rows that have no place: loads under a condition would wait
// for one another.
__device__ __attribute__((aligned(16))) const uint32_t kNoRow[8] = {};

// Lane group r of a workgroup has row r % per of every (256 / LANES / per)-th
// token of the run (per: a token's rows, k and v of every head), or where a token
// has more rows than there are groups, every such row of each token.
template <class T, bool FP8, bool WRITE, int LANES>
__global__ __launch_bounds__(kBlock) void k_cache_rows(tc_cache c, Divider page_size, int num_seqs,
                                                       const int32_t *__restrict__ offsets,
                                                       int32_t total, int32_t run, tc_rows k,
                                                       tc_rows v) {
    constexpr int GROUPS = kBlock / LANES;
    const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
    const int per = 2 * c.num_kv_heads;
    const int side = max(GROUPS / per, 1);  // tokens side by side
    const int first = blockIdx.x * run, end = min(first + run, total);
    const bool mine = lane * 8 < c.head_dim;
    if (group / min(per, GROUPS) >= side) return;  // a remainder of groups
    const int64_t places = int64_t(c.max_pages) * c.page_size;
    int b = seq_of_token(offsets, num_seqs, first);
    int next = offsets[b + 1];
    for (int t0 = first + (per < GROUPS ? group / per : 0); t0 < end; t0 += side * kTokens) {
        bool in[kTokens], held[kTokens];
        int64_t data[kTokens], slot[kTokens];
#pragma unroll
        for (int n = 0; n < kTokens; n++) {
            const int t = t0 + n * side;
            in[n] = t < end;
            held[n] = false;
            data[n] = slot[n] = 0;
            if (!in[n]) continue;
            while (t >= next && b + 1 < num_seqs) {
                b++;
                next = offsets[b + 1];
            }
            const int64_t pos = int64_t(c.lens[b]) - (next - t);
            held[n] = pos >= 0 && pos < places;
            if (!held[n]) continue;
            const int p = divide(int(pos), page_size), s = int(pos) - p * c.page_size;
            const int64_t page = c.page_table[int64_t(b) * c.max_pages + p];
            data[n] = page * c.page_stride + s * c.slot_stride + lane * 8;
            slot[n] = (page * c.page_size + s) * c.num_kv_heads;
        }
        for (int which = group % min(per, GROUPS); which < per; which += GROUPS) {
            const int h = which >> 1;
            const bool is_v = which & 1;
            const tc_rows &rw = is_v ? v : k;
            T *row = static_cast<T *>(rw.data) + h * rw.head_stride + (mine ? lane * 8 : 0);
            void *base = is_v ? c.v : c.k;
            uint8_t *exps = is_v ? c.v_exp : c.k_exp;
            float x[kTokens][8];
            if (WRITE) {
#pragma unroll
                for (int n = 0; n < kTokens; n++)
                    load8(row + int64_t(min(t0 + n * side, end - 1)) * rw.token_stride, x[n]);
                if (FP8) {
#pragma unroll
                    for (int n = 0; n < kTokens; n++) {
#pragma unroll
                        for (int e = 0; e < 8; e++) x[n][e] = mine ? x[n][e] : 0.0f;
                        uint32_t e;
                        const u32x2 q = quantise<LANES>(x[n], e);
                        if (!held[n]) continue;
                        const int64_t at = data[n] + h * c.head_stride;
                        if (mine) *reinterpret_cast<u32x2 *>(static_cast<uint8_t *>(base) + at) = q;
                        if (lane == 0) exps[slot[n] + h] = uint8_t(e);
                    }
                } else {
#pragma unroll
                    for (int n = 0; n < kTokens; n++)
                        if (held[n] && mine)
                            store8(static_cast<T *>(base) + data[n] + h * c.head_stride, x[n]);
                }
            } else {
                if (FP8) {
                    u32x2 q[kTokens];
                    uint32_t e[kTokens];
#pragma unroll
                    for (int n = 0; n < kTokens; n++) {
                        const auto *none = reinterpret_cast<const uint8_t *>(kNoRow);
                        const int64_t at = data[n] + h * c.head_stride;
                        q[n] = *reinterpret_cast<const u32x2 *>(
                            held[n] && mine ? static_cast<const uint8_t *>(base) + at : none);
                        e[n] = *(held[n] ? exps + slot[n] + h : none);
                    }
#pragma unroll
                    for (int n = 0; n < kTokens; n++) dequantise(q[n], e[n], x[n]);
                } else {
#pragma unroll
                    for (int n = 0; n < kTokens; n++)
                        load8(held[n] && mine
                                  ? static_cast<const T *>(base) + data[n] + h * c.head_stride
                                  : reinterpret_cast<const T *>(kNoRow),
                              x[n]);
                }
#pragma unroll
                for (int n = 0; n < kTokens; n++)
                    if (in[n] && mine)
                        store8(row + int64_t(t0 + n * side) * rw.token_stride, x[n]);
            }
        }
    }
}

template <class T, bool FP8, bool WRITE>
void launch_rows(const tc_cache &c, int num_seqs, const int32_t *offsets, int64_t total, tc_rows k,
                 tc_rows v, hipStream_t stream) {
    int lanes = 1;
    while (lanes * 8 < c.head_dim) lanes *= 2;
    // a run is what a workgroup has under way at a time, or more so that a few
    // workgroups a CU have them all
    const int groups = kBlock / lanes, per = 2 * c.num_kv_heads;
    const int64_t once = int64_t(groups / per > 1 ? groups / per : 1) * kTokens;
    const int64_t most = int64_t(device_cus()) * 16;
    int64_t run = (total + most - 1) / most;
    run = (run + once - 1) / once * once;
    if (total < 2 * most) run = once / kTokens;  // few tokens: one in each lane group
    const dim3 grid(unsigned((total + run - 1) / run));
    const Divider d = make_divider(uint32_t(c.page_size));
#define TC_LAUNCH(L)                                                                               \
    case L:                                                                                        \
        hipLaunchKernelGGL((k_cache_rows<T, FP8, WRITE, L>), grid, dim3(kBlock), 0, stream, c, d,  \
                           num_seqs, offsets, int32_t(total), int32_t(run), k, v);                 \
        break;
    switch (lanes) {
        TC_LAUNCH(1) TC_LAUNCH(2) TC_LAUNCH(4) TC_LAUNCH(8) TC_LAUNCH(16)
    }
#undef TC_LAUNCH
}

tc_status cache_call(const char *fn, bool write, const tc_cache *c, int32_t dtype, int32_t num_seqs,
                     const int32_t *offsets, int64_t total, tc_rows k, tc_rows v,
                     hipStream_t stream) {
    clear_error();
    TC_REQUIRE(dtype == TC_F32 || dtype == TC_BF16, TC_ERR_INVALID_ARG,
               "%s: dtype %d is neither TC_F32 nor TC_BF16", fn, dtype);
    const tc_status st = check_cache(fn, c, dtype);
    if (st != TC_OK) return st;
    TC_REQUIRE(num_seqs >= 0 && total >= 0 && total < (int64_t(1) << 30), TC_ERR_INVALID_ARG,
               "%s: num_seqs and total must not be negative, total below 2^30", fn);
    if (total == 0) return TC_OK;
    TC_REQUIRE(num_seqs > 0, TC_ERR_INVALID_ARG, "%s: rows but no sequences", fn);
    TC_REQUIRE(offsets && c->page_table && c->lens, TC_ERR_INVALID_ARG, "%s: null pointer", fn);
    tc_status rs = check_rows(fn, "k", k, dtype, true);
    if (rs != TC_OK) return rs;
    rs = check_rows(fn, "v", v, dtype, true);
    if (rs != TC_OK) return rs;
    const bool q8 = c->dtype == TC_FP8;
#define TC_CACHE(T, FP8)                                                                \
    (write ? launch_rows<T, FP8, true>(*c, num_seqs, offsets, total, k, v, stream)      \
           : launch_rows<T, FP8, false>(*c, num_seqs, offsets, total, k, v, stream))
    if (dtype == TC_F32)
        q8 ? TC_CACHE(float, true) : TC_CACHE(float, false);
    else
        q8 ? TC_CACHE(bf16, true) : TC_CACHE(bf16, false);
#undef TC_CACHE
    return check_launch(write ? "tc_cache_write: k_cache_rows" : "tc_cache_read: k_cache_rows");
}

}  // namespace

namespace attn {

tc_status check_rows(const char *fn, const char *name, const tc_rows &r, int32_t dtype,
                     bool required) {
    if (!r.data) {
        TC_REQUIRE(!required, TC_ERR_INVALID_ARG, "%s: null pointer: %s", fn, name);
        return TC_OK;
    }
    const int64_t unit = dtype == TC_F32 ? 4 : 8;  // elements of 16 bytes
    TC_REQUIRE(r.token_stride >= 0 && r.head_stride >= 0, TC_ERR_INVALID_ARG,
               "%s: %s has a negative stride", fn, name);
    // (a tile's rows are found by 32-bit offsets from its first)
    TC_REQUIRE(r.token_stride < (int64_t(1) << 24), TC_ERR_UNSUPPORTED,
               "%s: rows of %s are 2^24 elements or more apart", fn, name);
    TC_REQUIRE(aligned16(r.data) && r.token_stride % unit == 0 && r.head_stride % unit == 0,
               TC_ERR_UNSUPPORTED, "%s: rows of %s must start at multiples of 16 bytes", fn, name);
    return TC_OK;
}

tc_status check_cache(const char *fn, const tc_cache *c, int32_t dtype) {
    TC_REQUIRE(c, TC_ERR_INVALID_ARG, "%s: null cache", fn);
    TC_REQUIRE(c->dtype == TC_FP8 || c->dtype == dtype, TC_ERR_UNSUPPORTED,
               "%s: a cache of dtype %d takes rows of that type only, not %d", fn, c->dtype, dtype);
    TC_REQUIRE(c->page_size >= 1 && c->page_size <= (1 << 20), TC_ERR_INVALID_ARG,
               "%s: page_size %d is not in [1, 2^20]", fn, c->page_size);
    TC_REQUIRE(c->num_kv_heads >= 1 && c->num_kv_heads <= (1 << 16), TC_ERR_INVALID_ARG,
               "%s: num_kv_heads %d is not in [1, 65536]", fn, c->num_kv_heads);
    TC_REQUIRE(c->head_dim >= 8 && c->head_dim <= kMaxHeadDim && c->head_dim % 8 == 0,
               TC_ERR_UNSUPPORTED, "%s: head_dim %d is not a multiple of 8 in [8, %d]", fn,
               c->head_dim, kMaxHeadDim);
    TC_REQUIRE(c->max_pages >= 0, TC_ERR_INVALID_ARG, "%s: max_pages is negative", fn);
    TC_REQUIRE(int64_t(c->max_pages) * c->page_size < (int64_t(1) << 31), TC_ERR_INVALID_ARG,
               "%s: max_pages * page_size must be below 2^31", fn);
    TC_REQUIRE(c->k && c->v, TC_ERR_INVALID_ARG, "%s: null pointer: the cache's k or v", fn);
    TC_REQUIRE(c->dtype != TC_FP8 || (c->k_exp && c->v_exp), TC_ERR_INVALID_ARG,
               "%s: null pointer: the exponents of a TC_FP8 cache", fn);
    TC_REQUIRE(c->page_stride >= 0 && c->slot_stride >= 0 && c->head_stride >= 0,
               TC_ERR_INVALID_ARG, "%s: the cache has a negative stride", fn);
    const int64_t unit = c->dtype == TC_F32 ? 4 : 8;
    const uintptr_t mask = c->dtype == TC_FP8 ? 7u : 15u;
    TC_REQUIRE(((reinterpret_cast<uintptr_t>(c->k) | reinterpret_cast<uintptr_t>(c->v)) & mask) == 0 &&
                   c->page_stride % unit == 0 && c->slot_stride % unit == 0 &&
                   c->head_stride % unit == 0,
               TC_ERR_UNSUPPORTED, "%s: rows of the cache must start at multiples of %d bytes", fn,
               int(mask) + 1);
    return TC_OK;
}

}  // namespace attn
}  // namespace tc

extern "C" tc_status tc_cache_write(const tc_cache *c, int32_t dtype, int32_t num_seqs,
                                    const int32_t *offsets, int64_t total, tc_rows k, tc_rows v,
                                    hipStream_t stream) {
    return tc::cache_call("tc_cache_write", true, c, dtype, num_seqs, offsets, total, k, v, stream);
}

extern "C" tc_status tc_cache_read(const tc_cache *c, int32_t dtype, int32_t num_seqs,
                                   const int32_t *offsets, int64_t total, tc_rows k, tc_rows v,
                                   hipStream_t stream) {
    return tc::cache_call("tc_cache_read", false, c, dtype, num_seqs, offsets, total, k, v, stream);
}
