// Attention forward over ragged bags (tc_attn_forward) and over a paged cache
// (tc_attn_paged).
#include "tc_attn.h"

namespace tc {
namespace {

using namespace attn;

// One wavefront per (query, head).
template <class T, class CT, bool PAGED>
__global__ __launch_bounds__(kWave) void k_attn_rows(Args a, Source src, tc_rows q, tc_rows out,
                                                     bf16 *out_low, float *lse) {
    const int i = blockIdx.x, h = blockIdx.y;
    const Seq s = seq_at<PAGED>(a, src, blockIdx.z);
    if (i >= s.qn) return;
    const auto kv = KvOf<CT, PAGED>::make(src, s, h / a.group);
    const int64_t t = s.q0 + i;
    RowState st{-INFINITY, 0.0f, {0.0f, 0.0f}};
    const T *qp = static_cast<const T *>(q.data) + t * q.token_stride + h * q.head_stride;
    row_forward(a, kv, load_row(qp, 0, a.dim), h, i + s.shift, 0, limit(a, s, i), st);
    const float inv = st.l == 0.0f ? 0.0f : 1.0f / st.l;
    const Row2 o{st.o.a * inv, st.o.b * inv};
    store_row(static_cast<T *>(out.data) + t * out.token_stride + h * out.head_stride, o, a.dim);
    if (out_low)
        store_row(out_low + (t * a.heads + h) * a.dim,
                  Row2{o.a - float(bf16(o.a)), o.b - float(bf16(o.b))}, a.dim);
    if (lse && (threadIdx.x & 63) == 0)
        lse[h * a.total_q + t] = st.l == 0.0f ? -INFINITY : (st.m + __log2f(st.l)) * kLn2;
}

tc_status forward(const char *fn, const tc_attn &p, const Source &src, int32_t cache_type,
                  tc_rows q, tc_rows out, bf16 *out_low, float *lse, hipStream_t stream) {
    const Args a = make_args(p);
    const dim3 grid(p.max_q, p.num_heads, p.num_seqs);
#define TC_LAUNCH(T, CT, PAGED)                                                                  \
    hipLaunchKernelGGL((k_attn_rows<T, CT, PAGED>), grid, dim3(kWave), 0, stream, a, src, q, out, \
                       out_low, lse)
    if (p.dtype == TC_F32) {
        if (!src.paged)
            TC_LAUNCH(float, float, false);
        else if (cache_type == TC_FP8)
            TC_LAUNCH(float, fp8, true);
        else
            TC_LAUNCH(float, float, true);
    } else {
        if (!src.paged)
            TC_LAUNCH(bf16, bf16, false);
        else if (cache_type == TC_FP8)
            TC_LAUNCH(bf16, fp8, true);
        else
            TC_LAUNCH(bf16, bf16, true);
    }
#undef TC_LAUNCH
    return check_launch(fn);
}

}  // namespace

namespace attn {

tc_status check_attn(const char *fn, const tc_attn *a, bool paged) {
    TC_REQUIRE(a, TC_ERR_INVALID_ARG, "%s: null tc_attn", fn);
    TC_REQUIRE(a->dtype == TC_F32 || a->dtype == TC_BF16, TC_ERR_INVALID_ARG,
               "%s: dtype %d is neither TC_F32 nor TC_BF16", fn, a->dtype);
    TC_REQUIRE(a->num_seqs >= 0 && a->max_q >= 0 && a->max_k >= 0 && a->total_q >= 0 &&
                   (paged || a->total_k >= 0),
               TC_ERR_INVALID_ARG, "%s: negative size", fn);
    TC_REQUIRE(a->num_kv_heads >= 1 && a->num_heads >= 1 && a->num_heads <= 4096 &&
                   a->num_heads % a->num_kv_heads == 0,
               TC_ERR_INVALID_ARG,
               "%s: num_heads %d must be in [1, 4096], a multiple of num_kv_heads %d", fn,
               a->num_heads, a->num_kv_heads);
    TC_REQUIRE(a->head_dim >= 8 && a->head_dim <= kMaxHeadDim && a->head_dim % 8 == 0,
               TC_ERR_UNSUPPORTED, "%s: head_dim %d is not a multiple of 8 in [8, %d]", fn,
               a->head_dim, kMaxHeadDim);
    const int64_t lim = int64_t(1) << 30;
    TC_REQUIRE(a->total_q < lim && (paged || a->total_k < lim) && a->max_q < lim &&
                   a->max_k < lim && a->num_seqs < lim,
               TC_ERR_INVALID_ARG, "%s: queries, keys and sequences must be below 2^30", fn);
    TC_REQUIRE(a->cap >= 0.0f && a->cap <= 3.0e38f, TC_ERR_INVALID_ARG,
               "%s: cap must be finite and not negative", fn);
    TC_REQUIRE(a->scale >= -3.0e38f && a->scale <= 3.0e38f, TC_ERR_INVALID_ARG,
               "%s: scale must be finite", fn);
    TC_REQUIRE(a->causal == 0 || a->causal == 1, TC_ERR_INVALID_ARG, "%s: causal must be 0 or 1", fn);
    TC_REQUIRE(!a->prefix_lens || a->causal, TC_ERR_INVALID_ARG,
               "%s: prefix_lens without causal (every key is visible)", fn);
    if (a->bias_table) {
        TC_REQUIRE(a->bucket_of, TC_ERR_INVALID_ARG, "%s: null pointer: bucket_of", fn);
        TC_REQUIRE(a->reach >= 0 && a->reach <= kMaxReach, TC_ERR_INVALID_ARG,
                   "%s: reach %d is not in [0, %d]", fn, a->reach, kMaxReach);
        TC_REQUIRE(a->num_buckets >= 1 && a->num_buckets <= (1 << 20), TC_ERR_INVALID_ARG,
                   "%s: num_buckets %d is not in [1, 2^20]", fn, a->num_buckets);
    }
    if (a->total_q > 0 && a->num_seqs > 0)
        TC_REQUIRE(a->q_offsets && (paged || a->k_offsets), TC_ERR_INVALID_ARG,
                   "%s: null pointer: offsets", fn);
    TC_REQUIRE(a->total_q == 0 || (a->num_seqs > 0 && a->max_q > 0), TC_ERR_INVALID_ARG,
               "%s: queries, but num_seqs or max_q is 0", fn);
    return TC_OK;
}

}  // namespace attn
}  // namespace tc

using namespace tc;
using namespace tc::attn;

extern "C" size_t tc_attn_workspace_bytes(const tc_attn *a, int32_t paged) { return 0; }

extern "C" tc_status tc_attn_forward(const tc_attn *a, tc_rows q, tc_rows k, tc_rows v, tc_rows out,
                                     void *out_low, float *lse, void *workspace,
                                     size_t workspace_bytes, hipStream_t stream) {
    const char *fn = "tc_attn_forward";
    clear_error();
    tc_status st = check_attn(fn, a, false);
    if (st != TC_OK) return st;
    if (a->total_q == 0) return TC_OK;
    if ((st = check_rows(fn, "q", q, a->dtype, true)) != TC_OK) return st;
    if ((st = check_rows(fn, "k", k, a->dtype, a->total_k > 0)) != TC_OK) return st;
    if ((st = check_rows(fn, "v", v, a->dtype, a->total_k > 0)) != TC_OK) return st;
    if ((st = check_rows(fn, "out", out, a->dtype, true)) != TC_OK) return st;
    TC_REQUIRE(!out_low || a->dtype == TC_BF16, TC_ERR_INVALID_ARG,
               "%s: out_low is for TC_BF16 only", fn);
    TC_REQUIRE(aligned16(out_low), TC_ERR_UNSUPPORTED, "%s: out_low must be 16-byte aligned", fn);
    return forward(fn, *a, dense_source(k, v), a->dtype, q, out, static_cast<bf16 *>(out_low), lse,
                   stream);
}

extern "C" tc_status tc_attn_paged(const tc_attn *a, tc_rows q, const tc_cache *c, tc_rows out,
                                   float *lse, void *workspace, size_t workspace_bytes,
                                   hipStream_t stream) {
    const char *fn = "tc_attn_paged";
    clear_error();
    tc_status st = check_attn(fn, a, true);
    if (st != TC_OK) return st;
    if ((st = check_cache(fn, c, a->dtype)) != TC_OK) return st;
    TC_REQUIRE(c->num_kv_heads == a->num_kv_heads && c->head_dim == a->head_dim,
               TC_ERR_INVALID_ARG, "%s: the cache's num_kv_heads or head_dim differs from a's", fn);
    if (a->total_q == 0) return TC_OK;
    TC_REQUIRE(c->page_table && c->lens, TC_ERR_INVALID_ARG, "%s: null pointer", fn);
    if ((st = check_rows(fn, "q", q, a->dtype, true)) != TC_OK) return st;
    if ((st = check_rows(fn, "out", out, a->dtype, true)) != TC_OK) return st;
    return forward(fn, *a, paged_source(*c), c->dtype, q, out, nullptr, lse, stream);
}
