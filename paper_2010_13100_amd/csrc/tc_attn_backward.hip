// Attention backward over ragged bags (tc_attn_backward), with the gradient
// of the learned distance bias.
#include "tc_attn.h"

namespace tc {
namespace {

using namespace attn;

// Workgroups per head of the query-side kernel: the number of partial sums of
// a distance's bias gradient.
constexpr int kBiasParts = 256;

struct Grads {
    tc_rows q, k, v, out, grad_out, dq, dk, dv;
    const bf16 *out_low;
    const float *lse;
    float *delta;      // [heads x total_q]: <grad_out, out> of every row
    float *bias_part;  // [heads x parts x (2*reach + 1)], or nullptr
};

// One pair (query, key): p, and ds = p * (dp - delta) with respect to s.
__device__ __forceinline__ void pair_grad(const Args &a, float z, float bias, float lse2, float dp,
                                          float delta, float &p, float &ds, float &g) {
    float t = 0.0f, x = a.c1 * z;
    if (a.capped) {
        t = tanh_of(x);
        x = a.c2 * t;
    }
    p = exp2_fast(x + bias - lse2);
    ds = p * (dp - delta);
    g = ds * a.scale;
    if (a.capped) g *= 1.0f - t * t;
}

template <class T>
__device__ __forceinline__ Row2 row_at(const tc_rows &r, int64_t t, int h, int dim) {
    return load_row(static_cast<const T *>(r.data) + t * r.token_stride + h * r.head_stride, 0, dim);
}
template <class T>
__device__ __forceinline__ void put_row(const tc_rows &r, int64_t t, int h, int dim, Row2 x) {
    store_row(static_cast<T *>(r.data) + t * r.token_stride + h * r.head_stride, x, dim);
}

template <class T>
__device__ float row_delta(const Args &a, const Grads &g, int64_t t, int h, Row2 go) {
    Row2 o = row_at<T>(g.out, t, h, a.dim);
    if (g.out_low) {
        const Row2 r = load_row(g.out_low + (t * a.heads + h) * a.dim, 0, a.dim);
        o.a += r.a;
        o.b += r.b;
    }
    return dot(go, o);
}

// Gradient of one query's row; bias terms into dist[2*reach + 1].
template <class T>
__device__ void row_dq(const Args &a, const Grads &g, const Seq &s, int i, int h, float *dist) {
    const int64_t t = s.q0 + i;
    const int kvh = h / a.group;
    const Row2 q = row_at<T>(g.q, t, h, a.dim), go = row_at<T>(g.grad_out, t, h, a.dim);
    const float delta = row_delta<T>(a, g, t, h, go);
    const float lse2 = g.lse[h * a.total_q + t] * kLog2e;
    if ((threadIdx.x & 63) == 0) g.delta[h * a.total_q + t] = delta;
    Row2 dq{0.0f, 0.0f};
    const int n = limit(a, s, i), pos = i + s.shift;
    for (int j = 0; j < n; j++) {
        const Row2 k = row_at<T>(g.k, s.k0 + j, kvh, a.dim), v = row_at<T>(g.v, s.k0 + j, kvh, a.dim);
        float p, ds, gs;
        pair_grad(a, dot(q, k), a.table ? log2_bias(a, h, j - pos) : 0.0f, lse2, dot(go, v), delta,
                  p, ds, gs);
        dq.a += gs * k.a;
        dq.b += gs * k.b;
        if (dist && (threadIdx.x & 63) == 0)
            dist[min(max(j - pos, -a.reach), a.reach) + a.reach] += ds;
    }
    put_row<T>(g.dq, t, h, a.dim, dq);
}

// Gradients of one key's rows, over the queries and heads that see it.
template <class T>
__device__ void row_dkv(const Args &a, const Grads &g, const Seq &s, int j, int kvh) {
    const Row2 k = row_at<T>(g.k, s.k0 + j, kvh, a.dim), v = row_at<T>(g.v, s.k0 + j, kvh, a.dim);
    Row2 dk{0.0f, 0.0f}, dv{0.0f, 0.0f};
    for (int h = kvh * a.group; h < (kvh + 1) * a.group; h++) {
        for (int i = first_query(a, s, j); i < s.qn; i++) {
            const int64_t t = s.q0 + i;
            const Row2 q = row_at<T>(g.q, t, h, a.dim), go = row_at<T>(g.grad_out, t, h, a.dim);
            float p, ds, gs;
            pair_grad(a, dot(q, k), a.table ? log2_bias(a, h, j - i - s.shift) : 0.0f,
                      g.lse[h * a.total_q + t] * kLog2e, dot(go, v), g.delta[h * a.total_q + t], p,
                      ds, gs);
            dk.a += gs * q.a;
            dk.b += gs * q.b;
            dv.a += p * go.a;
            dv.b += p * go.b;
        }
    }
    put_row<T>(g.dk, s.k0 + j, kvh, a.dim, dk);
    put_row<T>(g.dv, s.k0 + j, kvh, a.dim, dv);
}

template <class T>
__global__ __launch_bounds__(kWave) void k_attn_dq_rows(Args a, Grads g, int max_q) {
    __shared__ float dist[2 * kMaxReach + 1];
    const int h = blockIdx.y, width = 2 * a.reach + 1;
    for (int d = threadIdx.x; d < width; d += kWave) dist[d] = 0.0f;
    for (int64_t w = blockIdx.x; w < int64_t(max_q) * a.num_seqs; w += gridDim.x) {
        const Seq s = seq_of(a, int(w / max_q), -1);
        const int i = int(w % max_q);
        if (i < s.qn) row_dq<T>(a, g, s, i, h, g.bias_part ? dist : nullptr);
    }
    if (g.bias_part)
        for (int d = threadIdx.x; d < width; d += kWave)
            g.bias_part[(int64_t(h) * gridDim.x + blockIdx.x) * width + d] = dist[d];
}

template <class T>
__global__ __launch_bounds__(kWave) void k_attn_dkv_rows(Args a, Grads g) {
    const Seq s = seq_of(a, blockIdx.z, -1);
    if (int(blockIdx.x) < s.kn) row_dkv<T>(a, g, s, blockIdx.x, blockIdx.y);
}

// Sums the parts of every (head, distance), in order, into part 0.
__global__ __launch_bounds__(kBlock) void k_bias_parts(float *part, int parts, int width) {
    __shared__ float sum[4][kWave];
    const int d = blockIdx.x * kWave + threadIdx.x % kWave, w = threadIdx.x / kWave;
    float *p = part + int64_t(blockIdx.y) * parts * width;
    float x = 0.0f;
    if (d < width)
        for (int i = w; i < parts; i += 4) x += p[int64_t(i) * width + d];
    sum[w][threadIdx.x % kWave] = x;
    __syncthreads();
    if (w == 0 && d < width) {
        const int l = threadIdx.x;
        p[d] = (sum[0][l] + sum[1][l]) + (sum[2][l] + sum[3][l]);
    }
}

// Sums the distances of every (bucket, head), in order: a wavefront each.
__global__ __launch_bounds__(kWave) void k_bias_buckets(Args a, const float *part, int parts,
                                                        int width, float *grad) {
    const float *p = part + int64_t(blockIdx.y) * parts * width;
    float x = 0.0f;
    for (int d = threadIdx.x; d < width; d += kWave)
        if (a.bucket_of[d] == int(blockIdx.x)) x += p[d];
    x = wave_sum(x);
    if (threadIdx.x == 0) grad[int64_t(blockIdx.x) * a.heads + blockIdx.y] = x;
}

template <class T>
void backward(const tc_attn &p, const Args &a, const Grads &g, float *grad_bias,
              hipStream_t stream) {
    if (p.total_q > 0)
        hipLaunchKernelGGL((k_attn_dq_rows<T>), dim3(kBiasParts, a.heads), dim3(kWave), 0, stream,
                           a, g, p.max_q);
    if (p.total_k > 0)
        hipLaunchKernelGGL((k_attn_dkv_rows<T>), dim3(p.max_k, a.kv_heads, a.num_seqs),
                           dim3(kWave), 0, stream, a, g);
    if (grad_bias) {
        const int width = 2 * a.reach + 1;
        hipLaunchKernelGGL(k_bias_parts, dim3((width + 63) / 64, a.heads), dim3(kBlock), 0, stream,
                           g.bias_part, kBiasParts, width);
        hipLaunchKernelGGL(k_bias_buckets, dim3(p.num_buckets, a.heads), dim3(kWave), 0, stream, a,
                           g.bias_part, kBiasParts, width, grad_bias);
    }
}

size_t up256(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace
}  // namespace tc

using namespace tc;
using namespace tc::attn;

extern "C" size_t tc_attn_backward_workspace_bytes(const tc_attn *a) {
    if (!a || a->total_q <= 0 || a->num_heads <= 0) return 0;
    const size_t delta = up256(sizeof(float) * size_t(a->num_heads) * size_t(a->total_q));
    const size_t bias = a->bias_table ? up256(sizeof(float) * size_t(a->num_heads) * kBiasParts *
                                              size_t(2 * a->reach + 1))
                                      : 0;
    return delta + bias;
}

extern "C" tc_status tc_attn_backward(const tc_attn *a, tc_rows q, tc_rows k, tc_rows v,
                                      tc_rows out, const void *out_low, const float *lse,
                                      tc_rows grad_out, tc_rows grad_q, tc_rows grad_k,
                                      tc_rows grad_v, float *grad_bias, void *workspace,
                                      size_t workspace_bytes, hipStream_t stream) {
    const char *fn = "tc_attn_backward";
    clear_error();
    tc_status st = check_attn(fn, a, false);
    if (st != TC_OK) return st;
    TC_REQUIRE(a->total_k == 0 || (a->num_seqs > 0 && a->max_k > 0 && a->k_offsets && a->q_offsets),
               TC_ERR_INVALID_ARG, "%s: keys, but no offsets, num_seqs or max_k", fn);
    const bool rq = a->total_q > 0, rk = a->total_k > 0;
    const struct {
        const char *name;
        tc_rows r;
        bool required;
    } rows[] = {{"q", q, rq}, {"k", k, rk}, {"v", v, rk}, {"out", out, rq},
                {"grad_out", grad_out, rq}, {"grad_q", grad_q, rq}, {"grad_k", grad_k, rk},
                {"grad_v", grad_v, rk}};
    for (const auto &r : rows)
        if ((st = check_rows(fn, r.name, r.r, a->dtype, r.required)) != TC_OK) return st;
    TC_REQUIRE(lse || !rq, TC_ERR_INVALID_ARG, "%s: null pointer: lse", fn);
    TC_REQUIRE(!out_low || a->dtype == TC_BF16, TC_ERR_INVALID_ARG,
               "%s: out_low is for TC_BF16 only", fn);
    TC_REQUIRE(aligned16(out_low), TC_ERR_UNSUPPORTED, "%s: out_low must be 16-byte aligned", fn);
    TC_REQUIRE(!grad_bias || a->bias_table, TC_ERR_INVALID_ARG,
               "%s: grad_bias without bias_table", fn);
    const size_t need = tc_attn_backward_workspace_bytes(a);
    TC_REQUIRE(need == 0 || (workspace && workspace_bytes >= need &&
                             (reinterpret_cast<uintptr_t>(workspace) & 255u) == 0),
               TC_ERR_WORKSPACE, "%s: needs a 256-byte aligned workspace of %zu bytes, got %zu", fn,
               need, workspace_bytes);
    if (!rq && !rk && !grad_bias) return TC_OK;
    const Args args = make_args(*a);
    char *ws = static_cast<char *>(workspace);
    Grads g{q, k, v, out, grad_out, grad_q, grad_k, grad_v, static_cast<const bf16 *>(out_low),
            lse, reinterpret_cast<float *>(ws), nullptr};
    if (grad_bias)
        g.bias_part = reinterpret_cast<float *>(
            ws + up256(sizeof(float) * size_t(a->num_heads) * size_t(a->total_q)));
    if (a->dtype == TC_F32)
        backward<float>(*a, args, g, grad_bias, stream);
    else
        backward<bf16>(*a, args, g, grad_bias, stream);
    return check_launch(fn);
}
