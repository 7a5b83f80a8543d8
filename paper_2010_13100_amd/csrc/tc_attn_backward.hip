// Attention backward over ragged bags (tc_attn_backward), with the gradient
// of the learned distance bias.
#include "tc_attn_tile.h"

namespace tc {
namespace {

using namespace attn;

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

// Adds the entries of a block of ds (rows are keys, columns queries, distance
// `rel` at row 0, column 0) to the sums by distance, which belong to this
// wavefront. Entry (key, query) goes to row (key - query) mod 32 of `buf`, whose
// 32 entries are those of two distances, r for the first 32 - r queries and
// r - 32 for the others; a lane adds up half a row.
constexpr int kSkew = 33;
__device__ __forceinline__ void add_distances(const Args &a, const f32x16 &ds, int rel, float *buf,
                                              float *dist, float &far_left, float &far_right) {
    const int l = threadIdx.x & 63, half = l >> 5, c = l & 31;
    if (rel + 31 <= -a.reach || rel - 31 >= a.reach) {
        float x = 0.0f;
#pragma unroll
        for (int r = 0; r < 16; r++) x += ds[r];
        if (rel < 0)
            far_left += x;
        else
            far_right += x;
        return;
    }
#pragma unroll
    for (int r = 0; r < 16; r++) buf[((4 * half + reg_row(r) - c) & 31) * kSkew + c] = ds[r];
    __builtin_amdgcn_wave_barrier();
    float lo = 0.0f, hi = 0.0f;
#pragma unroll
    for (int n = 0; n < 16; n++) {
        const int col = 16 * half + n;
        const float x = buf[c * kSkew + col];
        const bool first = col < 32 - c;
        lo += first ? x : 0.0f;
        hi += first ? 0.0f : x;
    }
    __builtin_amdgcn_wave_barrier();
    lo += __shfl_xor(lo, 32, kWave);
    hi += __shfl_xor(hi, 32, kWave);
    const int d = rel + (half ? c - 32 : c);
    const float x = half ? hi : lo;
    if (d <= -a.reach)
        far_left += x;
    else if (d >= a.reach)
        far_right += x;
    else
        dist[d + a.reach] += x;
}

// Gradient of the queries, and the bias gradient by distance. A wavefront has
// 32 queries, the workgroup shares tiles of BN keys and values; a workgroup
// takes every gridDim.x-th tile of its head and keeps one sum per distance and
// wavefront in LDS throughout, so that their order is fixed.
template <class T, int DH, int NW, int BN>
__global__ __launch_bounds__(NW * 64) void k_attn_dq(Args a, Grads g, int slots) {
    typedef Tile<T, DH> Tl;
    constexpr int BM = NW * 32, NT = NW * 64, CPR = DH / 8, IT = BN * CPR / NT;
    constexpr int KS = DH / 16, DB = DH / 32;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ int first_bad;
    T *kt = reinterpret_cast<T *>(lds), *vt = kt + BN * DH;
    const int wave = threadIdx.x >> 6, l = threadIdx.x & 63, half = l >> 5;
    const int width = 2 * a.reach + 1;
    float *skew = reinterpret_cast<float *>(vt + BN * DH) + wave * 32 * kSkew;
    float *bias = skew + (NW - wave) * 32 * kSkew;
    float *dists = bias + (a.table ? 2 * (a.reach + kBiasPad) + 1 : 0), *dist = dists + wave * width;
    const int h = blockIdx.y, kvh = h / a.group;
    if (a.table) load_bias(a, h, bias);
    if (g.bias_part)
        for (int d = threadIdx.x; d < NW * width; d += NT) dists[d] = 0.0f;
    float far_left = 0.0f, far_right = 0.0f;
    const int row0 = threadIdx.x / CPR, col = threadIdx.x % CPR;
    const bool live = col * 8 < a.dim;

    for (int slot = slots - 1 - int(blockIdx.x); slot >= 0; slot -= int(gridDim.x)) {
        int tile;
        const int b = seq_of_slot(a.q_off, a.num_seqs, slot, BM, tile);
        const Seq s = seq_of(a, b, -1);
        const int i0 = tile * BM;
        if (i0 >= s.qn) continue;
        const int end = limit(a, s, min(i0 + BM, s.qn) - 1), block_first = limit(a, s, i0);
        const auto kv = KvOf<T, false>::make({g.k, g.v, {}, 0, 0}, s, kvh);
        const int w0 = i0 + wave * 32, i = w0 + (l & 31);
        const int lim = limit(a, s, min(i, s.qn - 1));
        const int lim_first = limit(a, s, min(w0, s.qn - 1));
        const int lim_last = limit(a, s, min(w0 + 31, s.qn - 1));
        const int64_t t = s.q0 + min(i, s.qn - 1);

        V8<T> qf[KS], of[KS];
        float delta = 0.0f;
        {
            const T *qp = static_cast<const T *>(g.q.data) + t * g.q.token_stride + h * g.q.head_stride;
            const T *gp = static_cast<const T *>(g.grad_out.data) + t * g.grad_out.token_stride +
                          h * g.grad_out.head_stride;
            const T *op = static_cast<const T *>(g.out.data) + t * g.out.token_stride +
                          h * g.out.head_stride;
            // <grad_out, out> as the diagonal of a product of the same form as
            // <grad_out, v> below: where one key has all the weight, out is v,
            // and their difference is 0 to the last bit
            f32x16 x = zero16();
#pragma unroll
            for (int ks = 0; ks < KS; ks++) {
                const int c = 2 * ks + half;
                qf[ks] = chunk_of(qp, c, a.dim);
                of[ks] = chunk_of(gp, c, a.dim);
                x = mma(chunk_of(op, c, a.dim), of[ks], x);
            }
            if constexpr (sizeof(T) == 2) {
                if (g.out_low) {
#pragma unroll
                    for (int ks = 0; ks < KS; ks++)
                        x = mma(chunk_of(g.out_low + (t * a.heads + h) * a.dim, 2 * ks + half, a.dim),
                                of[ks], x);
                }
            }
#pragma unroll
            for (int r = 0; r < 16; r++)
                delta = 4 * half + reg_row(r) == (l & 31) ? x[r] : delta;
            // the other half has the entry if this one does not
            const float other = __shfl_xor(delta, 32, kWave);
            delta = ((l & 31) >> 2 & 1) == half ? delta : other;
            if (half == 0 && i < s.qn) g.delta[h * a.total_q + t] = delta;
        }
        // rows past the last one repeat it with probability 0
        const float lse2 = i < s.qn ? g.lse[h * a.total_q + t] * kLog2e : INFINITY;

        f32x16 acc[DB];
#pragma unroll
        for (int db = 0; db < DB; db++) acc[db] = zero16();
        Raw<T> kr[IT], vr[IT];
        auto fetch = [&](int kb) {
#pragma unroll
            for (int n = 0; n < IT; n++) {
                const int j = kb + row0 + n * (NT / CPR);
                kr[n] = zero_raw<T>();
                vr[n] = zero_raw<T>();
                if (j < end && live) {
                    const Loc at = kv.loc(j);
                    kr[n] = load_raw(kv.k(at) + col * 8, 0);
                    vr[n] = load_raw(kv.v(at) + col * 8, 0);
                }
            }
        };
        __syncthreads();  // the last tile's flag has been read
        if (threadIdx.x == 0) first_bad = INT32_MAX;
        fetch(0);
        for (int kb = 0; kb < end; kb += BN) {
            const bool mixed = min(kb + BN, end) > block_first;
            __syncthreads();
#pragma unroll
            for (int n = 0; n < IT; n++) {
                const int row = row0 + n * (NT / CPR);
                V8<T> x;
                expand(kr[n], x);
                if (mixed && clean(x)) atomicMin(&first_bad, kb + row);
                Tl::put(kt, row, col, x);
                expand(vr[n], x);
                Tl::put(vt, row, col, x);
            }
            __syncthreads();
            if (kb + BN < end) fetch(kb + BN);
#pragma unroll
            for (int n = 0; n < BN / 32; n++) {
                const int k0 = kb + 32 * n, rel = k0 - (w0 + s.shift);
                if (k0 >= lim_last) break;
                f32x16 x = zero16(), dp = zero16();
#pragma unroll
                for (int ks = 0; ks < KS; ks++) {
                    x = mma(Tl::rows(kt, 32 * n, ks), qf[ks], x);
                    dp = mma(Tl::rows(vt, 32 * n, ks), of[ks], dp);
                }
                f32x16 f;  // d(score)/d(product), with the scale
                if (a.capped) {
#pragma unroll
                    for (int r = 0; r < 16; r++) {
                        const float th = tanh_of(a.c1 * x[r]);
                        x[r] = a.c2 * th;
                        f[r] = a.scale * __builtin_fmaf(-th, th, 1.0f);
                    }
                } else {
#pragma unroll
                    for (int r = 0; r < 16; r++) {
                        x[r] *= a.c1;
                        f[r] = a.scale;
                    }
                }
                if (a.table) add_bias(a, bias, rel, x);
#pragma unroll
                for (int r = 0; r < 16; r++) x[r] = exp2_fast(x[r] - lse2) * (dp[r] - delta);
                if (k0 + 32 > lim_first) {
                    const int left = lim - k0 - 4 * half;
#pragma unroll
                    for (int r = 0; r < 16; r++) x[r] = reg_row(r) < left ? x[r] : 0.0f;
                }
                if (g.bias_part) add_distances(a, x, rel, skew, dist, far_left, far_right);
#pragma unroll
                for (int r = 0; r < 16; r++) x[r] *= f[r];
#pragma unroll
                for (int u = 0; u < 2; u++) {
                    V8<T> p;
                    pack(x, u, p);
#pragma unroll
                    for (int db = 0; db < DB; db++)
                        acc[db] = mma(Tl::cols(kt, 32 * n + 16 * u, db), p, acc[db]);
                }
            }
        }
        __syncthreads();
        const int bad = first_bad;
        if (bad < lim_last)
            for (int r = 0; r < min(32, s.qn - w0); r++)
                if (limit(a, s, w0 + r) > bad) {
                    row_dq<T>(a, g, s, w0 + r, h, nullptr);
                    if (g.bias_part && l == 0) dist[a.reach] = __builtin_nanf("");
                }
        if (i < s.qn && lim <= bad) {
            T *dp = static_cast<T *>(g.dq.data) + t * g.dq.token_stride + h * g.dq.head_stride;
#pragma unroll
            for (int db = 0; db < DB; db++) store_block(dp, acc[db], 1.0f, db, a.dim);
        }
    }
    if (!g.bias_part) return;
    far_left = wave_sum(far_left);
    far_right = wave_sum(far_right);
    if (l == 0) {
        dist[0] += far_left;
        dist[width - 1] += far_right;
    }
    __syncthreads();
    for (int d = threadIdx.x; d < width; d += NT) {
        float x = dists[d];
#pragma unroll
        for (int w = 1; w < NW; w++) x += dists[w * width + d];
        g.bias_part[(int64_t(h) * gridDim.x + blockIdx.x) * width + d] = x;
    }
}

// Gradients of the keys and values: a wavefront has 32 keys, the workgroup
// shares tiles of BQ queries and their output gradients and takes the heads
// that share the keys one after another, so that their sum needs no atomics.
// Blocks have queries as rows here (the products that follow sum over them).
template <class T, int DH, int NW, int BQ>
__global__ __launch_bounds__(NW * 64) void k_attn_dkv(Args a, Grads g, int slots) {
    typedef Tile<T, DH> Tl;
    constexpr int BM = NW * 32, NT = NW * 64, CPR = DH / 8, IT = BQ * CPR / NT;
    constexpr int KS = DH / 16, DB = DH / 32;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ int last_bad;
    __shared__ __attribute__((aligned(16))) float stat[2][BQ];  // lse (in log 2) and delta
    T *qt = reinterpret_cast<T *>(lds), *ot = qt + BQ * DH;
    float *bias = reinterpret_cast<float *>(ot + BQ * DH);
    const int wave = threadIdx.x >> 6, l = threadIdx.x & 63, half = l >> 5;
    const int id = blockIdx.x, kvh = id % a.kv_heads;
    int tile;
    const int b = seq_of_slot(a.k_off, a.num_seqs, id / a.kv_heads, BM, tile);
    const Seq s = seq_of(a, b, -1);
    const int j0 = tile * BM;
    if (j0 >= s.kn) return;
    const int w0 = j0 + wave * 32, j = w0 + (l & 31);
    const int begin = first_query(a, s, j0) / BQ * BQ;
    const int block_last = first_query(a, s, min(j0 + BM, s.kn) - 1);
    const int fq = first_query(a, s, min(j, s.kn - 1));
    const int fq_first = first_query(a, s, min(w0, s.kn - 1));
    const int fq_last = first_query(a, s, min(w0 + 31, s.kn - 1));
    if (threadIdx.x == 0) last_bad = -1;

    V8<T> kf[KS], vf[KS];
    {
        const int64_t t = s.k0 + min(j, s.kn - 1);
        const T *kp = static_cast<const T *>(g.k.data) + t * g.k.token_stride + kvh * g.k.head_stride;
        const T *vp = static_cast<const T *>(g.v.data) + t * g.v.token_stride + kvh * g.v.head_stride;
#pragma unroll
        for (int ks = 0; ks < KS; ks++) {
            kf[ks] = chunk_of(kp, 2 * ks + half, a.dim);
            vf[ks] = chunk_of(vp, 2 * ks + half, a.dim);
        }
    }
    f32x16 dk[DB], dv[DB];
#pragma unroll
    for (int db = 0; db < DB; db++) dk[db] = dv[db] = zero16();

    const int row0 = threadIdx.x / CPR, col = threadIdx.x % CPR;
    const bool live = col * 8 < a.dim;
    Raw<T> qr[IT], gr[IT];
    float lse_r = 0.0f, delta_r = 0.0f;
    auto fetch = [&](int h, int qb) {
#pragma unroll
        for (int n = 0; n < IT; n++) {
            const int i = qb + row0 + n * (NT / CPR);
            qr[n] = zero_raw<T>();
            gr[n] = zero_raw<T>();
            if (i < s.qn && live) {
                const int64_t t = s.q0 + i;
                qr[n] = load_raw(static_cast<const T *>(g.q.data) + t * g.q.token_stride +
                                     h * g.q.head_stride + col * 8, 0);
                gr[n] = load_raw(static_cast<const T *>(g.grad_out.data) +
                                     t * g.grad_out.token_stride + h * g.grad_out.head_stride +
                                     col * 8, 0);
            }
        }
        if (threadIdx.x < BQ) {
            const int i = qb + int(threadIdx.x);
            const bool in = i < s.qn;  // queries past the last one: probability 0
            lse_r = in ? g.lse[h * a.total_q + s.q0 + i] * kLog2e : INFINITY;
            delta_r = in ? g.delta[h * a.total_q + s.q0 + i] : 0.0f;
        }
    };
    for (int hg = 0; hg < a.group; hg++) {
        const int h = kvh * a.group + hg;
        if (begin < s.qn) fetch(h, begin);
        if (a.table) {
            __syncthreads();
            load_bias(a, h, bias);
        }
        for (int qb = begin; qb < s.qn; qb += BQ) {
            const bool mixed = qb < block_last;
            __syncthreads();
#pragma unroll
            for (int n = 0; n < IT; n++) {
                const int row = row0 + n * (NT / CPR);
                V8<T> x, y;
                expand(qr[n], x);
                expand(gr[n], y);
                if (mixed) {
                    const bool bx = clean(x), by = clean(y);
                    if (bx || by) atomicMax(&last_bad, qb + row);
                }
                Tl::put(qt, row, col, x);
                Tl::put(ot, row, col, y);
            }
            if (threadIdx.x < BQ) {
                stat[0][threadIdx.x] = lse_r;
                stat[1][threadIdx.x] = delta_r;
            }
            __syncthreads();
            if (qb + BQ < s.qn) fetch(h, qb + BQ);
#pragma unroll
            for (int n = 0; n < BQ / 32; n++) {
                const int q0 = qb + 32 * n;
                if (q0 + 32 <= fq_first || q0 >= s.qn) continue;
                f32x16 x = zero16(), dp = zero16();
#pragma unroll
                for (int ks = 0; ks < KS; ks++) {
                    x = mma(Tl::rows(qt, 32 * n, ks), kf[ks], x);
                    dp = mma(Tl::rows(ot, 32 * n, ks), vf[ks], dp);
                }
                f32x16 f;
                if (a.capped) {
#pragma unroll
                    for (int r = 0; r < 16; r++) {
                        const float th = tanh_of(a.c1 * x[r]);
                        x[r] = a.c2 * th;
                        f[r] = a.scale * __builtin_fmaf(-th, th, 1.0f);
                    }
                } else {
#pragma unroll
                    for (int r = 0; r < 16; r++) {
                        x[r] *= a.c1;
                        f[r] = a.scale;
                    }
                }
                if (a.table) add_bias_queries(a, bias, w0 - (q0 + s.shift), x);
#pragma unroll
                for (int c = 0; c < 4; c++) {
                    const f32x4 lse = *reinterpret_cast<const f32x4 *>(&stat[0][32 * n + 8 * c + 4 * half]);
                    const f32x4 del = *reinterpret_cast<const f32x4 *>(&stat[1][32 * n + 8 * c + 4 * half]);
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        const int r = 4 * c + e;
                        x[r] = exp2_fast(x[r] - lse[e]);
                        dp[r] = x[r] * (dp[r] - del[e]) * f[r];
                    }
                }
                if (q0 < fq_last) {
                    const int from = fq - q0 - 4 * half;
#pragma unroll
                    for (int r = 0; r < 16; r++) {
                        x[r] = reg_row(r) >= from ? x[r] : 0.0f;
                        dp[r] = reg_row(r) >= from ? dp[r] : 0.0f;
                    }
                }
#pragma unroll
                for (int u = 0; u < 2; u++) {
                    V8<T> p, d;
                    pack(x, u, p);
                    pack(dp, u, d);
#pragma unroll
                    for (int db = 0; db < DB; db++) {
                        dv[db] = mma(Tl::cols(ot, 32 * n + 16 * u, db), p, dv[db]);
                        dk[db] = mma(Tl::cols(qt, 32 * n + 16 * u, db), d, dk[db]);
                    }
                }
            }
        }
    }
    __syncthreads();
    const int bad = last_bad;
    if (bad >= fq_first)
        for (int r = 0; r < min(32, s.kn - w0); r++)
            if (first_query(a, s, w0 + r) <= bad) row_dkv<T>(a, g, s, w0 + r, kvh);
    if (j >= s.kn || fq <= bad) return;
    const int64_t t = s.k0 + j;
    T *kp = static_cast<T *>(g.dk.data) + t * g.dk.token_stride + kvh * g.dk.head_stride;
    T *vp = static_cast<T *>(g.dv.data) + t * g.dv.token_stride + kvh * g.dv.head_stride;
#pragma unroll
    for (int db = 0; db < DB; db++) {
        store_block(kp, dk[db], 1.0f, db, a.dim);
        store_block(vp, dv[db], 1.0f, db, a.dim);
    }
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

// Tiles and workgroups of a call, from its sizes alone.
struct Plan {
    int q_waves, k_waves;     // of a workgroup of k_attn_dq, of k_attn_dkv
    int64_t q_slots, k_slots;
    int parts;                // workgroups a head of k_attn_dq
};

Plan plan_of(const tc_attn &a) {
    Plan p{};
    const int64_t n = a.num_seqs > 0 ? a.num_seqs : 1;
    p.q_waves = a.max_q <= 32 || a.total_q / n <= 64 ? 1 : 4;
    p.k_waves = a.max_k <= 32 || a.total_k / n <= 64 ? 1 : 4;
    p.q_slots = tile_slots(a.total_q, a.num_seqs, 32 * p.q_waves);
    p.k_slots = tile_slots(a.total_k, a.num_seqs, 32 * p.k_waves);
    const int64_t most = int64_t(device_cus()) * 8 / a.num_heads + 1;
    p.parts = int(p.q_slots < most ? p.q_slots : most);
    return p;
}

template <class T, int DH>
void launch(const tc_attn &t, const Args &a, const Plan &p, const Grads &g, hipStream_t stream) {
    constexpr int BN = sizeof(T) == 4 ? 32 : 64;
    const size_t bias = a.table ? bias_entries(a.reach) * sizeof(float) : 0;
    const size_t dist = g.bias_part ? (2 * a.reach + 1) * sizeof(float) : 0;
    if (t.total_q > 0) {
        const dim3 grid(p.parts, a.heads);
        const size_t wave = 32 * kSkew * sizeof(float) + dist;
        if (p.q_waves == 1)
            hipLaunchKernelGGL((k_attn_dq<T, DH, 1, 32>), grid, dim3(64),
                               2 * 32 * DH * sizeof(T) + bias + wave, stream, a, g, int(p.q_slots));
        else
            hipLaunchKernelGGL((k_attn_dq<T, DH, 4, BN>), grid, dim3(256),
                               2 * BN * DH * sizeof(T) + bias + 4 * wave, stream, a, g,
                               int(p.q_slots));
    }
    if (t.total_k > 0) {
        const dim3 grid(unsigned(p.k_slots * a.kv_heads));
        if (p.k_waves == 1)
            hipLaunchKernelGGL((k_attn_dkv<T, DH, 1, 32>), grid, dim3(64),
                               2 * 32 * DH * sizeof(T) + bias, stream, a, g, int(p.k_slots));
        else
            hipLaunchKernelGGL((k_attn_dkv<T, DH, 4, 32>), grid, dim3(256),
                               2 * 32 * DH * sizeof(T) + bias, stream, a, g, int(p.k_slots));
    }
}

void backward(const tc_attn &p, const Plan &plan, const Args &a, const Grads &g, float *grad_bias,
              hipStream_t stream) {
    if (p.dtype == TC_F32)
        p.head_dim <= 64 ? launch<float, 64>(p, a, plan, g, stream)
                         : launch<float, 128>(p, a, plan, g, stream);
    else
        p.head_dim <= 64 ? launch<bf16, 64>(p, a, plan, g, stream)
                         : launch<bf16, 128>(p, a, plan, g, stream);
    if (!grad_bias) return;
    // without queries there are no parts, and every sum is 0
    const int width = p.total_q > 0 ? 2 * a.reach + 1 : 0;
    if (width > 0)
        hipLaunchKernelGGL(k_bias_parts, dim3((width + 63) / 64, a.heads), dim3(kBlock), 0, stream,
                           g.bias_part, plan.parts, width);
    hipLaunchKernelGGL(k_bias_buckets, dim3(p.num_buckets, a.heads), dim3(kWave), 0, stream, a,
                       g.bias_part, plan.parts, width, grad_bias);
}

size_t up256(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace
}  // namespace tc

using namespace tc;
using namespace tc::attn;

extern "C" size_t tc_attn_backward_workspace_bytes(const tc_attn *a) {
    if (!a || a->total_q <= 0 || a->num_seqs <= 0 || a->num_heads <= 0 || a->reach < 0) return 0;
    const size_t delta = up256(sizeof(float) * size_t(a->num_heads) * size_t(a->total_q));
    const size_t bias = a->bias_table ? up256(sizeof(float) * size_t(a->num_heads) *
                                              size_t(plan_of(*a).parts) * size_t(2 * a->reach + 1))
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
    const Plan plan = plan_of(*a);
    TC_REQUIRE(plan.k_slots * a->num_kv_heads < (int64_t(1) << 31) &&
                   plan.q_slots < (int64_t(1) << 31),
               TC_ERR_INVALID_ARG, "%s: more than 2^31 workgroups", fn);
    backward(*a, plan, args, g, grad_bias, stream);
    return check_launch(fn);
}
