// Attention backward over ragged bags (tc_attn_backward), with the gradient
// of the learned distance bias.
#include "tc_attn_tile.h"

namespace tc {
namespace {

using namespace attn;

struct Grads {
    tc_rows q, k, v, out, grad_out, dq, dk, dv;
    const float *lse;
    float *delta;      // [heads x total_q]: sum over j of p*dp of every row
    float *bias_part;  // [heads x parts x (2*reach + 1)], or nullptr
    float *part;       // dk, then dv: [heads x total_k x dim] each, or nullptr
    int64_t total_k;
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

// Gradient of one query's row, from the delta that k_attn_dq started with.
template <class T>
__device__ void row_dq(const Args &a, const Grads &g, const Seq &s, int i, int h) {
    const int64_t t = s.q0 + i;
    const int kvh = h / a.group;
    const Row2 q = row_at<T>(g.q, t, h, a.dim), go = row_at<T>(g.grad_out, t, h, a.dim);
    const float delta = dot(go, row_at<T>(g.out, t, h, a.dim));
    const float lse2 = g.lse[h * a.total_q + t] * kLog2e;
    Row2 dq{0.0f, 0.0f};
    float rest = 0.0f;
    const int n = limit(a, s, i), pos = i + s.shift;
    for (int j = 0; j < n; j++) {
        const Row2 k = row_at<T>(g.k, s.k0 + j, kvh, a.dim), v = row_at<T>(g.v, s.k0 + j, kvh, a.dim);
        float p, ds, gs;
        pair_grad(a, dot(q, k), a.table ? log2_bias(a, h, j - pos) : 0.0f, lse2, dot(go, v), delta,
                  p, ds, gs);
        dq.a += gs * k.a;
        dq.b += gs * k.b;
        rest += ds;
    }
    if ((threadIdx.x & 63) == 0) g.delta[h * a.total_q + t] = delta + rest;
    put_row<T>(g.dq, t, h, a.dim, dq);
}

// Gradients of one key's rows, over the queries that see it and heads h0 ..
// h0 + span - 1.
template <class T>
__device__ void row_dkv(const Args &a, const Grads &g, const Seq &s, int j, int h0, int span) {
    const int kvh = h0 / a.group;
    const Row2 k = row_at<T>(g.k, s.k0 + j, kvh, a.dim), v = row_at<T>(g.v, s.k0 + j, kvh, a.dim);
    Row2 dk{0.0f, 0.0f}, dv{0.0f, 0.0f};
    for (int h = h0; h < h0 + span; h++) {
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
    if (g.part) {
        float *p = g.part + (h0 * g.total_k + s.k0 + j) * a.dim;
        store_row(p, dk, a.dim);
        store_row(p + int64_t(a.heads) * g.total_k * a.dim, dv, a.dim);
        return;
    }
    put_row<T>(g.dk, s.k0 + j, kvh, a.dim, dk);
    put_row<T>(g.dv, s.k0 + j, kvh, a.dim, dv);
}

// Adds the entries of a block of ds (rows are queries, columns keys, distance
// `rel` at row 0, column 0) to the sums by distance, which belong to this
// wavefront. Entry (query, key) goes to row (key - query) mod 32 of `buf`, whose
// 32 entries are those of two distances, r for the keys from r on and r - 32 for
// those before; a lane adds up half a row.
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
    for (int r = 0; r < 16; r++) buf[((c - 4 * half - reg_row(r)) & 31) * kSkew + c] = ds[r];
    __builtin_amdgcn_wave_barrier();
    float lo = 0.0f, hi = 0.0f;  // of distance c, of distance c - 32
#pragma unroll
    for (int n = 0; n < 16; n++) {
        const int col = 16 * half + n;
        const float x = buf[c * kSkew + col];
        lo += col >= c ? x : 0.0f;
        hi += col >= c ? 0.0f : x;
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

// Gradient of the queries. A wavefront has 32 queries, the workgroup shares
// tiles of BN keys and values.
//
// delta = sum_j p_j dp_j is <grad_out, out>, but out has been rounded, and the
// bias gradient adds up so many terms p*(dp - delta) that cancel that this
// shows. The terms of a row add up to 0, so what they do add up to here is
// the error of delta: k_attn_dkv gets the sum of the two, exact to fp32.
template <class T, int DH, int NW, int BN>
__global__ __launch_bounds__(NW * 64, sizeof(T) * DH <= 256 ? 2 : 1) void k_attn_dq(Args a, Grads g, int slots) {
    typedef Tile<T, DH> Tl;
    constexpr int BM = NW * 32, NT = NW * 64, CPR = DH / 8, IT = BN * CPR / NT;
    constexpr int KS = DH / 16, DB = DH / 32;
    constexpr bool AHEAD = NW > 1;  // a lone wavefront has no registers for it
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ int first_bad;
    T *kt = reinterpret_cast<T *>(lds), *vt = kt + BN * DH;
    float *bias = reinterpret_cast<float *>(vt + BN * DH);
    const int wave = threadIdx.x >> 6, l = threadIdx.x & 63, half = l >> 5;
    const int id = blockIdx.x;
    const int kvh = id % a.kv_heads, h = kvh * a.group + (id / a.kv_heads) % a.group;
    int tile;
    const int b = seq_of_slot(a.q_off, a.num_seqs, slots - 1 - id / a.heads, BM, tile);
    const Seq s = seq_of(a, b, -1);
    const int i0 = tile * BM;
    if (i0 >= s.qn) return;
    const int end = limit(a, s, min(i0 + BM, s.qn) - 1), block_first = limit(a, s, i0);
    const auto kv = KvOf<T, false>::make({g.k, g.v, {}, 0, 0}, s, kvh);
    const int w0 = i0 + wave * 32, i = w0 + (l & 31);
    const int lim = limit(a, s, min(i, s.qn - 1));
    const int lim_first = limit(a, s, min(w0, s.qn - 1));
    const int lim_last = limit(a, s, min(w0 + 31, s.qn - 1));
    const int64_t t = s.q0 + min(i, s.qn - 1);
    const int row0 = threadIdx.x / CPR, col = threadIdx.x % CPR;
    const bool live = col * 8 < a.dim;
    if (a.table) load_bias(a, h, bias);
    if (threadIdx.x == 0) first_bad = INT32_MAX;

    V8<T> qf[KS], of[KS];
    float delta = 0.0f, rest = 0.0f;
    {
        const T *qp = static_cast<const T *>(g.q.data) + t * g.q.token_stride + h * g.q.head_stride;
        const T *gp = static_cast<const T *>(g.grad_out.data) + t * g.grad_out.token_stride +
                      h * g.grad_out.head_stride;
        const T *op = static_cast<const T *>(g.out.data) + t * g.out.token_stride +
                      h * g.out.head_stride;
        // <grad_out, out> as the diagonal of a product of the same form as
        // <grad_out, v> below: where one key has all the weight, out is v, and
        // their difference is 0 to the last bit
        f32x16 x = zero16();
#pragma unroll
        for (int ks = 0; ks < KS; ks++) {
            const int c = 2 * ks + half;
            qf[ks] = chunk_of(qp, c, a.dim);
            of[ks] = chunk_of(gp, c, a.dim);
            x = mma(chunk_of(op, c, a.dim), of[ks], x);
        }
#pragma unroll
        for (int r = 0; r < 16; r++) delta = 4 * half + reg_row(r) == (l & 31) ? x[r] : delta;
        // the other half has the entry if this one does not
        const float other = __shfl_xor(delta, 32, kWave);
        delta = ((l & 31) >> 2 & 1) == half ? delta : other;
    }
    const float lse2 = g.lse[h * a.total_q + t] * kLog2e;

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
    if (AHEAD) fetch(0);
    for (int kb = 0; kb < end; kb += BN) {
        const bool mixed = min(kb + BN, end) > block_first;
        if (!AHEAD) fetch(kb);
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
        if (AHEAD && kb + BN < end) fetch(kb + BN);
#pragma unroll
        for (int n = 0; n < BN / 32; n++) {
            const int k0 = kb + 32 * n;
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
            if (a.table) add_bias(a, bias, k0 - (w0 + s.shift), x);
#pragma unroll
            for (int r = 0; r < 16; r++) x[r] = exp2_fast(x[r] - lse2) * (dp[r] - delta);
            if (k0 + 32 > lim_first) {
                const int left = lim - k0 - 4 * half;
#pragma unroll
                for (int r = 0; r < 16; r++) x[r] = reg_row(r) < left ? x[r] : 0.0f;
            }
#pragma unroll
            for (int r = 0; r < 16; r++) {
                rest += x[r];
                x[r] *= f[r];
            }
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
    rest += __shfl_xor(rest, 32, kWave);
    __syncthreads();
    const int bad = first_bad;
    if (bad < lim_last)
        for (int r = 0; r < min(32, s.qn - w0); r++)
            if (limit(a, s, w0 + r) > bad) row_dq<T>(a, g, s, w0 + r, h);
    if (i >= s.qn || lim > bad) return;
    if (half == 0) g.delta[h * a.total_q + t] = delta + rest;
    T *dp = static_cast<T *>(g.dq.data) + t * g.dq.token_stride + h * g.dq.head_stride;
#pragma unroll
    for (int db = 0; db < DB; db++) store_block(dp, acc[db], 1.0f, db, a.dim);
}

// Gradients of the keys and values, and the bias gradient by distance. A
// wavefront has 32 keys, the workgroup shares tiles of BQ queries and their
// output gradients and takes the heads that share the keys one after another,
// so that their sum needs no atomics. Blocks have queries as rows here (the
// products that follow sum over them).
//
// A workgroup takes every gridDim.x-th tile of its heads and, with DIST, keeps
// one sum per head, distance and wavefront in LDS throughout, so that the order
// of the terms is fixed. Where those of all its heads do not fit (kept = 1) it
// keeps one head's and adds them to its own row in the workspace after each.
// It has all heads that share a key head (span = group), or one (span = 1) and
// leaves its part of the sum over them to k_attn_sum_heads.
template <class T, int DH, int NW, int BQ, bool DIST>
__global__ __launch_bounds__(NW * 64, sizeof(T) * DH <= 128 ? 2 : 1) void k_attn_dkv(
    Args a, Grads g, int slots, int span, int kept) {
    typedef Tile<T, DH> Tl;
    constexpr int BM = NW * 32, NT = NW * 64, CPR = DH / 8, IT = BQ * CPR / NT;
    constexpr int KS = DH / 16, DB = DH / 32;
    constexpr bool AHEAD = NW > 1;  // a lone wavefront has no registers for it
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ int last_bad;
    __shared__ __attribute__((aligned(16))) float stat[2][BQ];  // lse (in log 2) and delta
    T *qt = reinterpret_cast<T *>(lds), *ot = qt + BQ * DH;
    float *bias = reinterpret_cast<float *>(ot + BQ * DH);
    const int wave = threadIdx.x >> 6, l = threadIdx.x & 63, half = l >> 5;
    const int h0 = blockIdx.y * span, kvh = h0 / a.group, width = 2 * a.reach + 1;
    float *skew = bias + (a.table ? 2 * (a.reach + kBiasPad) + 1 : 0) + wave * 32 * kSkew;
    float *dists = skew + (NW - wave) * 32 * kSkew;  // [kept][NW][width]
    float far_left = 0.0f, far_right = 0.0f;
    if (DIST)
        for (int d = threadIdx.x; d < kept * NW * width; d += NT) dists[d] = 0.0f;
    const int row0 = threadIdx.x / CPR, col = threadIdx.x % CPR;
    const bool live = col * 8 < a.dim;
    // the workgroup's sums of the head in dists + at into its row; with `add`
    // to what the row holds
    auto flush = [&](int h, int at, bool add) {
        __syncthreads();
        float *p = g.bias_part + (int64_t(h) * gridDim.x + blockIdx.x) * width;
        for (int d = threadIdx.x; d < width; d += NT) {
            float x = dists[at + d];
#pragma unroll
            for (int w = 1; w < NW; w++) x += dists[at + w * width + d];
            p[d] = add ? p[d] + x : x;
        }
    };
    bool begun = false, nan_seen = false;

    for (int slot = blockIdx.x; slot < slots; slot += int(gridDim.x)) {
    int tile;
    const int b = seq_of_slot(a.k_off, a.num_seqs, slot, BM, tile);
    const Seq s = seq_of(a, b, -1);
    const int j0 = tile * BM;
    if (j0 >= s.kn) continue;
    const int w0 = j0 + wave * 32, j = w0 + (l & 31);
    const int begin = first_query(a, s, j0) / BQ * BQ;
    const int block_last = first_query(a, s, min(j0 + BM, s.kn) - 1);
    const int fq = first_query(a, s, min(j, s.kn - 1));
    const int fq_first = first_query(a, s, min(w0, s.kn - 1));
    const int fq_last = first_query(a, s, min(w0 + 31, s.kn - 1));
    __syncthreads();  // the last tile's flag has been read
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
    for (int hg = 0; hg < span; hg++) {
        const int h = h0 + hg;
        if (AHEAD && begin < s.qn) fetch(h, begin);
        if (a.table) {
            __syncthreads();
            load_bias(a, h, bias);
        }
        float *dist = dists + ((kept > 1 ? hg : 0) * NW + wave) * width;
        for (int qb = begin; qb < s.qn; qb += BQ) {
            const bool mixed = qb < block_last;
            if (!AHEAD) fetch(h, qb);
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
            if (AHEAD && qb + BQ < s.qn) fetch(h, qb + BQ);
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
                        dp[r] = x[r] * (dp[r] - del[e]);
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
                if (DIST) {
                    if (w0 + 32 > s.kn) {  // keys past the last one repeat it
#pragma unroll
                        for (int r = 0; r < 16; r++) dp[r] = j < s.kn ? dp[r] : 0.0f;
                    }
                    add_distances(a, dp, w0 - (q0 + s.shift), skew, dist, far_left, far_right);
                }
#pragma unroll
                for (int r = 0; r < 16; r++) dp[r] *= f[r];
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
        if (DIST) {
            far_left = wave_sum(far_left);
            far_right = wave_sum(far_right);
            if (l == 0) {
                dist[0] += far_left;
                dist[width - 1] += far_right;
            }
            far_left = far_right = 0.0f;
        }
        if (DIST && kept < span) {
            flush(h, 0, begun);
            __syncthreads();
            for (int d = threadIdx.x; d < NW * width; d += NT) dists[d] = 0.0f;
        }
    }
    begun = true;
    __syncthreads();
    const int bad = last_bad;
    if (bad >= fq_first)
        for (int r = 0; r < min(32, s.kn - w0); r++)
            if (first_query(a, s, w0 + r) <= bad) {
                row_dkv<T>(a, g, s, w0 + r, h0, span);
                if (DIST && l == 0) nan_seen = true;
            }
    if (j < s.kn && fq > bad) {
        const int64_t t = s.k0 + j;
        if (g.part) {
            float *kp = g.part + (h0 * g.total_k + t) * a.dim;
            float *vp = kp + int64_t(a.heads) * g.total_k * a.dim;
#pragma unroll
            for (int db = 0; db < DB; db++) {
                store_block(kp, dk[db], 1.0f, db, a.dim);
                store_block(vp, dv[db], 1.0f, db, a.dim);
            }
        } else {
            T *kp = static_cast<T *>(g.dk.data) + t * g.dk.token_stride + kvh * g.dk.head_stride;
            T *vp = static_cast<T *>(g.dv.data) + t * g.dv.token_stride + kvh * g.dv.head_stride;
#pragma unroll
            for (int db = 0; db < DB; db++) {
                store_block(kp, dk[db], 1.0f, db, a.dim);
                store_block(vp, dv[db], 1.0f, db, a.dim);
            }
        }
    }
    }
    if (!DIST) return;
    for (int hg = 0; hg < span; hg++) {
        if (kept == span) {
            if (nan_seen) dists[(hg * NW + wave) * width + a.reach] = __builtin_nanf("");
            flush(h0 + hg, hg * NW * width, false);
        } else {
            // no tile: zeros; otherwise what the last head left, zeros too
            if (nan_seen) dists[wave * width + a.reach] = __builtin_nanf("");
            flush(h0 + hg, 0, begun);
        }
    }
}

// The gradients of keys and values from their parts, over the heads that share
// a key head, in order: a lane has 4 elements.
template <class T>
__global__ __launch_bounds__(kBlock) void k_attn_sum_heads(Args a, Grads g) {
    const int per = a.dim / 4;
    const int64_t n = g.total_k * a.kv_heads * per;
    for (int64_t i = int64_t(blockIdx.x) * kBlock + threadIdx.x; i < 2 * n;
         i += int64_t(gridDim.x) * kBlock) {
        const bool is_v = i >= n;
        int64_t r = is_v ? i - n : i;
        const int d = int(r % per) * 4;
        r /= per;
        const int kvh = int(r % a.kv_heads);
        const int64_t t = r / a.kv_heads;
        const float *p = g.part + ((is_v ? a.heads : 0) + int64_t(kvh) * a.group) * g.total_k * a.dim +
                         t * a.dim + d;
        f32x4 x = *reinterpret_cast<const f32x4 *>(p);
        for (int hg = 1; hg < a.group; hg++)
            x += *reinterpret_cast<const f32x4 *>(p + hg * g.total_k * a.dim);
        const float y[4] = {x[0], x[1], x[2], x[3]};
        const tc_rows &o = is_v ? g.dv : g.dk;
        store4(static_cast<T *>(o.data) + t * o.token_stride + kvh * o.head_stride + d, y);
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
    int q_waves, k_waves;  // of a workgroup of k_attn_dq, of k_attn_dkv
    int64_t q_slots, k_slots;
    int span, parts;  // of k_attn_dkv: heads of a workgroup, workgroups of a head
};

Plan plan_of(const tc_attn &a) {
    Plan p{};
    const int64_t n = a.num_seqs > 0 ? a.num_seqs : 1;
    const int group = a.num_heads / a.num_kv_heads;
    p.q_waves = a.max_q <= 32 || a.total_q / n <= 64 ? 1 : 4;
    p.k_waves = a.max_k <= 32 || a.total_k / n <= 64 ? 1 : 4;
    p.q_slots = tile_slots(a.total_q, a.num_seqs, 32 * p.q_waves);
    p.k_slots = tile_slots(a.total_k, a.num_seqs, 32 * p.k_waves);
    const int64_t cus = device_cus();
    p.span = p.k_slots * p.k_waves * a.num_kv_heads >= 16 * cus ? group : 1;
    const int64_t most = 8 * cus * p.span / a.num_heads + 1;
    p.parts = int(p.k_slots < most ? p.k_slots : most);
    return p;
}

size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// The parts of a workspace.
struct Space {
    size_t bias, part, bytes;  // delta is at 0
};

Space space_of(const tc_attn &a) {
    Space s{};
    if (a.total_q <= 0 || a.num_seqs <= 0 || a.num_kv_heads <= 0 || a.num_heads < a.num_kv_heads ||
        a.reach < 0 || a.total_k < 0 || a.head_dim <= 0)
        return s;
    const Plan p = plan_of(a);
    const size_t h = a.num_heads;
    s.bias = up256(sizeof(float) * h * size_t(a.total_q));
    s.part = s.bias + (a.bias_table ? up256(sizeof(float) * h * size_t(p.parts) *
                                            size_t(2 * a.reach + 1))
                                    : 0);
    s.bytes = s.part;
    if (p.span < a.num_heads / a.num_kv_heads)
        s.bytes += up256(2 * sizeof(float) * h * size_t(a.total_k) * size_t(a.head_dim));
    return s;
}

template <class T, int DH, int NW, bool DIST>
void launch_dkv(const Args &a, const Plan &p, const Grads &g, hipStream_t stream) {
    const size_t width = DIST ? (2 * a.reach + 1) * sizeof(float) : 0;
    // sums by distance of all heads of a workgroup in 32 KB, or of one
    const int kept = size_t(p.span) * NW * width <= (32 << 10) ? p.span : 1;
    const size_t bytes = 2 * 32 * DH * sizeof(T) +
                         (a.table ? bias_entries(a.reach) * sizeof(float) : 0) +
                         (DIST ? NW * 32 * kSkew * sizeof(float) : 0) + kept * NW * width;
    hipLaunchKernelGGL((k_attn_dkv<T, DH, NW, 32, DIST>), dim3(p.parts, a.heads / p.span),
                       dim3(NW * 64), bytes, stream, a, g, int(p.k_slots), p.span, kept);
}

template <class T, int DH>
void launch(const tc_attn &t, const Args &a, const Plan &p, const Grads &g, hipStream_t stream) {
    constexpr int BN = sizeof(T) == 4 ? 32 : 64;
    const size_t bias = a.table ? bias_entries(a.reach) * sizeof(float) : 0;
    if (t.total_q > 0) {
        const dim3 grid(unsigned(p.q_slots * a.heads));
        if (p.q_waves == 1)
            hipLaunchKernelGGL((k_attn_dq<T, DH, 1, 32>), grid, dim3(64),
                               2 * 32 * DH * sizeof(T) + bias, stream, a, g, int(p.q_slots));
        else
            hipLaunchKernelGGL((k_attn_dq<T, DH, 4, BN>), grid, dim3(256),
                               2 * BN * DH * sizeof(T) + bias, stream, a, g, int(p.q_slots));
    }
    if (t.total_k > 0) {
        if (p.k_waves == 1)
            g.bias_part ? launch_dkv<T, DH, 1, true>(a, p, g, stream)
                        : launch_dkv<T, DH, 1, false>(a, p, g, stream);
        else
            g.bias_part ? launch_dkv<T, DH, 4, true>(a, p, g, stream)
                        : launch_dkv<T, DH, 4, false>(a, p, g, stream);
        if (g.part) {
            const int64_t n = 2 * t.total_k * t.num_kv_heads * (t.head_dim / 4);
            hipLaunchKernelGGL((k_attn_sum_heads<T>),
                               dim3(grid_for(n, kBlock, int64_t(device_cus()) * 16)), dim3(kBlock),
                               0, stream, a, g);
        }
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
    // without queries or keys there are no parts, and every sum is 0
    const int width = p.total_q > 0 && p.total_k > 0 ? 2 * a.reach + 1 : 0;
    if (width > 0)
        hipLaunchKernelGGL(k_bias_parts, dim3((width + 63) / 64, a.heads), dim3(kBlock), 0, stream,
                           g.bias_part, plan.parts, width);
    hipLaunchKernelGGL(k_bias_buckets, dim3(p.num_buckets, a.heads), dim3(kWave), 0, stream, a,
                       g.bias_part, plan.parts, width, grad_bias);
}

}  // namespace
}  // namespace tc

using namespace tc;
using namespace tc::attn;

extern "C" size_t tc_attn_backward_workspace_bytes(const tc_attn *a) {
    return a ? space_of(*a).bytes : 0;
}

extern "C" tc_status tc_attn_backward(const tc_attn *a, tc_rows q, tc_rows k, tc_rows v,
                                      tc_rows out, const float *lse,
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
    TC_REQUIRE(!grad_bias || a->bias_table, TC_ERR_INVALID_ARG,
               "%s: grad_bias without bias_table", fn);
    const Space space = space_of(*a);
    const size_t need = space.bytes;
    TC_REQUIRE(need == 0 || (workspace && workspace_bytes >= need &&
                             (reinterpret_cast<uintptr_t>(workspace) & 255u) == 0),
               TC_ERR_WORKSPACE, "%s: needs a 256-byte aligned workspace of %zu bytes, got %zu", fn,
               need, workspace_bytes);
    if (!rq && !rk && !grad_bias) return TC_OK;
    const Args args = make_args(*a);
    char *ws = static_cast<char *>(workspace);
    const Plan plan = plan_of(*a);
    // without queries nothing is kept, and the gradients of the keys are 0
    Grads g{q, k, v, out, grad_out, grad_q, grad_k, grad_v, lse, reinterpret_cast<float *>(ws),
            nullptr, nullptr, a->total_k};
    if (grad_bias && rq) g.bias_part = reinterpret_cast<float *>(ws + space.bias);
    if (rq && plan.span < args.group) g.part = reinterpret_cast<float *>(ws + space.part);
    TC_REQUIRE(plan.q_slots * a->num_heads < (int64_t(1) << 31), 
               TC_ERR_INVALID_ARG, "%s: more than 2^31 workgroups", fn);
    backward(*a, plan, args, g, grad_bias, stream);
    return check_launch(fn);
}
