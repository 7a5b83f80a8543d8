"""Attention over ragged bags (forward and backward) against the definition in
64 bits.

Tolerances, derived from the roundings: in fp32 a score carries about
sqrt(D)*2^-24 times the sum |q||k| of its products (scale*sum is about 8 here)
and a few 2^-24 of the cap, so probabilities are within about 1e-5; bounds are
2e-5 for the relative L2 error of a tensor and 1e-4 of its largest value for
the worst element. In bf16 the inputs are exact and products sum in fp32; the
probabilities (their gradients) and then the result are each rounded to bf16,
relative RMS 2^-9/sqrt(3)*1.5 = 1.7e-3 each, 2.4e-3 together: bounds 4e-3
(backward 5e-3, one more rounded factor) and 2^-5 of the largest value. The
log-sum and the bias gradient are fp32 in both: 2e-5 and 1e-4."""
import numpy as np
import pytest
import torch

from tests import attn_reference as R

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
L2 = {F32: 2e-5, BF16: 4e-3}
WORST = {F32: 1e-4, BF16: 2.0 ** -5}


def close(got, ref, dtype, what, slack=1.0):
    got, ref = got.double(), ref.double()
    fin = torch.isfinite(ref)
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), what + ": NaN"
    assert torch.equal(got[~fin & ~torch.isnan(ref)], ref[~fin & ~torch.isnan(ref)]), what
    d, r = (got - ref)[fin], ref[fin]
    if r.numel() == 0:
        return
    norm, top = r.norm().item(), r.abs().max().item()
    print(f"  {what}: L2 {d.norm().item() / max(norm, 1e-30):.2e} worst "
          f"{d.abs().max().item() / max(top, 1e-30):.2e}", flush=True)
    assert d.norm().item() <= L2[dtype] * slack * norm + 1e-12, what
    assert d.abs().max().item() <= WORST[dtype] * slack * top + 1e-12, what


def rows(gen, n, heads, dim, dtype, layout="rows", sigma=1.0):
    if layout == "heads":
        return (torch.randn((heads, n, dim), generator=gen, device="cuda") * sigma).to(dtype).transpose(0, 1)
    if layout == "padded":  # rows 8 elements apart, tokens further
        x = torch.full((n, heads, dim + 8), float("nan"), device="cuda").to(dtype)
        x[:, :, :dim] = (torch.randn((n, heads, dim), generator=gen, device="cuda") * sigma).to(dtype)
        return x[:, :, :dim]
    return (torch.randn((n, heads, dim), generator=gen, device="cuda") * sigma).to(dtype)


def make(q_lens, k_lens=None, *, heads=1, kv=None, dim=64, dtype=F32, causal=False, prefix=None,
         cap=0.0, buckets=0, reach=0, layout="rows", seed=0, train=True, scale=None):
    from paper_2010_13100_amd import tc
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    k_lens = q_lens if k_lens is None else k_lens
    kv = heads if kv is None else kv
    table = bucket_of = None
    if buckets:
        table = torch.randn((buckets, heads), generator=gen, device="cuda") * 0.7
        # buckets in no order, every distance any of them
        bucket_of = torch.randint(0, buckets, (2 * reach + 1,), generator=gen, device="cuda",
                                  dtype=torch.int32)
    p = R.Problem(list(q_lens), list(k_lens), heads, kv, dim, causal, prefix, scale, cap, table,
                  bucket_of)
    tq, tk = sum(q_lens), sum(k_lens)
    x = dict(q=rows(gen, tq, heads, dim, dtype, layout, 1.5),
             k=rows(gen, tk, kv, dim, dtype, layout), v=rows(gen, tk, kv, dim, dtype, layout),
             dout=rows(gen, tq, heads, dim, dtype, layout))
    a = tc.BagAttention(num_seqs=len(q_lens), num_heads=heads, num_kv_heads=kv, head_dim=dim,
                        dtype=dtype, total_q=tq, total_k=tk, max_q=max(q_lens, default=0),
                        max_k=max(k_lens, default=0), causal=causal, scale=p.scale, cap=cap,
                        bias_table=table, bucket_of=bucket_of, train=train)
    off = dict(q_offsets=torch.from_numpy(p.offsets("q")).cuda(),
               k_offsets=torch.from_numpy(p.offsets("k")).cuda(),
               prefix_lens=None if prefix is None else torch.tensor(prefix, dtype=torch.int32,
                                                                    device="cuda"))
    return p, a, x, off


def poison(a):
    for n in ("out", "lse", "dq", "dk", "dv", "grad_bias", "workspace"):
        t = getattr(a, n, None)
        if t is not None:
            t.view(torch.uint8).fill_(0xff)  # NaN in every type


def run(p, a, x, off):
    poison(a)
    a.forward(x["q"], x["k"], x["v"], **off)
    a.backward(x["q"], x["k"], x["v"], x["dout"], **off)
    torch.cuda.synchronize()


def check(p, a, x, off, dtype):
    run(p, a, x, off)
    ref = R.attention(p, x["q"], x["k"], x["v"], x["dout"])
    close(a.out, ref["out"], dtype, "out")
    close(a.lse, ref["lse"], F32, "lse")
    close(a.dq, ref["dq"], dtype, "dq", 1.25)
    close(a.dk, ref["dk"], dtype, "dk", 1.25)
    close(a.dv, ref["dv"], dtype, "dv", 1.25)
    if a.grad_bias is not None and p.table.shape[0] == 1:
        # one bucket for all keys: softmax does not notice it, the gradient is
        # exactly 0 and what remains is the rounding of terms that cancel
        assert a.grad_bias.abs().max().item() <= 2e-5 * ref["terms"]
    elif a.grad_bias is not None:
        close(a.grad_bias, ref["dtable"], F32, "dtable")


SHAPES = [
    # one token, one key; tiles just missed, met and passed; empty sequences
    dict(q_lens=[1]),
    dict(q_lens=[1, 0, 2, 31, 32, 33, 0, 63, 64, 65], heads=2, kv=1, buckets=5, reach=7, causal=True),
    dict(q_lens=[127, 128, 129, 5], heads=2, dim=128, buckets=32, reach=128, cap=15.0),
    dict(q_lens=[200, 1, 77], heads=3, kv=1, dim=40, causal=True, cap=5.0, buckets=9, reach=20),
    dict(q_lens=[300], heads=4, kv=2, dim=128, causal=True, buckets=32, reach=128),
    # prefixes of nothing, a part, all
    dict(q_lens=[100, 100, 100, 70], prefix=[0, 37, 100, 64], heads=2, dim=72, causal=True,
         buckets=11, reach=300, cap=8.0),
    # more queries than keys: the first ones see nothing; fewer; no keys at all
    dict(q_lens=[70, 5, 40, 3, 0, 130], k_lens=[30, 200, 0, 3, 17, 129], heads=2, kv=2, causal=True,
         buckets=13, reach=40),
    dict(q_lens=[70, 5, 40, 3, 0], k_lens=[30, 200, 0, 3, 17], heads=2, kv=1, dim=8, cap=2.0),
    # many short bags
    dict(q_lens=[(i * 7) % 41 for i in range(150)], heads=2, dim=64, buckets=32, reach=128),
    # reach 0: one bias for all; a table of one bucket
    dict(q_lens=[50, 90], heads=2, buckets=1, reach=0, causal=True),
    # the widest reach
    dict(q_lens=[1500], heads=1, dim=64, buckets=64, reach=1024, causal=True),
    dict(q_lens=[700, 130], heads=2, kv=1, dim=128, buckets=32, reach=16),
]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n", range(len(SHAPES)))
def test_shapes(n, dtype):
    print(f"\n[attn] shape {n} {SHAPES[n]} {dtype}", flush=True)
    check(*make(dtype=dtype, seed=n, **SHAPES[n]), dtype)


@pytest.mark.parametrize("layout", ["heads", "padded"])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_strides(layout, dtype):
    print(f"\n[attn] layout {layout} {dtype}", flush=True)
    check(*make([90, 33, 140], heads=4, kv=2, dim=56, causal=True, cap=10.0, buckets=16, reach=50,
                layout=layout, dtype=dtype), dtype)


def test_q_k_v_side_by_side():
    p, a, x, off = make([90, 33, 140], heads=4, kv=2, dim=64, dtype=BF16, causal=True)
    row = torch.cat([x["q"], x["k"], x["v"]], 1)
    x["q"], x["k"], x["v"] = row[:, :4], row[:, 4:6], row[:, 6:]
    check(p, a, x, off, BF16)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_large_scores(dtype):
    """Scores of several hundred: without the running maximum exp overflows;
    scores carry 2^-24 of their size, so probabilities lose that factor."""
    p, a, x, off = make([150, 64], heads=2, dim=64, dtype=dtype, causal=True, scale=3.0)
    run(p, a, x, off)
    ref = R.attention(p, x["q"], x["k"], x["v"])
    close(a.out, ref["out"], dtype, "out", 20.0 if dtype is F32 else 1.0)
    assert torch.isfinite(a.dq.float()).all() and torch.isfinite(a.dk.float()).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_masked_values_do_not_enter(bad, dtype):
    """Keys, values, queries and gradients that a row does not see hold NaN or
    infinities: its results are those of finite ones there, bit for bit."""
    n, at = 150, 100  # rows before `at` must not notice rows from `at` on
    p, a, x, off = make([n, 40], heads=2, kv=1, dim=64, dtype=dtype, causal=True, buckets=8, reach=9)
    run(p, a, x, off)
    keep = {s: getattr(a, s).clone() for s in ("out", "lse", "dq", "dk", "dv")}
    y = {s: t.clone() for s, t in x.items()}
    for s in ("k", "v"):
        y[s][at:n] = bad
    run(p, a, y, off)
    assert torch.equal(a.out[:at], keep["out"][:at])
    assert torch.equal(a.lse[:, :at], keep["lse"][:, :at])
    assert torch.equal(a.dq[:at], keep["dq"][:at])
    assert torch.isnan(a.out[at:n].float()).any(-1).all()
    for s in ("out", "dq", "dk", "dv"):  # the other sequence
        assert torch.equal(getattr(a, s)[n:], keep[s][n:]), s
    # queries before `at` are not seen by later keys' gradients
    y = {s: t.clone() for s, t in x.items()}
    y["q"][:at] = bad
    y["dout"][:at] = bad
    run(p, a, y, off)
    for s in ("dk", "dv"):
        assert torch.equal(getattr(a, s)[at:], keep[s][at:]), s
    assert torch.equal(a.out[at:], keep["out"][at:]) and torch.equal(a.dq[at:], keep["dq"][at:])


def test_repeats_bit_for_bit():
    p, a, x, off = make([333, 64, 500, 7], heads=4, kv=2, dim=128, dtype=BF16, causal=True, cap=9.0,
                        buckets=32, reach=128)
    run(p, a, x, off)
    keep = {s: getattr(a, s).clone() for s in ("out", "lse", "dq", "dk", "dv", "grad_bias")}
    for _ in range(3):
        run(p, a, x, off)
        for s, t in keep.items():
            assert torch.equal(getattr(a, s), t), s


@pytest.mark.parametrize("cap,causal", [(0.0, True), (3.0, False)])
def test_gradients_against_differences(cap, causal):
    """<gradient, direction> against central differences of the definition:
    step h = 1e-4 in 64 bits leaves an error of about h^2 = 1e-8 relative to
    third derivatives of order one; the kernel's fp32 gradients are within
    1e-5 of norms, and an inner product over n elements within 1e-5*sqrt(n) of
    an element's size: bound 2e-5 of |gradient| |direction|."""
    p, a, x, off = make([20, 9], heads=2, kv=1, dim=16, dtype=F32, causal=causal, cap=cap,
                        buckets=6, reach=8)
    run(p, a, x, off)
    grads = dict(q=a.dq, k=a.dk, v=a.dv, table=a.grad_bias)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    table = p.table.double()
    for name, g in grads.items():
        base = table if name == "table" else x[name].double()
        d = torch.randn(base.shape, generator=gen, device="cuda", dtype=torch.float64)
        d /= d.norm()
        loss = []
        for h in (1e-4, -1e-4):
            y = dict(q=x["q"].double(), k=x["k"].double(), v=x["v"].double())
            p.table = table
            if name == "table":
                p.table = table + h * d
            else:
                y[name] = base + h * d
            loss.append((R.attention(p, y["q"], y["k"], y["v"])["out"] * x["dout"].double()).sum())
        p.table = table
        want = ((loss[0] - loss[1]) / 2e-4).item()
        got = (g.double() * d).sum().item()
        print(f"  d{name}: {got:.6f} against {want:.6f}", flush=True)
        assert abs(got - want) <= 2e-5 * g.double().norm().item() + 1e-7


def test_forward_without_training_outputs():
    p, a, x, off = make([65, 3], heads=2, dim=64, dtype=BF16, causal=True, train=False)
    poison(a)
    a.forward(x["q"], x["k"], x["v"], **off)
    close(a.out, R.attention(p, x["q"], x["k"], x["v"])["out"], BF16, "out")


def test_other_stream_and_graph():
    """The calls on a stream of their own, then captured and replayed with
    eager work between the replays."""
    p, a, x, off = make([100, 30, 64], heads=2, dim=64, dtype=BF16, causal=True, buckets=8, reach=30)
    run(p, a, x, off)
    names = ("out", "dq", "dk", "dv", "grad_bias")
    keep = {s: getattr(a, s).clone() for s in names}
    side = torch.cuda.Stream()
    poison(a)
    side.wait_stream(torch.cuda.current_stream())
    a.forward(x["q"], x["k"], x["v"], stream=side, **off)
    a.backward(x["q"], x["k"], x["v"], x["dout"], stream=side, **off)
    side.synchronize()
    for s in names:
        assert torch.equal(getattr(a, s), keep[s]), s
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        a.forward(x["q"], x["k"], x["v"], **off)
        a.backward(x["q"], x["k"], x["v"], x["dout"], **off)
    for _ in range(3):
        poison(a)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for s in names:
            assert torch.equal(getattr(a, s), keep[s]), s


def test_offsets_past_2_31_elements():
    """Rows beyond 2^31 elements of one array."""
    heads, dim, n = 4, 128, 4_300_000  # 2.2e9 elements of bf16
    from paper_2010_13100_amd import tc
    big = torch.zeros((n, heads, dim), dtype=BF16, device="cuda")
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    big[-90:] = rows(gen, 90, heads, dim, BF16)
    lens = [n - 90, 90]
    # only the last sequence has queries
    off_k = torch.tensor([0, n - 90, n], dtype=torch.int32, device="cuda")
    off_q = torch.tensor([0, 0, 90], dtype=torch.int32, device="cuda")
    q = rows(gen, 90, heads, dim, BF16)
    a = tc.BagAttention(num_seqs=2, num_heads=heads, head_dim=dim, dtype=BF16, max_q=90, max_k=n,
                        total_q=90, total_k=n, causal=True)
    a.forward(q, big, big, off_q, off_k)
    p = R.Problem([90], [90], heads, heads, dim, causal=True)
    close(a.out, R.attention(p, q, big[-90:], big[-90:])["out"], BF16, "out")
    assert sum(lens) == n


# Batches that fill the chip, so that every kernel's own form is taken: tiles of
# 128 rows (long sequences) and 32 rows of several short sequences side by side.
MANY = [
    dict(q_lens=[700] * 8, heads=8, kv=4, dim=128, causal=True, cap=20.0, buckets=32, reach=128),
    dict(q_lens=[333, 900, 77, 650, 1000, 129], heads=12, kv=12, dim=64, buckets=16, reach=60,
         causal=True, prefix=[100, 0, 77, 300, 999, 5]),
    dict(q_lens=[500] * 4, k_lens=[300, 800, 500, 257], heads=16, kv=4, dim=72, causal=True),
    dict(q_lens=[(i * 13) % 61 for i in range(900)], heads=4, kv=2, dim=64, causal=True, buckets=32,
         reach=128, cap=6.0),
    dict(q_lens=[1 + i % 3 for i in range(6000)], heads=3, kv=3, dim=40, buckets=9, reach=4),
    # cross lengths: every sequence's keys are offset differently from its queries
    dict(q_lens=[(i * 7) % 50 for i in range(900)], k_lens=[(i * 11) % 43 for i in range(900)],
         heads=4, kv=4, dim=128, causal=True, buckets=12, reach=20),
    dict(q_lens=[(i * 7) % 40 for i in range(1200)], k_lens=[(i * 11) % 90 for i in range(1200)],
         heads=2, kv=1, dim=64, buckets=12, reach=20, causal=True,
         prefix=[(i * 5) % 60 for i in range(1200)]),
    # a wide reach with shared heads: sums by distance of one head at a time
    dict(q_lens=[60] * 1100, heads=8, kv=2, dim=64, causal=True, buckets=40, reach=1024),
]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n", range(len(MANY)))
def test_full_chip(n, dtype):
    print(f"\n[attn] many {n} {dtype}", flush=True)
    check(*make(dtype=dtype, seed=20 + n, **MANY[n]), dtype)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("lens", [[37] * 1000, [600] * 8], ids=["short", "long"])
def test_masked_values_do_not_enter_full_chip(lens, dtype):
    """As above where the chip is full: sequences beside a bad one, and rows
    before a bad key, keep their bits."""
    heads = 2 if lens[0] < 100 else 8
    p, a, x, off = make(lens, heads=heads, kv=heads // 2, dim=64, dtype=dtype, causal=True, buckets=8,
                        reach=9)
    run(p, a, x, off)
    keep = {s: getattr(a, s).clone() for s in ("out", "lse", "dq", "dk", "dv")}
    n, at = lens[0], lens[0] // 2  # sequence 3, keys from `at` on
    first, end = 3 * n, 4 * n
    y = {s: t.clone() for s, t in x.items()}
    for s in ("k", "v"):
        y[s][first + at:end] = float("nan")
    run(p, a, y, off)
    same = torch.ones(sum(lens), dtype=torch.bool, device="cuda")
    same[first + at:end] = False
    for s in ("out", "dq"):
        assert torch.equal(getattr(a, s)[same], keep[s][same]), s
    assert torch.equal(a.lse[:, same], keep["lse"][:, same])
    assert torch.isnan(a.out[~same].float()).any(-1).all()
    same[first:end] = False
    for s in ("dk", "dv"):
        assert torch.equal(getattr(a, s)[same], keep[s][same]), s
    y = {s: t.clone() for s, t in x.items()}
    y["q"][first:first + at] = float("inf")
    y["dout"][first:first + at] = float("nan")
    run(p, a, y, off)
    same[:] = True
    same[first:first + at] = False
    for s in ("out", "dq", "dk", "dv"):
        assert torch.equal(getattr(a, s)[same], keep[s][same]), s
