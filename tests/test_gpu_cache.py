"""The paged cache: rows written (8 bits or as they are) and read back, and
attention over it, against the definition in 64 bits. Stored codes and
exponents have to be equal; read values exactly what the codes stand for."""
import numpy as np
import pytest
import torch

from tests import attn_reference as R
from tests.test_gpu_attn import BF16, F32, close, rows

pytestmark = pytest.mark.gpu


def pages(lens, page_size, seed=0, spare=2, width=0):
    """A page table over pages in random order; unused entries are -1."""
    g = np.random.default_rng(seed)
    counts = [-(-n // page_size) for n in lens]
    order = g.permutation(sum(counts) + spare)
    table = np.full((len(lens), max(max(counts, default=0), 1) + width), -1, np.int32)
    at = 0
    for b, c in enumerate(counts):
        table[b, :c] = order[at:at + c]
        at += c
    return torch.from_numpy(table).cuda(), sum(counts) + spare


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def offsets(lens):
    return ints([0] + list(np.cumsum(lens)))


def slots(table, lens, new, page_size):
    """(page, slot) of every new row."""
    t = table.cpu().numpy()
    return [(t[b, p // page_size], p % page_size) for b, (n, m) in enumerate(zip(lens, new))
            for p in range(n - m, n)]


@pytest.mark.parametrize("dim,heads,page", [(128, 8, 16), (64, 1, 5), (8, 3, 1), (72, 2, 64)])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("kind", ["fp8", "same"])
def test_write_and_read(dim, heads, page, dtype, kind):
    from paper_2010_13100_amd import tc
    print(f"\n[cache] {dim} {heads} {page} {dtype} {kind}", flush=True)
    lens, new = [1, 70, 33, 5, 200], [1, 7, 33, 0, 130]
    table, n = pages(lens, page, seed=dim)
    c = tc.PagedCache.empty(n, page, heads, dim, torch.float8_e4m3fn if kind == "fp8" else dtype)
    store = dict(k=c.k, v=c.v)
    for t in store.values():
        t.view(torch.uint8).fill_(0x55)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(dim + page)
    total = sum(new)
    x = {s: rows(gen, total, heads, dim, dtype) for s in "kv"}
    # rows of every magnitude, zeros, subnormals, ties, and a row at the limit
    for s in "kv":
        power = torch.randint(-130, 120, (total, heads, 1), generator=gen, device="cuda")
        x[s] = (x[s].double() * torch.exp2(power.double())).to(dtype)
        x[s][0] = 0
        x[s][1, 0] = 448.0 * 2.0 ** -3
        x[s][2, 0, : 8] = torch.tensor([448.0, 17.0, 19.0, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10, -1.0625, -0.0],
                                       device="cuda").to(dtype)
        x[s][3, 0, 0] = 1.75 * 2.0 ** 90
        x[s][4, 0, 0] = 1.7578125 * 2.0 ** 90
    c.write(x["k"], x["v"], offsets(new), table, ints(lens))
    back = {s: torch.full_like(x[s], 7.0) for s in "kv"}
    c.read(back["k"], back["v"], offsets(new), table, ints(lens))
    where = slots(table, lens, new, page)
    p, s = np.array([w[0] for w in where]), np.array([w[1] for w in where])
    for name, exp in (("k", c.k_exp), ("v", c.v_exp)):
        got = store[name].view(torch.uint8 if kind == "fp8" else dtype)[p, s]
        if kind == "same":
            assert torch.equal(got, x[name]) and torch.equal(back[name], x[name])
            continue
        code, e = R.quantise_rows(x[name].double().cpu().numpy())
        assert np.array_equal(exp[p, s].cpu().numpy(), e)
        assert np.array_equal(got.cpu().numpy(), code)
        value = R.e4m3_value(code) * 2.0 ** (e[..., None].astype(np.float64) - 127)
        want = torch.from_numpy(value).cuda().to(dtype)
        assert torch.equal(back[name], want)
        assert torch.equal(torch.signbit(back[name]), torch.signbit(x[name]))
    # slots that no row went to are as they were
    untouched = np.ones((n, page), bool)
    untouched[p, s] = False
    for t in store.values():
        assert (t.view(torch.uint8)[torch.from_numpy(untouched).cuda()] == 0x55).all()


def test_rows_that_are_not_finite():
    from paper_2010_13100_amd import tc
    c = tc.PagedCache.empty(1, 4, 2, 64)
    k = torch.ones((3, 2, 64), dtype=BF16, device="cuda")
    k[0, 0, 63], k[1, 1, 5], k[2, 0, 9] = float("nan"), float("inf"), -float("inf")
    table = ints([[0]])
    c.write(k, k, offsets([3]), table, ints([3]))
    a, b = torch.empty_like(k), torch.empty_like(k)
    c.read(a, b, offsets([3]), table, ints([3]))
    bad = ~torch.isfinite(k.float()).all(-1)
    assert torch.equal(torch.isnan(a.float()).all(-1), bad) and torch.equal(a[~bad], k[~bad])
    assert (c.k_exp[0, :3][bad] == 255).all()


def test_rows_without_a_place():
    """Rows before position 0 and past the page table are left out when
    writing, zeros when read; nothing else is touched."""
    from paper_2010_13100_amd import tc
    c = tc.PagedCache.empty(3, 4, 1, 16, BF16)
    c.k.fill_(3.0)
    c.v.fill_(3.0)
    table = ints([[0], [1]])  # room for 4 positions each; page 2 is nobody's
    gen = torch.Generator(device="cuda")
    gen.manual_seed(0)
    k = rows(gen, 11, 1, 16, BF16)
    # sequence 0: 5 rows end at position 3 (the first is before 0);
    # sequence 1: 6 rows end at position 7 (the last four are past the table)
    c.write(k, k, offsets([5, 6]), table, ints([4, 8]))
    assert torch.equal(c.k[0, :, 0], k[1:5, 0]) and torch.equal(c.k[1, 2:, 0], k[5:7, 0])
    assert (c.k[1, :2] == 3.0).all() and (c.k[2] == 3.0).all()
    a, b = torch.full_like(k, 9.0), torch.full_like(k, 9.0)
    c.read(a, b, offsets([5, 6]), table, ints([4, 8]))
    want = k.clone()
    want[0] = 0
    want[7:] = 0
    assert torch.equal(a, want) and torch.equal(b, want)


PAGED = [
    # single tokens over short and long histories, page sizes that end inside tiles
    dict(lens=[1, 2, 31, 32, 33, 400, 1000], new=1, heads=8, kv=8, dim=128, page=16),
    dict(lens=[700, 1, 63, 129], new=1, heads=8, kv=1, dim=64, page=5, cap=10.0, buckets=16, reach=40),
    dict(lens=[3000, 5, 260], new=1, heads=4, kv=2, dim=128, page=64, buckets=32, reach=128),
    dict(lens=[300, 77], new=1, heads=40, kv=1, dim=72, page=1, buckets=32, reach=128),
    # chunks, some as long as their history, one token apart from it
    dict(lens=[200, 64, 65, 1000], new=[200, 64, 64, 3], heads=4, kv=2, dim=128, page=16, cap=20.0,
         buckets=32, reach=128),
    dict(lens=[500, 90, 0, 7], new=[130, 1, 0, 7], heads=6, kv=2, dim=40, page=7, buckets=9, reach=30),
    dict(lens=[5000, 300], new=[70, 33], heads=2, kv=1, dim=64, page=256, mask="full"),
    dict(lens=[150, 90], new=[40, 90], heads=2, kv=1, dim=64, page=16, prefix=[140, 50], buckets=9,
         reach=30),
    # more queries than the cache holds: the first ones see nothing
    dict(lens=[3, 0, 40], new=[10, 2, 50], heads=2, kv=2, dim=64, page=8),
]


@pytest.mark.parametrize("kind", ["fp8", "same"])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n", range(len(PAGED)))
def test_paged_attention(n, dtype, kind):
    from paper_2010_13100_amd import tc
    s = dict(PAGED[n])
    print(f"\n[paged] {n} {s} {dtype} {kind}", flush=True)
    lens = s["lens"]
    new = [s["new"]] * len(lens) if isinstance(s["new"], int) else s["new"]
    heads, kv, dim, page = s["heads"], s["kv"], s["dim"], s["page"]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(n)
    table, num = pages(lens, page, seed=n, width=n % 2)
    ctype = torch.float8_e4m3fn if kind == "fp8" else dtype
    c = tc.PagedCache.empty(num, page, kv, dim, ctype)
    for t in (c.k, c.v, c.k_exp, c.v_exp):
        if t is not None:
            t.view(torch.uint8).fill_(0xff)  # slots that hold no row: NaN
    full = sum(lens)
    k, v = (rows(gen, full, kv, dim, dtype) for _ in range(2))
    c.write(k, v, offsets(lens), table, ints(lens))
    c.read(k, v, offsets(lens), table, ints(lens))  # the values that the cache holds
    q = rows(gen, sum(new), heads, dim, dtype, sigma=1.5)
    bias = bucket_of = None
    if s.get("buckets"):
        bias = torch.randn((s["buckets"], heads), generator=gen, device="cuda") * 0.7
        bucket_of = torch.randint(0, s["buckets"], (2 * s["reach"] + 1,), generator=gen,
                                  device="cuda", dtype=torch.int32)
    causal = s.get("mask") != "full"
    prefix = s.get("prefix")
    a = tc.BagAttention(num_seqs=len(lens), num_heads=heads, num_kv_heads=kv, head_dim=dim,
                        dtype=dtype, max_q=max(new), max_k=max(lens), total_q=sum(new),
                        causal=causal, cap=s.get("cap", 0.0), bias_table=bias,
                        bucket_of=bucket_of, paged=True)
    a.out.view(torch.uint8).fill_(0xff)
    if a.workspace is not None:
        a.workspace.fill_(0xff)
    a.lse = torch.full((heads, sum(new)), float("nan"), device="cuda")
    a.forward_paged(q, c, offsets(new), table, ints(lens),
                    prefix_lens=None if prefix is None else ints(prefix))
    p = R.Problem(new, lens, heads, kv, dim, causal, prefix, None, s.get("cap", 0.0), bias, bucket_of)
    ref = R.attention(p, q, k, v)
    close(a.out, ref["out"], dtype, "out")
    close(a.lse, ref["lse"], F32, "lse")
    keep = a.out.clone()
    a.forward_paged(q, c, offsets(new), table, ints(lens),
                    prefix_lens=None if prefix is None else ints(prefix))
    assert torch.equal(a.out, keep)


def test_heads_outermost_cache():
    """A cache whose pages hold [head][slot] rows, through a view."""
    from paper_2010_13100_amd import tc
    lens, page, kv, dim = [100, 37], 16, 2, 64
    table, num = pages(lens, page)
    c = tc.PagedCache(*(torch.full((num, kv, page, dim), float("nan"), dtype=BF16,
                                   device="cuda").transpose(1, 2) for _ in range(2)))
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    k, v = (rows(gen, sum(lens), kv, dim, BF16) for _ in range(2))
    c.write(k, v, offsets(lens), table, ints(lens))
    q = rows(gen, 2, 4, dim, BF16)
    a = tc.BagAttention(num_seqs=2, num_heads=4, num_kv_heads=kv, head_dim=dim, max_q=1, max_k=100,
                        total_q=2, causal=True, paged=True)
    a.forward_paged(q, c, offsets([1, 1]), table, ints(lens))
    p = R.Problem([1, 1], lens, 4, kv, dim, causal=True)
    close(a.out, R.attention(p, q, k, v)["out"], BF16, "out")


def test_cache_past_2_31_elements():
    from paper_2010_13100_amd import tc
    page, kv, dim = 64, 8, 128
    num = (1 << 31) // (page * kv * dim) + 8
    c = tc.PagedCache.empty(num, page, kv, dim, torch.float8_e4m3fn)
    assert c.k.numel() > 1 << 31
    lens = [130, 64]
    table = ints([[num - 1, 3, num - 4], [num - 2, -1, -1]])
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    k, v = (rows(gen, sum(lens), kv, dim, BF16) for _ in range(2))
    c.write(k, v, offsets(lens), table, ints(lens))
    c.read(k, v, offsets(lens), table, ints(lens))
    assert torch.isfinite(k.float()).all()
    q = rows(gen, 2, 8, dim, BF16)
    a = tc.BagAttention(num_seqs=2, num_heads=8, head_dim=dim, max_q=1, max_k=130, total_q=2,
                        causal=True, paged=True)
    a.forward_paged(q, c, offsets([1, 1]), table, ints(lens))
    p = R.Problem([1, 1], lens, 8, 8, dim, causal=True)
    close(a.out, R.attention(p, q, k, v)["out"], BF16, "out")
