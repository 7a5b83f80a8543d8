"""How exact the gradients of short bags are, over all entries together, where a
rounding too many shows: few keys leave no average over terms."""
import pytest
import torch

from tests import test_gpu_attn as A

pytestmark = pytest.mark.gpu


def off(got, want):
    want = want.double().cpu()
    return float((got.double().cpu() - want).norm() / want.norm())


@pytest.mark.parametrize("lens", [[2] * 40, [11] * 60, [3, 9, 17, 31, 32] * 12])
@pytest.mark.parametrize("dim", [64, 128])
def test_capped_scores_far_below_the_cap(lens, dim):
    """fp32: scores of a few units under a cap of 50 carry some 2^-24 of
    themselves, so weights and what is made of them are 1e-6 off at most."""
    print(f"\n[attn] cap 50, {len(lens)} bags of {lens[:5]}, {dim}", flush=True)
    p, a, x, offsets = A.make(lens, heads=2, dim=dim, dtype=A.F32, causal=True, cap=50.0, seed=5)
    A.run(p, a, x, offsets)
    ref = A.R.attention(p, x["q"], x["k"], x["v"], x["dout"])
    for name in ("out", "dq", "dk", "dv"):
        assert off(getattr(a, name), ref[name]) <= 1e-6, name


@pytest.mark.parametrize("lens", [[2] * 40, [11] * 60, [3, 9, 17, 31, 32] * 12])
@pytest.mark.parametrize("dim", [64, 128])
def test_bf16_gradients_err_by_two_roundings(lens, dim):
    """A rounding to bf16 errs by at most 2^-9 of a value, evenly spread by
    2^-9 / sqrt 3 times a mean of 1.5 over a binade: 0.0017. Two of them, of the terms
    and of the result, are 0.0024; a fifth more for the samples' spread."""
    print(f"\n[attn] bf16, {len(lens)} bags of {lens[:5]}, {dim}", flush=True)
    p, a, x, offsets = A.make(lens, heads=2, dim=dim, dtype=A.BF16, causal=True, seed=6)
    A.run(p, a, x, offsets)
    ref = A.R.attention(p, x["q"], x["k"], x["v"], x["dout"])
    for name in ("dq", "dk", "dv"):
        assert off(getattr(a, name), ref[name]) <= 0.0029, name
