"""How exactly softmax weights enter the value products of the attention over shared prefixes: the same for every number of rows that a
batch gives a prefix, whatever is written of the result.

A weight goes as bf16 terms.  d = 128: two.  The first one is cut (7 explicit bits: what is left is below 2^-7 of the weight), the second one
rounded (2^-8 of what is left): 2^-15 of the weight at the most.  d = 64: three, the first two of them cut: 2^-22."""
import math

import pytest
import torch

from tests.test_gpu_shared_prefix import BF16, F32, U, Batch, _of

pytestmark = pytest.mark.gpu
TERMS = {128: 2.0 ** -15, 64: 2.0 ** -22}
COUNTS = [2, 6, 12, 30, 70]   # sequences of 8 heads over two prefixes: tiles of 16, 32, 64, 128 and 256 rows


def _near(got, want, bound):
    got = got.double().cpu()
    same = (got == want) & torch.isinf(want)
    off = torch.where(same, torch.zeros_like(want), (got - want).abs())
    assert bool((off <= bound).all()), (float((off - bound).max()), float(off.max()))


def _check(b, other=True):
    """An output is a mean of values with these weights: its error is at most twice the weights' (numerator and sum) times the mean of
    the |v|; `out` is rounded by half a step of bf16."""
    out, lse, mean_v, err = b.want(other)
    weights = 2 * (err + TERMS[b.d])[..., None] * mean_v + 1e-30
    lse_bound = 2 * err + 8 * U * lse.abs().nan_to_num(posinf=0.0)
    if b.out is not None:
        _near(b.out, out, weights + 2.0 ** -8 * out.abs())
        _near(b.lse, lse, lse_bound)
    if b.o is not None:
        _near(b.o, out, weights + 4 * U * out.abs())
        _near(b.m.double().cpu() + b.l.double().cpu().log(), lse, lse_bound)


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("n", COUNTS)
@pytest.mark.parametrize("lens", [[3, 40], [1500, 131]])
def test_every_tile_of_rows(d, n, lens):
    """A few tokens, whose values do not average out; several tiles of tokens, the last of them not full.  The result alone, the joined
    partial alone, both."""
    b = Batch(n + d, BF16, d, 32, 8, 2, lens, _of(2, n), p_host=0.2 if lens[0] > 1000 else 0.0)
    for partial, result, other in ((False, True, True), (True, False, True), (True, True, False)):
        _check(b.run(partial=partial, result=result, other=other), other)


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("n", [3, 10, 20, 40])
def test_weights_above_one(d, n):
    """Queries ten times as long: sums are kept relative to a number that may lie far below a later maximum."""
    b = Batch(n, BF16, d, 32, 8, 1, [2000], [0] * n, sharp=10.0)
    _check(b.run(partial=True))
    _check(b.run())


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("n", COUNTS)
def test_terms_of_a_weight(d, n):
    """Three tokens whose logits are single products, which binary32 holds exactly, and values that read one weight each.  What is left beside
    the terms: a logit x (below 6) is scaled and shifted, 3 roundings of 1.45 |x|, the exponential 2, sums of three numbers, the fold and the
    division 8: 36 u."""
    b = Batch(n, BF16, d, 32, 8, 2, [3, 3], _of(2, n), other=False, scale=0.125)
    gen = torch.Generator().manual_seed(n)
    b.q = torch.zeros(b.q.shape, dtype=BF16)
    b.q[..., 5] = (4 * torch.rand(n, b.Hq, generator=gen) + 1).to(BF16)
    for p in range(2):
        for g in range(b.Hkv):
            s = int(b.table[p, g, 0])
            b.k[s, :3] = 0.0
            b.k[s, :3, 5] = torch.tensor([3.0, -4.0, 1.0 + p]).to(BF16)
            b.v[s, :3] = torch.eye(3, d).to(BF16)
    b.k_dev, b.v_dev = b.k.cuda(), b.v.cuda()
    b.run(partial=True)
    want = b.want()[0]
    assert float(want[..., :3].max()) > 0.6
    has = torch.tensor([p >= 0 for p in b.of])
    assert bool((want[has][..., :3] > 0).all())
    _near(b.o, want, (TERMS[d] + 36 * U) * want)


def test_fp32_keeps_its_weights_whole():
    b = Batch(5, F32, 64, 16, 8, 1, [3, 700], _of(2, 30))
    b.run(partial=True).check()
    assert math.isfinite(float(b.o.abs().max()))


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("n", COUNTS)
def test_large_values_without_weight(d, n):
    """The largest finite value of tokens whose logits are 400 below the others': their weights are zero in binary32 and below 2^-577 in
    truth, and nothing of the value may be seen."""
    b = Batch(n, BF16, d, 32, 8, 2, [40, 300], _of(2, n), scale=0.125)
    b.q = torch.zeros(b.q.shape, dtype=BF16)
    b.q[..., 5] = 4.0
    b.k = torch.where(b.k.isnan(), b.k, torch.zeros_like(b.k))
    for p, tokens in ((0, (7, 33)), (1, (0, 130, 299))):
        for g in range(b.Hkv):
            for t in tokens:
                s = int(b.table[p, g, t // 32])
                b.k[s, t % 32, 5] = -800.0
                b.v[s, t % 32] = torch.finfo(BF16).max
    b.k_dev, b.v_dev = b.k.cuda(), b.v.cuda()
    _check(b.run(partial=True))
    _check(b.run())
