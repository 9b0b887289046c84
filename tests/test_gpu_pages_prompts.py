"""A prompt joins a cache whose sequences share slots: it takes the slots of all its blocks from reserve_blocks, and is forked, freed and
compacted as any other."""
import numpy as np
import pytest
import torch

from paper_2603_27138_amd import binding as B
from tests.test_gpu_pages import Cache

pytestmark = pytest.mark.gpu


def _admit(c, b, length):
    """The prompt becomes sequence b of length tokens; the blocks for which no slot was left are -1."""
    nb, i32 = -(-length // c.S), dict(dtype=torch.int32, device="cuda")
    zeros, new, short = torch.zeros(nb, **i32), torch.full((nb, c.Hkv), 77, **i32), torch.full((1,), 77, **i32)
    p = B.make_problem(nb, c.p.Hq, c.Hkv, c.p.d, c.S, c.p.dtype, c.mb, 1, zeros)
    B.reserve_blocks(p, zeros, c.n_slots, c.pages, new, short)
    c.table[b, :, :nb] = new.t()
    c.ctx[b] = length
    bk = c.book
    got = bk.take(nb * c.Hkv)
    bk.table[b, :, :nb] = np.array([-1 if s is None else s for s in got], np.int32).reshape(nb, c.Hkv).T
    bk.ctx[b] = length
    assert short.item() == got.count(None)
    c.check(("admit", b, length))


@pytest.mark.parametrize("dtype,Hkv,S,d,n_slots", [(torch.bfloat16, 2, 32, 128, 400), (torch.float32, 3, 16, 64, 61), (torch.bfloat16, 1, 16, 64, 0)])
def test_prompts_come_and_go(dtype, Hkv, S, d, n_slots):
    rng = np.random.default_rng([Hkv, S, n_slots])
    c = Cache(rng, 6, Hkv, S, d, dtype, 9, n_slots, [4 * S + 3, -1, 2 * S, -1, -1, -1])
    _admit(c, 1, 9 * S)            # as long as a row
    c.fork([1, 0], [3, 4])
    c.free([0, 2])
    c.compact()
    _admit(c, 0, 1)
    _admit(c, 2, 5 * S + 1)        # in the slots that became free
    c.fork([2], [5], deep=True)
    c.advance()
    c.check("append")
    c.free([1, 2, 3])
    c.compact()
    c.free([0, 4, 5])
    assert not c.book.refs.any()
    c.check("all given back")


def test_a_prompt_of_many_blocks():
    """More blocks than a sequence of the batch may have heads for: 65 000 takers in one call."""
    n, Hkv, n_slots = 8125, 8, 70_000
    i32 = dict(dtype=torch.int32, device="cuda")
    zeros, new, short = torch.zeros(n, **i32), torch.empty(n, Hkv, **i32), torch.empty(1, **i32)
    p = B.make_problem(n, Hkv, Hkv, 64, 16, B.BF16, 1, 1, zeros)
    pages, table = B.alloc_pages(n_slots), torch.full((1, Hkv, 16384), -1, **i32)
    ctx = torch.full((1,), -1, **i32)
    B.pages_init(B.make_problem(1, Hkv, Hkv, 64, 16, B.BF16, 16384, 1, ctx), ctx, table, n_slots, pages)
    B.reserve_blocks(p, zeros, n_slots, pages, new, short)
    assert short.item() == 0 and torch.equal(new.view(-1), torch.arange(n * Hkv, **i32))
    assert torch.equal(pages[:n_slots], (torch.arange(n_slots, device="cuda") < n * Hkv).to(torch.int32))
    B.reserve_blocks(p, zeros, n_slots, pages, new, short)
    left = n_slots - n * Hkv
    assert short.item() == n * Hkv - left
    assert torch.equal(new.view(-1)[:left], torch.arange(n * Hkv, n_slots, **i32)) and bool((new.view(-1)[left:] == -1).all())
