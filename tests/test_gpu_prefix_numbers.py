"""Numbers of prefixes and blocks beyond 32 bits are refused, not cut down to ones that the library would take."""
import pytest
import torch

from paper_2603_27138_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_prefix,blocks", [(2 ** 32 + 1, 4), (1, 2 ** 32 + 4), (-2 ** 32 + 1, 4), (2 ** 63, 4)])
@pytest.mark.parametrize("recorded", [False, True])
def test_beyond_32_bits(n_prefix, blocks, recorded):
    i32 = dict(dtype=torch.int32, device="cuda")
    ctx, of, length = torch.zeros(2, **i32), torch.zeros(2, **i32), torch.full((1,), 50, **i32)
    p = B.make_problem(2, 4, 1, 64, 16, B.BF16, 4, 1, ctx)
    plan, ws = B.alloc_prefix_plan(p, 1), B.alloc_workspace(p)
    before = plan.fill_(0x5a).clone()
    k = torch.zeros(4, 16, 64, dtype=torch.bfloat16, device="cuda")
    q, out = (torch.zeros(2, 4, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.arange(4, **i32).view(1, 1, 4)

    def call(f, *args):
        with pytest.raises(B.ScoutError):
            B.prepare(f, *args)() if recorded else f(*args)

    call(B.prefix_plan, p, n_prefix, blocks, of, length, plan)
    call(B.shared_prefix_attn, p, n_prefix, blocks, plan, q, k, k, 4, table, None, None, None, None, None, None, out, None, ws)
    if blocks == 4:
        with pytest.raises(B.ScoutError):
            B.prefix_plan_bytes(p, n_prefix)
    torch.cuda.synchronize()
    assert torch.equal(plan, before)
