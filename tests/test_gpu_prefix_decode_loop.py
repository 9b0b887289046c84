"""Answers to prompts that stay in the cache, decoded together: slots reserved, tokens appended, the prompts attended to once for all of
their answers, each answer's own tokens by scout_layer_step with that partial, beams dropped and forked, the pool compacted.  Every step's
output against attention over all of a sequence's tokens in 64 bits."""
import math

import pytest
import torch

from paper_2603_27138_amd import binding as B

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype,d,S,G,n", [(BF16, 128, 16, 4, 6), (BF16, 128, 32, 8, 20), (BF16, 64, 16, 8, 40), (F32, 64, 16, 2, 5)])
def test_sampling_loop(dtype, d, S, G, n):
    gen = torch.Generator().manual_seed(n)
    Hkv, mb = 2, 12
    Hq, prompts = G * Hkv, [7 * S + 5, 3 * S]
    P, rows = len(prompts), n + len(prompts)
    i32 = dict(dtype=torch.int32, device="cuda")
    randn = lambda *shape: torch.randn(*shape, generator=gen).to(dtype)  # noqa: E731
    n_slots = sum(-(-x // S) for x in prompts) * Hkv + n * Hkv * 3 + 9
    k_pool, v_pool = (torch.full((n_slots, S, d), math.nan, dtype=dtype, device="cuda") for _ in range(2))
    table = torch.full((rows, Hkv, mb), -1, **i32)
    ctx = torch.full((rows,), -1, **i32)
    digest = torch.zeros(rows, Hkv, mb, 2, d, dtype=dtype, device="cuda")
    history = [None] * rows   # what each row's sequence holds: (keys, values) [tokens][Hkv][d] on the CPU
    slots = torch.randperm(n_slots, generator=gen).tolist()
    for r, length in enumerate(prompts):
        k, v = randn(length, Hkv, d), randn(length, Hkv, d)
        history[n + r] = (k, v)
        ctx[n + r] = length
        for g in range(Hkv):
            for j in range(-(-length // S)):
                s = slots.pop()
                table[n + r, g, j] = s
                part = slice(j * S, min(length, (j + 1) * S))
                k_pool[s, :part.stop - part.start] = k[part, g].cuda()
                v_pool[s, :part.stop - part.start] = v[part, g].cuda()
    code = B.BF16 if dtype == BF16 else B.F32
    every = B.make_problem(rows, Hq, Hkv, d, S, code, mb, mb, ctx)
    answers = B.make_problem(n, Hq, Hkv, d, S, code, mb, mb, ctx)
    pages = B.alloc_pages(n_slots)
    B.pages_init(every, ctx, table, n_slots, pages)
    ctx[:n] = 0   # answers begin without tokens of their own
    for b in range(n):
        history[b] = (randn(0, Hkv, d), randn(0, Hkv, d))
    of = torch.tensor([b % 3 - 1 if b % 3 < 2 else 1 for b in range(n)], **i32)   # some have no prompt
    prefix_len = ctx[n:].clone()
    ws, plan = B.alloc_workspace(answers), B.alloc_prefix_plan(answers, P)
    f32 = dict(dtype=F32, device="cuda")
    o, m, l = torch.empty(n, Hq, d, **f32), torch.empty(n, Hq, **f32), torch.empty(n, Hq, **f32)
    lists = [torch.full((n, Hkv, mb), -1, **i32) for _ in range(3)]
    n_gpu, n_host = torch.zeros(n, Hkv, **i32), torch.zeros(n, Hkv, **i32)
    sel_host = torch.full((n, Hkv, mb), -1, **i32)
    out, lse = torch.empty(n, Hq, d, dtype=dtype, device="cuda"), torch.empty(n, Hq, **f32)
    new_slot, short = torch.empty(n, Hkv, **i32), torch.empty(1, **i32)
    cache = (ctx, digest, table, k_pool, v_pool, n_slots, pages)
    for step in range(2 * S + 3):
        if step in (S // 2, S + 3):   # beams: every third answer gives way to a fork of another one
            losers = list(range(1, n, 3))
            winners = [(b + 1) % n if (b + 1) % n not in losers else 0 for b in losers]
            B.free_sequences(every, torch.tensor(losers, **i32), ctx, table, n_slots, pages)
            status = torch.empty(len(losers), **i32)
            B.fork_sequences(every, torch.tensor(winners, **i32), torch.tensor(losers, **i32), step > S, *cache, status)
            assert not status.any()
            for a, b in zip(winners, losers):
                history[b] = tuple(x.clone() for x in history[a])
                of[b] = of[a]
        if step in (S + 1, S + 4):
            slot_map, live = torch.empty(n_slots, **i32), torch.empty(1, **i32)
            B.compact_pool(every, table, k_pool, v_pool, n_slots, pages, slot_map, live)
            assert int(table.max()) < live.item()
        if step in (0, S // 2, S + 3):
            B.prefix_plan(answers, P, mb, of, prefix_len, plan)
        q, k_new, v_new = randn(n, Hq, d), randn(n, Hkv, d), randn(n, Hkv, d)
        qd = q.cuda()
        B.reserve_blocks(answers, ctx, n_slots, pages, new_slot, short)
        B.append_token(answers, ctx, k_new.cuda(), v_new.cuda(), new_slot, digest, table, k_pool, v_pool, n_slots)
        B.shared_prefix_attn(answers, P, mb, plan, qd, k_pool, v_pool, n_slots, table[n:], None, None, None, o, m, l, None, None, ws)
        B.layer_step(answers, qd, digest, table, k_pool, v_pool, n_slots, o, m, l, None, lists[0], lists[1], lists[2], n_gpu, sel_host, n_host,
                     out, lse, ws)
        torch.cuda.synchronize()
        assert short.item() == 0 and not n_host.any()
        for b in range(n):
            history[b] = (torch.cat([history[b][0], k_new[b:b + 1]]), torch.cat([history[b][1], v_new[b:b + 1]]))
        held = (table >= 0).sum().item()
        assert int(pages[:n_slots].sum()) == held
        if step % 4 and step not in (S // 2, S // 2 + 1, S + 1, S + 3, S + 4):
            continue
        for b in range(n):
            p = int(of[b])
            keys, vals = history[b] if p < 0 else tuple(torch.cat([x, y]) for x, y in zip(history[n + p], history[b]))
            for h in range(Hq):
                x = keys[:, h // G].double() @ q[b, h].double() / math.sqrt(d)
                w = torch.softmax(x, 0)
                v = vals[:, h // G].double()
                want, size = w @ v, w @ v.abs()
                # weights of the answer's own part are rounded to bf16 for d = 128 (2^-8), all else is far below; out itself by 2^-8
                tol = (2 * 2.0 ** -8 * size + 2.0 ** -8 * want.abs()) if dtype == BF16 else 2e-6 * (size + want.abs())
                assert bool(((out[b, h].double().cpu() - want).abs() <= tol).all()), (step, b, h)
                assert abs(float(lse[b, h]) - float(torch.logsumexp(x, 0))) < (2.0 ** -8 if dtype == BF16 else 1e-5)
