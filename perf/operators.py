"""Sequences that share a long prefix: attention over the prefix computed once for all of them, and the pages of the cache that
such sequences share, copy, give back and move together.

A case is a dict of plain values:

  kind        "attend"    one decode step of a batch over its shared prefixes: the plan of who shares what, made once, and
                          shared_prefix_attn on every layer, merged with what each sequence attended to of its own
              "samples"   answers to prompts that stay in the cache: the old ones are freed, new ones forked from the prompts,
                          slots reserved for the blocks they open, and their first token appended
              "churn"     answers that own their tiles (a recall moves blocks in and out of them): the older half leaves, the
                          pool is compacted, new ones are copied from the prompts, and the same for the other half
  Hq, Hkv, d, S, dtype        as in scout_problem
  len_lo, len_hi   tokens of a prefix or prompt, uniform in [len_lo, len_hi]; the first one has len_hi
  prefixes    how many of them there are
  B           sequences of the batch ("attend") or answers ("samples", "churn")
  alone       share of the sequences of an "attend" batch that have no prefix
  other       whether each sequence's own part (o, m, l) is merged in
  p_host      share of the blocks that live on the host (no slot: not attended to, not copied)
  layers      layers that a pass goes through, each with a cache of its own

`own` says whether run() computes the plain form or calls the library.
"""
import math

import torch

own = False

PLANTED = 0.05  # share of blocks whose keys point along the batch's queries


def listed():
    c8b = dict(Hq=32, Hkv=8, d=128, S=32, dtype="bf16")
    c32b = dict(Hq=64, Hkv=8, d=128, S=32, dtype="bf16")
    return [
        # the repository's smallest shape: three answers to a prompt of a few blocks, fp32; latency is all there is
        dict(name="attend_tiny_f32", kind="attend", B=3, Hq=4, Hkv=1, d=64, S=16, dtype="f32", prefixes=1, len_lo=117, len_hi=117,
             alone=0.0, other=1, p_host=0.0, layers=1),
        # four answers to one question over a document of 8k tokens: few rows, all of it reading
        dict(name="attend_4", kind="attend", B=4, prefixes=1, len_lo=8192, len_hi=8192, alone=0.0, other=1, p_host=0.0, layers=4, **c8b),
        # the headline batch, all with the same 32k tokens in front
        dict(name="attend_16", kind="attend", B=16, prefixes=1, len_lo=32768, len_hi=32768, alone=0.0, other=1, p_host=0.0, layers=2, **c32b),
        # many answers to one long prompt: 512 rows for each KV head, as much arithmetic as reading and more
        dict(name="attend_64", kind="attend", B=64, prefixes=1, len_lo=32768, len_hi=32768, alone=0.0, other=1, p_host=0.0, layers=2, **c32b),
        # a serving batch: five system prompts of unequal lengths, some requests without one, a quarter of the blocks on the host,
        # groups of five heads
        dict(name="attend_ragged", kind="attend", B=48, Hq=40, Hkv=8, d=128, S=32, dtype="bf16", prefixes=5, len_lo=1000, len_hi=24001,
             alone=0.15, other=1, p_host=0.25, layers=2),
        # heads of 64 channels, blocks of 16 tokens, nothing of the sequences' own yet
        dict(name="attend_heads_of_64", kind="attend", B=24, Hq=32, Hkv=8, d=64, S=16, dtype="bf16", prefixes=2, len_lo=12000, len_hi=16384,
             alone=0.0, other=0, p_host=0.0, layers=2),
        # fp32 cache
        dict(name="attend_f32", kind="attend", B=8, Hq=16, Hkv=4, d=128, S=32, dtype="f32", prefixes=1, len_lo=8191, len_hi=8191, alone=0.0,
             other=1, p_host=0.0, layers=1),
        # a few answers to a short prompt: launches and little else
        dict(name="samples_4", kind="samples", B=4, Hq=4, Hkv=1, d=64, S=16, dtype="f32", prefixes=1, len_lo=2039, len_hi=2039, p_host=0.25, layers=1),
        # sixteen answers to one prompt of 32k tokens that fills its last block
        dict(name="samples_16", kind="samples", B=16, prefixes=1, len_lo=32768, len_hi=32768, p_host=0.5, layers=1, **c32b),
        # a serving batch: answers to four prompts of unequal lengths, most of which end inside a block
        dict(name="samples_ragged", kind="samples", B=48, prefixes=4, len_lo=4000, len_hi=40001, p_host=0.25, layers=1, **c8b),
        # answers with tiles of their own, a short prompt
        dict(name="churn_small", kind="churn", B=4, prefixes=1, len_lo=1021, len_hi=1021, p_host=0.0, layers=1, Hq=8, Hkv=2, d=64, S=16, dtype="f32"),
        # the same with a long one
        dict(name="churn_long", kind="churn", B=8, prefixes=1, len_lo=32749, len_hi=32749, p_host=0.5, layers=1, **c32b),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(["attend", "samples", "churn"], [6, 3, 2])[0]
    Hkv, G, d = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 4, 5, 7, 8, 8, 16]), rng.choice([128, 128, 64])
    S, dtype = rng.choice([16, 32, 32, 64]), "f32" if rng.random() < 0.2 else "bf16"
    hi = _log_int(rng, 40, 32768)
    c = dict(kind=kind, Hkv=Hkv, Hq=G * Hkv, d=d, S=S, dtype=dtype, prefixes=_log_int(rng, 1, 8), len_hi=hi,
             len_lo=hi if rng.random() < 0.4 else rng.randint(max(1, hi // 8), hi), p_host=rng.choice([0.0, 0.0, 0.25, 0.5]))
    c["layers"] = rng.randint(1, 2)
    row = Hkv * hi * d * (2 if dtype == "bf16" else 4)  # the keys of one of the longest prefixes
    if kind == "attend":
        c["B"] = max(c["prefixes"], _log_int(rng, 1, 64))
        c["alone"], c["other"] = rng.choice([0.0, 0.0, 0.2]), int(rng.random() < 0.7)
        # rows x tokens: at most the largest listed case's, an eighth of it in fp32
        most = 64 * 64 * 32768 * 128 // (8 if dtype == "f32" else 1)
        while c["B"] > c["prefixes"] and c["B"] * c["Hq"] * hi * d > most:
            c["B"] -= 1
        while c["prefixes"] > 1 and c["prefixes"] * row > 4 * 8 * 32768 * 128 * 2:
            c["prefixes"] -= 1
    elif kind == "samples":
        c["B"] = max(c["prefixes"], _log_int(rng, 1, 48))
        while c["B"] > 1 and c["B"] * row // S > 48 * 8 * 32768 * 128 * 2 // 32:
            c["B"] -= 1
    else:
        c["prefixes"] = 1
        c["B"] = 2 * _log_int(rng, 1, 4)
    return c


# ------------------------------------------------------------------------------------------- inputs


class _State:
    pass


class _Layer:
    pass


def _torch_dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _lengths(case, gen):
    n = torch.randint(case["len_lo"], case["len_hi"] + 1, (case["prefixes"],), generator=gen, device="cuda", dtype=torch.int32)
    n[0] = case["len_hi"]
    return n


def _resident(case, lens, mb, gen):
    """Which of the blocks [prefixes][Hkv][mb] have a slot: the same share of the blocks of every pair."""
    nb = (lens + case["S"] - 1) // case["S"]
    beyond = torch.arange(mb, device="cuda") >= nb[:, None, None]
    rank = (torch.rand(len(lens), case["Hkv"], mb, generator=gen, device="cuda") + 2 * beyond).argsort(-1).argsort(-1)
    return rank < ((1 - case["p_host"]) * nb).round()[:, None, None]


def _normal(shape, dt, gen, scale=1.0):
    return torch.randn(shape, generator=gen, device="cuda", dtype=dt).mul_(scale)


def _prepare_attend(case, s, gen):
    Bn, Hq, Hkv, d, S, P = (case[f] for f in ("B", "Hq", "Hkv", "d", "S", "prefixes"))
    dt, dev, G = _torch_dtype(case), "cuda", case["Hq"] // case["Hkv"]
    s.prefix_len = _lengths(case, gen)
    s.blocks = (case["len_hi"] + S - 1) // S
    of = torch.randint(0, P, (Bn,), generator=gen, device=dev)
    of[:P] = torch.arange(P, device=dev)[:Bn]
    of[P:][torch.rand(max(0, Bn - P), generator=gen, device=dev) < case["alone"]] = -1
    s.prefix_of = of.to(torch.int32)
    s.ctx = torch.zeros(Bn, dtype=torch.int32, device=dev)
    for _ in range(case["layers"]):
        L = _Layer()
        L.q = _normal((Bn, Hq, d), dt, gen)
        keep = _resident(case, s.prefix_len, s.blocks, gen)
        at = keep.view(-1).nonzero().view(-1)
        L.n_slots = at.numel() + 3
        L.table = torch.full((P, Hkv, s.blocks), -1, dtype=torch.int32, device=dev)
        L.table.view(-1)[at] = torch.randperm(L.n_slots, generator=gen, device=dev, dtype=torch.int32)[:at.numel()]
        L.k_pool, L.v_pool = _normal((L.n_slots, S, d), dt, gen), _normal((L.n_slots, S, d), dt, gen)
        # some blocks matter to everybody: their keys point along the queries of their KV head
        u = L.q.float().view(Bn, Hkv, G, d).sum((0, 2))
        u = 3.0 * u / u.norm(dim=-1, keepdim=True)
        heavy = keep & (torch.rand(keep.shape, generator=gen, device=dev) < PLANTED)
        p, g, j = heavy.nonzero(as_tuple=True)
        slot = L.table[p, g, j].long()
        L.k_pool[slot] += u[g][:, None, :].to(dt)
        # what lies behind a prefix's last token is not to be read as numbers
        last = (s.prefix_len - 1) // S
        slot = L.table.gather(2, last.long()[:, None, None].expand(P, Hkv, 1))[..., 0]
        row = torch.arange(S, device=dev) >= (s.prefix_len - last * S)[:, None]
        p, r = row.nonzero(as_tuple=True)
        slots, rows = slot[p].reshape(-1), r[:, None].expand(-1, Hkv).reshape(-1)
        slots, rows = slots[slots >= 0].long(), rows[slots >= 0]
        L.k_pool[slots, rows] = float("nan")
        L.v_pool[slots, rows] = float("nan")
        L.o_b = L.m_b = L.l_b = None
        if case["other"]:  # a few hundred tokens of the sequence's own; a sequence that has none yet now and then
            L.o_b = _normal((Bn, Hq, d), torch.float32, gen, 0.1)
            L.m_b = 2.0 + _normal((Bn, Hq), torch.float32, gen, 0.3)
            L.l_b = torch.empty(Bn, Hq, device=dev).uniform_(50.0, 500.0, generator=gen)
            none = torch.rand(Bn, generator=gen, device=dev) < 0.1
            L.o_b[none], L.m_b[none], L.l_b[none] = 0.0, -math.inf, 0.0
        L.out, L.lse = torch.empty(Bn, Hq, d, dtype=dt, device=dev), torch.empty(Bn, Hq, device=dev)
        s.layers.append(L)
    # the batch ordered by prefix, as rows of one product for each of them: who sits where, and where each sequence is found
    order = torch.argsort(of, stable=True)
    place = torch.arange(Bn, device=dev) - torch.searchsorted(of[order].contiguous(), of[order].contiguous())
    most = int((place[of[order] >= 0] + 1).amax()) if bool((of >= 0).any()) else 1
    s.members = torch.zeros(P, most, dtype=torch.long, device=dev)
    has = of[order] >= 0
    s.members[of[order][has], place[has]] = order[has]
    s.found = torch.full((Bn,), -1, dtype=torch.long, device=dev)
    s.found[order[has]] = of[order][has] * most + place[has]


def _prepare_pages(case, s, gen):
    """Rows: the answers, then the prompts.  Slots: the prompts' first, shuffled; of "churn" then the answers' in the order that
    the last round left them."""
    n, Hkv, d, S, P = (case[f] for f in ("B", "Hkv", "d", "S", "prefixes"))
    dt, dev, churn = _torch_dtype(case), "cuda", case["kind"] == "churn"
    lens = _lengths(case, gen)
    mb, rows = (case["len_hi"] + S - 1) // S + 1, n + P
    s.max_blocks = mb
    parent = torch.randint(0, P, (n,), generator=gen, device=dev)
    parent[:P] = torch.arange(P, device=dev)[:n]
    s.src, s.dst = (n + parent).to(torch.int32), torch.arange(n, dtype=torch.int32, device=dev)
    if churn:  # the answers leave by halves
        half = torch.arange(n, dtype=torch.int32, device=dev)
        s.halves = [(s.src[:n // 2].clone(), half[:n // 2].clone()), (s.src[n // 2:].clone(), half[n // 2:].clone())]
    for _ in range(case["layers"]):
        L = _Layer()
        keep = _resident(case, lens, mb, gen)
        at = keep.view(-1).nonzero().view(-1)
        r = at.numel()
        room = P * Hkv * (int((1 - case["p_host"]) * mb) + 1)  # at least r, whatever the lengths
        L.n_slots = r * (n + 1) + 7 if churn else room + 2 * n * Hkv
        L.table = torch.full((rows, Hkv, mb), -1, dtype=torch.int32, device=dev)
        slots = torch.randperm(r, generator=gen, device=dev, dtype=torch.int32)
        L.table[n:].view(-1)[at] = slots
        L.ctx = torch.full((rows,), -1, dtype=torch.int32, device=dev)
        L.ctx[n:] = lens
        L.k_pool, L.v_pool = _normal((L.n_slots, S, d), dt, gen), _normal((L.n_slots, S, d), dt, gen)
        L.digest = torch.zeros(rows, Hkv, mb, 2, d, dtype=dt, device=dev)
        L.digest[n:, :, :, 0], L.digest[n:, :, :, 1] = (_normal((P, Hkv, mb, d), dt, gen) + x for x in (-2.0, 2.0))
        L.digest[n:][torch.arange(mb, device=dev).expand(P, Hkv, mb) >= ((lens + S - 1) // S)[:, None, None]] = 0
        if churn:  # every answer has a copy of the prompt, in the order of its blocks
            L.ctx[:n], L.digest[:n] = lens, L.digest[n:]
            mine = r + r * torch.arange(n, device=dev)[:, None] + torch.arange(r, device=dev)
            L.table[:n].view(n, -1)[:, at] = mine.to(torch.int32)
            for pool in (L.k_pool, L.v_pool):
                pool[r:r + n * r].view(n, r, S, d)[:] = pool[slots.long()]
        L.refs = torch.zeros(L.n_slots, dtype=torch.int32, device=dev)
        L.refs[:r * (n + 1) if churn else r] = 1
        L.k_new, L.v_new = _normal((n, Hkv, d), dt, gen), _normal((n, Hkv, d), dt, gen)
        i32 = dict(dtype=torch.int32, device=dev)
        L.new_slot, L.status, L.n_short = torch.empty(n, Hkv, **i32), torch.empty(n, **i32), torch.empty(1, **i32)
        L.slot_map, L.n_live = torch.empty(L.n_slots, **i32), torch.empty(1, **i32)
        s.layers.append(L)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = _State()
    s.case, s.layers = case, []
    (_prepare_attend if case["kind"] == "attend" else _prepare_pages)(case, s, gen)
    return s


# ------------------------------------------------------------------------------------------- the plain forms


def _plain_attend(s, L):
    Bn, Hq, d = L.q.shape
    P, Hkv, pb = L.table.shape
    G, S, M, dev = Hq // Hkv, L.k_pool.shape[1], s.members.shape[1], L.q.device
    token = torch.arange(pb * S, device=dev)
    held = (L.table >= 0).repeat_interleave(S, -1) & (token < s.prefix_len[:, None, None])
    slot = L.table.clamp(min=0).long()
    k = L.k_pool[slot].view(P, Hkv, pb * S, d).float().masked_fill(~held[..., None], 0.0)
    v = L.v_pool[slot].view(P, Hkv, pb * S, d).float().masked_fill(~held[..., None], 0.0)
    q = L.q[s.members].view(P, M, Hkv, G, d).transpose(1, 2).reshape(P, Hkv, M * G, d).float()
    x = (torch.matmul(q, k.transpose(-1, -2).contiguous()) / math.sqrt(d)).masked_fill(~held[:, :, None], -math.inf)
    m = x.amax(-1)
    w = (x - m.masked_fill(m == -math.inf, 0.0)[..., None]).exp()
    l = w.sum(-1)
    o = torch.matmul(w, v) / l.masked_fill(l == 0, 1.0)[..., None]

    def of_sequence(t, empty):
        t = t.view(P, Hkv, M, G, *t.shape[3:]).transpose(1, 2).reshape(P * M, Hq, *t.shape[3:])
        return t[s.found.clamp(min=0)].masked_fill((s.found < 0).view(Bn, *[1] * (t.dim() - 1)), empty)

    o, m, l = of_sequence(o, 0.0), of_sequence(m, -math.inf), of_sequence(l, 0.0)
    if L.o_b is None:
        both, top, total = o, m, l
    else:
        top = torch.maximum(m, L.m_b)
        base = top.masked_fill(top == -math.inf, 0.0)
        wa, wb = l * (m - base).exp(), L.l_b * (L.m_b - base).exp()
        total = wa + wb
        both = (wa[..., None] * o + wb[..., None] * L.o_b) / total.masked_fill(total == 0, 1.0)[..., None]
    return [both.to(L.q.dtype), top + total.log()]


def _row_of(L, seq, S):
    """Of the listed sequences: table rows, how many blocks they have, which of their blocks have a slot."""
    rows, ctx = L.table[seq], L.ctx[seq].clamp(min=0)
    nb = (ctx + S - 1) // S
    return rows, ctx, nb, (rows >= 0) & (torch.arange(rows.shape[-1], device=rows.device) < nb[:, None, None])


def _plain_free(L, seq, S):
    rows, _, _, held = _row_of(L, seq, S)
    L.refs.index_add_(0, rows.clamp(min=0).view(-1).long(), -held.view(-1).to(torch.int32))
    L.table[seq] = -1
    L.ctx[seq] = -1


def _lowest_free(L):
    """The free slots in ascending order (then the others), and how many there are."""
    return torch.argsort((L.refs > 0).to(torch.int8), stable=True).to(torch.int32), (L.refs <= 0).sum()


def _plain_fork(L, src, dst, deep, S):
    rows, ctx, nb, held = _row_of(L, src, S)
    j = torch.arange(rows.shape[-1], device=rows.device)
    copied = held if deep else held & (j == nb[:, None, None] - 1) & (ctx % S != 0)[:, None, None]
    slots, n_free = _lowest_free(L)
    rank = copied.view(-1).cumsum(0).view(copied.shape) - 1
    got = copied & (rank < n_free)
    new = torch.where(got, slots[rank.clamp(0, slots.numel() - 1)], -1)
    child = torch.where(copied, new, torch.where(held, rows, -1))
    L.refs.index_add_(0, child.clamp(min=0).view(-1).long(), (child >= 0).view(-1).to(torch.int32))
    if deep:
        to, at = new[got].long(), rows[got].long()
    else:  # a tail for every pair; one that has nothing to copy is copied onto itself
        last = (nb - 1).clamp(min=0).long()[:, None, None].expand(*rows.shape[:2], 1)
        at = rows.gather(2, last).clamp(min=0).view(-1).long()
        to = torch.where(got.gather(2, last), new.gather(2, last), rows.gather(2, last)).clamp(min=0).view(-1).long()
    L.k_pool[to], L.v_pool[to] = L.k_pool[at], L.v_pool[at]
    inside = (j < nb[:, None])[:, None, :, None, None]
    L.digest[dst] = torch.where(inside, L.digest[src], L.digest[dst])
    L.table[dst], L.ctx[dst] = child, L.ctx[src]
    return (copied & ~got).sum((1, 2)).to(torch.int32)


def _plain_reserve(L, n, S):
    ctx, mb = L.ctx[:n], L.table.shape[-1]
    opens = ((ctx >= 0) & (ctx < mb * S) & (ctx % S == 0))[:, None].expand(n, L.table.shape[1])
    slots, n_free = _lowest_free(L)
    rank = opens.reshape(-1).cumsum(0).view(opens.shape) - 1
    got = opens & (rank < n_free)
    new = torch.where(got, slots[rank.clamp(0, slots.numel() - 1)], -1)
    L.refs.index_add_(0, new.clamp(min=0).view(-1).long(), got.view(-1).to(torch.int32))
    return new, (opens & ~got).sum().view(1).to(torch.int32)


def _plain_append(L, n, new_slot, S):
    ctx, mb = L.ctx[:n].clone(), L.table.shape[-1]
    grows = ((ctx >= 0) & (ctx < mb * S))[:, None]
    t = ctx.clamp(0, mb * S - 1)
    b = torch.arange(n, device=ctx.device)[:, None]
    g, j, r = torch.arange(L.table.shape[1], device=ctx.device)[None], (t // S).long()[:, None], (t % S).long()[:, None]
    entry = L.table[b, g, j]
    slot = torch.where(r == 0, new_slot, entry)
    L.table[b, g, j] = torch.where(grows, slot, entry)
    lo, hi = L.digest[b, g, j, 0], L.digest[b, g, j, 1]
    first, more = (r == 0)[..., None], grows[..., None]
    L.digest[b, g, j, 0] = torch.where(more, torch.where(first | (L.k_new < lo), L.k_new, lo), lo)
    L.digest[b, g, j, 1] = torch.where(more, torch.where(first | (L.k_new > hi), L.k_new, hi), hi)
    here = (slot >= 0) & grows
    at = torch.where(here, slot, L.refs.numel() - 1).long()  # the pool's last slot is nobody's here: it stays as it is
    row = r.expand(at.shape)
    L.k_pool[at, row] = torch.where(here[..., None], L.k_new, L.k_pool[at, row])
    L.v_pool[at, row] = torch.where(here[..., None], L.v_new, L.v_pool[at, row])
    L.ctx[:n] = torch.where(grows[:, 0], ctx + 1, ctx)


def _plain_compact(L):
    used, at = L.refs > 0, torch.arange(L.refs.numel(), device=L.refs.device)
    n_live = used.sum()
    above, below = used & (at >= n_live), ~used & (at < n_live)
    source, target = above.nonzero().view(-1), below.nonzero().view(-1)
    slot_map = torch.where(used, at, -1).to(torch.int32)
    slot_map[source] = target.to(torch.int32)
    L.k_pool[target], L.v_pool[target] = L.k_pool[source], L.v_pool[source]
    L.refs[target], L.refs[source] = L.refs[source], 0
    L.table.copy_(torch.where(L.table >= 0, slot_map[L.table.clamp(min=0).long()], L.table))
    return slot_map, n_live.view(1).to(torch.int32)


def _plain(s):
    kind, S = s.case["kind"], s.case["S"]
    if kind == "attend":
        return [_plain_attend(s, L) for L in s.layers]
    got, n = [], s.case["B"]
    for L in s.layers:
        if kind == "samples":
            _plain_free(L, s.dst.long(), S)
            status = _plain_fork(L, s.src.long(), s.dst.long(), False, S)
            new_slot, n_short = _plain_reserve(L, n, S)
            _plain_append(L, n, new_slot, S)
            got.append([L.ctx, L.table, L.digest, L.k_pool, L.v_pool, L.refs, status, new_slot, n_short])
        else:
            for src, dst in s.halves:
                _plain_free(L, dst.long(), S)
                slot_map, n_live = _plain_compact(L)
                status = _plain_fork(L, src.long(), dst.long(), True, S)
            got.append([L.ctx, L.table, L.digest, L.k_pool, L.v_pool, L.refs, status, slot_map, n_live])
    return got


# ------------------------------------------------------------------------------------------- the library's calls


def _open(s):
    """The handles that a program keeps beside its cache: problems, workspace, the plan's memory, the pages' state."""
    from paper_2603_27138_amd import binding as B

    c = s.case
    dt = B.BF16 if c["dtype"] == "bf16" else B.F32
    shape = (c["Hq"], c["Hkv"], c["d"], c["S"], dt)
    s.B = B
    if c["kind"] == "attend":
        s.p = B.make_problem(c["B"], *shape, s.blocks, 1, s.ctx)
        s.ws, s.plan = B.alloc_workspace(s.p), B.alloc_prefix_plan(s.p, c["prefixes"])
        return
    for L in s.layers:
        L.p = B.make_problem(L.table.shape[0], *shape, s.max_blocks, 1, L.ctx)
        L.answers = B.make_problem(c["B"], *shape, s.max_blocks, 1, L.ctx)
        L.pages = B.alloc_pages(L.n_slots)
        B.pages_init(L.p, L.ctx, L.table, L.n_slots, L.pages)


def _library(s):
    if not hasattr(s, "B"):
        _open(s)
    B, c = s.B, s.case
    if c["kind"] == "attend":
        B.prefix_plan(s.p, c["prefixes"], s.blocks, s.prefix_of, s.prefix_len, s.plan)
        for L in s.layers:
            B.shared_prefix_attn(s.p, c["prefixes"], s.blocks, s.plan, L.q, L.k_pool, L.v_pool, L.n_slots, L.table, L.o_b, L.m_b, L.l_b,
                                 None, None, None, L.out, L.lse, s.ws)
        return [[L.out, L.lse] for L in s.layers]
    got = []
    for L in s.layers:
        cache = (L.ctx, L.digest, L.table, L.k_pool, L.v_pool, L.n_slots, L.pages)
        refs = L.pages[:L.n_slots]
        if c["kind"] == "samples":
            B.free_sequences(L.p, s.dst, L.ctx, L.table, L.n_slots, L.pages)
            B.fork_sequences(L.p, s.src, s.dst, False, *cache, L.status)
            B.reserve_blocks(L.answers, L.ctx, L.n_slots, L.pages, L.new_slot, L.n_short)
            B.append_token(L.answers, L.ctx, L.k_new, L.v_new, L.new_slot, L.digest, L.table, L.k_pool, L.v_pool, L.n_slots)
            got.append([L.ctx, L.table, L.digest, L.k_pool, L.v_pool, refs, L.status, L.new_slot, L.n_short])
        else:
            for src, dst in s.halves:
                B.free_sequences(L.p, dst, L.ctx, L.table, L.n_slots, L.pages)
                B.compact_pool(L.p, L.table, L.k_pool, L.v_pool, L.n_slots, L.pages, L.slot_map, L.n_live)
                B.fork_sequences(L.p, src, dst, True, *cache, L.status[:len(dst)])
            got.append([L.ctx, L.table, L.digest, L.k_pool, L.v_pool, refs, L.status[:len(dst)], L.slot_map, L.n_live])
    return got


def run(state):
    return _library(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------- work, and the values in 64 bits


def work(case):
    Hq, Hkv, d, S, n, P = (case[f] for f in ("Hq", "Hkv", "d", "S", "B", "prefixes"))
    es = 2 if case["dtype"] == "bf16" else 4
    mean = (case["len_lo"] + case["len_hi"]) / 2
    held = (case["len_hi"] + (P - 1) * mean) * (1 - case["p_host"])  # tokens of all prefixes that have a slot
    if case["kind"] == "attend":
        sharing = min(P, n) + max(0, n - P) * (1 - case["alone"])
        nbytes = held * Hkv * d * es * 2 + held / S * Hkv * 4 + n * Hq * (2 * d * es + 4 + (4 * (d + 2) if case["other"] else 0))
        return {"bytes": case["layers"] * nbytes, "flops": case["layers"] * 4 * sharing * Hq * d * held / P}
    blocks = (case["len_hi"] + (P - 1) * mean) / S * Hkv  # of all prompts
    if case["kind"] == "samples":
        # digests and table rows of the prompts read, those of the answers written (the old rows' entries read), a tail tile each
        entry, tile = 2 * d * es + 4, 2 * S * d * es
        return {"bytes": case["layers"] * (blocks * entry + n / P * blocks * (entry + 4) + 2 * n * Hkv * tile), "flops": 0}
    # every answer written anew from the prompt, and every answer moved once by the compaction of the other half
    tile = 2 * S * d * es * (1 - case["p_host"])
    entry = 2 * d * es + 4
    return {"bytes": case["layers"] * (2 * blocks * (tile + entry) + n * blocks * (tile + entry) + 2 * n * blocks * tile), "flops": 0}


def _exact_attend(case, s):
    got = []
    G, S, of, lens = case["Hq"] // case["Hkv"], case["S"], s.prefix_of.tolist(), s.prefix_len.tolist()
    for L in s.layers:
        out, lse = [None] * case["B"], [None] * case["B"]
        for b in range(case["B"]):
            empty = torch.zeros(case["Hkv"], G, 0, dtype=torch.float64, device="cuda")
            logit, weight_v = [], []
            if of[b] >= 0:
                for g in range(case["Hkv"]):
                    row = L.table[of[b], g, :(lens[of[b]] + S - 1) // S]
                    where = (row[:, None].long() * S + torch.arange(S, device="cuda")).view(-1)[:lens[of[b]]]
                    where = where[row.repeat_interleave(S)[:lens[of[b]]] >= 0]
                    k = L.k_pool.view(-1, case["d"])[where].double()
                    logit.append(L.q[b].view(case["Hkv"], G, -1)[g].double() @ k.T * case["d"] ** -0.5)
                    weight_v.append(L.v_pool.view(-1, case["d"])[where].double())
            else:
                logit, weight_v = list(empty), [torch.zeros(0, case["d"], dtype=torch.float64, device="cuda")] * case["Hkv"]
            o, z = [], []
            for g in range(case["Hkv"]):
                x, v = logit[g], weight_v[g]
                if L.o_b is not None:  # one more entry: what the sequence attended to of its own, at its weight
                    heads = slice(g * G, (g + 1) * G)
                    own_lse = L.m_b[b, heads].double() + L.l_b[b, heads].double().log()
                    x = torch.cat([x, own_lse[:, None]], 1)
                if x.shape[1] == 0:
                    o.append(torch.zeros(G, case["d"], dtype=torch.float64, device="cuda"))
                    z.append(torch.full((G,), -math.inf, dtype=torch.float64, device="cuda"))
                    continue
                total = torch.logsumexp(x, 1)
                share = torch.exp(x - total.masked_fill(total == -math.inf, 0.0)[:, None])
                y = share[:, :v.shape[0]] @ v
                if L.o_b is not None:
                    y = y + share[:, -1:] * L.o_b[b, heads].double()
                o.append(y)
                z.append(total)
            out[b], lse[b] = torch.cat(o), torch.cat(z)
        got.append([torch.stack(out), torch.stack(lse)])
    return got


class _Book:
    """A layer's cache kept sequence by sequence, block by block."""

    def __init__(self, case, L):
        self.S, self.L = case["S"], L
        self.table, self.ctx, self.refs = L.table.cpu().numpy().copy(), L.ctx.tolist(), L.refs.cpu().numpy().copy()

    def blocks(self, b):
        return (max(0, self.ctx[b]) + self.S - 1) // self.S

    def free(self, b):
        for g in range(self.table.shape[1]):
            for slot in self.table[b, g, :self.blocks(b)]:
                if slot >= 0:
                    self.refs[slot] -= 1
        self.table[b], self.ctx[b] = -1, -1

    def take(self, count):
        slots = (self.refs == 0).nonzero()[0][:count]
        assert len(slots) == count  # the cases have room for all
        self.refs[slots] = 1
        return slots.tolist()

    def fork(self, a, b, deep):
        nb = self.blocks(a)
        moves = []
        for g in range(self.table.shape[1]):
            for j in range(nb):
                slot = int(self.table[a, g, j])
                if slot >= 0 and (deep or (j == nb - 1 and self.ctx[a] % self.S)):
                    moves.append((g, j, slot))
                else:
                    self.table[b, g, j] = slot
                    if slot >= 0:
                        self.refs[slot] += 1
        new = self.take(len(moves))
        for (g, j, _), slot in zip(moves, new):
            self.table[b, g, j] = slot
        at, to = (torch.tensor(x, dtype=torch.long, device="cuda") for x in ([m[2] for m in moves], new))
        self.move(at, to)
        self.L.digest[b, :, :nb] = self.L.digest[a, :, :nb]
        self.ctx[b] = self.ctx[a]

    def move(self, at, to):
        for pool in (self.L.k_pool, self.L.v_pool):
            pool[to] = pool[at].clone()

    def compact(self):
        live = int((self.refs > 0).sum())
        holes = iter([i for i in range(live) if self.refs[i] == 0])
        where = [-1] * len(self.refs)
        for i in range(len(self.refs)):
            if self.refs[i] > 0:
                where[i] = i if i < live else next(holes)
        moved = [(i, w) for i, w in enumerate(where) if w not in (i, -1)]
        self.move(*(torch.tensor([m[e] for m in moved], dtype=torch.long, device="cuda") for e in (0, 1)))
        for i, w in moved:
            self.refs[w], self.refs[i] = self.refs[i], 0
        np_map = torch.tensor(where).numpy()
        self.table[self.table >= 0] = np_map[self.table[self.table >= 0]]
        return where, live

    def outputs(self, *more):
        L, i32 = self.L, dict(dtype=torch.int32)
        whole = [torch.tensor(self.ctx, **i32), torch.from_numpy(self.table), torch.from_numpy(self.refs)]
        return [whole[0], whole[1], L.digest.double(), L.k_pool.double(), L.v_pool.double(), whole[2], *(torch.tensor(x, **i32) for x in more)]


def _exact_pages(case, s):
    got, n, S = [], case["B"], case["S"]
    for L in s.layers:
        book = _Book(case, L)
        if case["kind"] == "churn":
            for src, dst in s.halves:
                for b in dst.tolist():
                    book.free(b)
                where, live = book.compact()
                for a, b in zip(src.tolist(), dst.tolist()):
                    book.fork(a, b, True)
            got.append(book.outputs([0] * len(dst), where, [live]))
            continue
        for a, b in zip(s.src.tolist(), s.dst.tolist()):
            book.free(b)
            book.fork(a, b, False)
        new_slot = [[-1] * case["Hkv"] for _ in range(n)]
        for b in range(n):
            t = book.ctx[b]
            j, r = t // S, t % S
            for g in range(case["Hkv"]):
                if r == 0:
                    new_slot[b][g] = book.table[b, g, j] = book.take(1)[0]
                slot, k = int(book.table[b, g, j]), L.k_new[b, g]
                L.digest[b, g, j, 0] = k if r == 0 else torch.minimum(L.digest[b, g, j, 0], k)
                L.digest[b, g, j, 1] = k if r == 0 else torch.maximum(L.digest[b, g, j, 1], k)
                if slot >= 0:
                    L.k_pool[slot, r], L.v_pool[slot, r] = k, L.v_new[b, g]
            book.ctx[b] = t + 1
        got.append(book.outputs([0] * n, new_slot, [0]))
    return got


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_attend(case, s) if case["kind"] == "attend" else _exact_pages(case, s)
