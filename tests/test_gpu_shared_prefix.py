"""Attention over shared prefixes against the definition in 64 bits, sequence by sequence.

Tolerances, from how the kernels compute (u = 2^-24, half a step of binary32):
  logits   products of d terms are summed in binary32: off by at most (d + 4) u sum_c |q_c k_c| scale; scaling and shifting rounds by 2 u |x|.
  weights  a logit that is off by e makes its weight off by e relatively (and the exponential itself by a few u).
  sums     of n tokens: a chain adds one term per 16 tokens, plus splits and waves: (n / 16 + 128) u relatively.
  bf16     where only `out` is written the weights enter the value product rounded to bf16: 2^-8 relatively at the most; where the partial
           is, as two terms: 2^-15 at the most (7 explicit bits are cut, 7 more are rounded).  `out` itself is rounded by 2^-8.
An output is a mean of values with these weights, so its error is at most twice the weights' (numerator and sum) times the mean of the |v|."""
import math

import pytest
import torch

from paper_2603_27138_amd import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16


class Batch:
    def __init__(self, seed, dtype, d, S, G, Hkv, lens, of, p_host=0.0, other=True, paired=False, scale=0.0, blocks=None, sharp=1.0,
                 spare=3):
        g = torch.Generator().manual_seed(seed)
        Bn, P, Hq = len(of), len(lens), G * Hkv
        self.Bn, self.Hq, self.Hkv, self.G, self.d, self.S, self.dtype, self.P, self.lens, self.of = Bn, Hq, Hkv, G, d, S, dtype, P, lens, of
        self.blocks = blocks or max(1, max([-(-n // S) for n in lens], default=1))
        nb = [min(self.blocks, max(0, -(-n // S))) for n in lens]
        self.n_slots = max(1, sum(nb) * Hkv) + spare
        self.table = torch.full((P, Hkv, self.blocks), -1, dtype=torch.int32)
        slots = iter(torch.randperm(self.n_slots, generator=g).tolist())
        for p in range(P):
            for h in range(Hkv):
                for j in range(nb[p]):
                    if torch.rand(1, generator=g).item() >= p_host:
                        self.table[p, h, j] = next(slots)
        k, v = (torch.randn(self.n_slots, S, d, generator=g).to(dtype) for _ in range(2))
        self.q = (sharp * torch.randn(Bn, Hq, d, generator=g)).to(dtype)
        for p in range(P):  # behind the last token of a prefix: nothing that may be read as a number
            n = min(max(0, lens[p]), self.blocks * S)
            if n % S:
                for h in range(Hkv):
                    s = int(self.table[p, h, n // S])
                    if s >= 0:
                        k[s, n % S:] = v[s, n % S:] = float("nan")
        self.k, self.v = k, v
        self.scale = scale or 1.0 / math.sqrt(d)
        self.other = None
        if other:
            l_b = torch.rand(Bn, Hq, generator=g) * 20 + 1
            m_b = torch.randn(Bn, Hq, generator=g)
            o_b = torch.randn(Bn, Hq, d, generator=g)
            l_b[::3], m_b[::3], o_b[::3] = 0.0, -math.inf, 0.0
            self.other = (o_b, m_b, l_b)
        self.ctx = torch.zeros(Bn, dtype=torch.int32, device="cuda")
        if paired:
            self.pool = torch.stack([k, v], 1).contiguous().cuda()
            self.k_dev, self.v_dev, stride = self.pool.view(-1), self.pool.view(-1)[S * d:], 2 * S * d
        else:
            self.k_dev, self.v_dev, stride = k.cuda(), v.cuda(), 0
        self.p = B.make_problem(Bn, Hq, Hkv, d, S, B.BF16 if dtype == BF16 else B.F32, 4, 1, self.ctx, sm_scale=scale, tile_stride=stride)
        i32 = dict(dtype=torch.int32, device="cuda")
        self.of_dev, self.len_dev = torch.tensor(of, **i32), torch.tensor(lens, **i32)
        self.ws, self.plan = B.alloc_workspace(self.p), B.alloc_prefix_plan(self.p, P)
        self.ws.fill_(0xff)   # NaNs
        self.plan.fill_(0xff)

    def run(self, partial=False, result=True, other=True, plan=True):
        f32 = dict(dtype=F32, device="cuda")
        nan = float("nan")
        self.out = torch.full((self.Bn, self.Hq, self.d), nan, dtype=self.dtype, device="cuda") if result else None
        self.lse = torch.full((self.Bn, self.Hq), nan, **f32) if result else None
        self.o = torch.full((self.Bn, self.Hq, self.d), nan, **f32) if partial else None
        self.m, self.l = (torch.full((self.Bn, self.Hq), nan, **f32) if partial else None for _ in range(2))
        ob = [t.cuda() for t in self.other] if other and self.other is not None else [None] * 3
        if plan:
            B.prefix_plan(self.p, self.P, self.blocks, self.of_dev, self.len_dev, self.plan)
        B.shared_prefix_attn(self.p, self.P, self.blocks, self.plan, self.q.cuda(), self.k_dev, self.v_dev, self.n_slots, self.table.cuda(), *ob,
                             self.o, self.m, self.l, self.out, self.lse, self.ws)
        torch.cuda.synchronize()
        return self

    def want(self, other=True):
        """out, lse, and the bounds on the weights' and sums' relative errors and the mean of |v|, per query head."""
        out, lse = torch.zeros(self.Bn, self.Hq, self.d, dtype=torch.float64), torch.full((self.Bn, self.Hq), -math.inf, dtype=torch.float64)
        mean_v, err = torch.zeros(self.Bn, self.Hq, self.d, dtype=torch.float64), torch.zeros(self.Bn, self.Hq, dtype=torch.float64)
        for b in range(self.Bn):
            for h in range(self.Hq):
                xs, vs = [], []
                g = h // self.G
                if 0 <= self.of[b] < self.P:
                    n = min(max(0, self.lens[self.of[b]]), self.blocks * self.S)
                    for j in range(-(-n // self.S)):
                        s = int(self.table[self.of[b], g, j])
                        if 0 <= s < self.n_slots:
                            c = min(self.S, n - j * self.S)
                            kk, vv = self.k[s, :c].double(), self.v[s, :c].double()
                            qk = kk * self.q[b, h].double()
                            xs.append(qk.sum(1) * self.scale)
                            err[b, h] = max(err[b, h], float((qk.abs().sum(1) * self.scale).max()) * (self.d + 8) * U)
                            vs.append(vv)
                n = sum(len(x) for x in xs)
                err[b, h] += (n / 16 + 128) * U
                if other and self.other is not None and self.other[2][b, h] > 0:
                    o_b, m_b, l_b = (t[b, h].double() for t in self.other)
                    xs.append((m_b + l_b.log()).view(1))
                    vs.append(o_b.view(1, -1))
                if xs:
                    x, v = torch.cat(xs), torch.cat(vs)
                    w = torch.softmax(x, 0)
                    out[b, h], lse[b, h], mean_v[b, h] = w @ v, torch.logsumexp(x, 0), w @ v.abs()
        return out, lse, mean_v, err

    def check(self, other=True):
        out, lse, mean_v, err = self.want(other)

        def near(got, want, bound):
            got = got.double().cpu()
            both_inf = (got == want) & torch.isinf(want)
            off = torch.where(both_inf, torch.zeros_like(want), (got - want).abs())
            assert bool((off <= bound).all()), (float((off - bound).max()), float(off.max()))
        bf16 = self.dtype == BF16
        if self.out is not None:
            weights = err + (2.0 ** -15 if bf16 and self.o is not None else 2.0 ** -8 if bf16 else 0.0)
            near(self.out, out, 2 * weights[..., None] * mean_v + (2.0 ** -8 if bf16 else 4 * U) * out.abs() + 1e-30)
            near(self.lse, lse, 2 * err + 8 * U * lse.abs().nan_to_num(posinf=0.0))
        if self.o is not None:
            weights = err + (2.0 ** -15 if bf16 else 0.0)
            near(self.o, out, 2 * weights[..., None] * mean_v + 4 * U * out.abs() + 1e-30)
            got = self.m.double().cpu() + self.l.double().cpu().log()
            near(got, lse, 2 * err + 8 * U * lse.abs().nan_to_num(posinf=0.0))
            empty = torch.isinf(lse)
            assert bool((self.l.cpu()[empty] == 0).all()) and bool((self.m.cpu()[empty] == -math.inf).all())
        return self


def _of(P, n):
    """n sequences over P prefixes, in no order, one of them with none."""
    return [(5 * b + 3) % (P + 1) - 1 if n > P else b for b in range(n)]


@pytest.mark.parametrize("dtype,d,S", [(BF16, 128, 32), (BF16, 128, 16), (BF16, 64, 16), (BF16, 64, 64), (F32, 64, 16), (F32, 128, 32)])
@pytest.mark.parametrize("G,Hkv,n", [(1, 1, 1), (4, 2, 3), (7, 1, 9), (16, 1, 5), (8, 3, 20), (5, 2, 40)])
def test_shapes(dtype, d, S, G, Hkv, n):
    """From one row to tiles of rows that end inside a sequence, prefixes of unequal lengths that end inside a block."""
    lens = [3 * S + 5, 300, 2 * S]
    Batch(n * G + d, dtype, d, S, G, Hkv, lens, _of(3, n)).run().check()


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 64), (F32, 128)])
@pytest.mark.parametrize("n", [2, 6, 30])
def test_partials(dtype, d, n):
    """The joined partial, alone and beside the result."""
    b = Batch(n, dtype, d, 32, 8, 2, [777, 64], _of(2, n), p_host=0.3)
    b.run(partial=True, result=False).check()
    b.run(partial=True, result=True).check()
    b.run(partial=True, result=False, other=False).check(other=False)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("length", [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 1000, 5000])
def test_lengths(dtype, length):
    for n in (2, 20):
        Batch(length, dtype, 128, 32, 8, 1, [length], [0] * n, other=False, blocks=-(-length // 32) + 2).run().check()


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 128)])
@pytest.mark.parametrize("n", [1, 9, 70])
def test_blocks_on_the_host(dtype, d, n):
    """Half of the blocks, and all of them, without a slot; entries beyond the pool."""
    Batch(n, dtype, d, 16, 4, 2, [700, 40], _of(2, n), p_host=0.5).run().check()
    b = Batch(n, dtype, d, 16, 4, 2, [700, 40], _of(2, n), p_host=0.5)
    b.table[0, 0, ::3] = b.n_slots
    b.table[0, 1, 1::3] = 2 ** 31 - 1
    b.table[1, 0, 0] = -2 ** 31
    b.run().check()
    b.table.fill_(-1)
    b.run().check()
    b.run(partial=True, other=False).check(other=False)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_who_has_what(dtype):
    """Nobody has a prefix; lengths beyond the table and below zero; more prefixes than sequences; no prefixes; numbers outside."""
    Batch(1, dtype, 64, 16, 2, 2, [100, 30], [-1] * 5).run().check()
    Batch(2, dtype, 64, 16, 2, 2, [100000, -5, 2 ** 31 - 1], [0, 1, 2, 0], blocks=9).run().check()
    Batch(3, dtype, 64, 16, 2, 1, [17 * (i + 1) for i in range(12)], [11, 3], other=False).run().check()
    Batch(4, dtype, 64, 16, 2, 1, [], [0, -1, 5]).run().check()
    Batch(5, dtype, 64, 16, 2, 1, [50, 60], [2, -2 ** 31, 2 ** 31 - 1, 1]).run().check()


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 64)])
def test_one_prefix_of_many_and_one_of_few(dtype, d):
    """Tile sizes go by the average; a prefix with far more rows than that, and prefixes with one sequence."""
    of = [0] * 37 + [1, 2, 3, -1, 4, 0, 0]
    Batch(6, dtype, d, 32, 4, 2, [900, 33, 1, 450, 64], of).run().check()


@pytest.mark.parametrize("dtype,d,n", [(BF16, 128, 3), (BF16, 128, 40), (BF16, 64, 20), (F32, 128, 4)])
def test_large_logits(dtype, d, n):
    """Queries ten times as long: a few tokens have all the weight, and the maximum moves while tiles pass."""
    Batch(7, dtype, d, 32, 8, 1, [2000], [0] * n, sharp=10.0).run().check()


@pytest.mark.parametrize("n", [3, 40])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_scale_and_adjacent_tiles(dtype, n):
    Batch(8, dtype, 128, 16, 4, 2, [333, 50], _of(2, n), paired=True, scale=0.2).run().check()


@pytest.mark.parametrize("dtype,n", [(BF16, 2), (BF16, 40), (F32, 3)])
def test_infinite_and_nan_values(dtype, n):
    """What lies in a prefix's own tokens counts: an infinite value gives an infinite output in its channel, a NaN a NaN, in every
    sequence that has the prefix and in no other, with one-term and two-term weights."""
    for partial in (False, True):
        b = Batch(9, dtype, 64, 16, 4, 1, [200, 200], [0, 1] * n, other=False)
        s = int(b.table[0, 0, 3])
        b.v_dev.view(b.n_slots, 16, 64)[s, 5, 7] = math.inf
        b.v_dev.view(b.n_slots, 16, 64)[s, 6, 9] = -math.inf
        b.v_dev.view(b.n_slots, 16, 64)[s, 7, 11] = math.nan
        b.run(partial=partial)
        out, want = b.out.float().cpu(), b.want()[0]
        hit, miss = out[0::2], out[1::2]
        assert bool((hit[..., 7] == math.inf).all()) and bool((hit[..., 9] == -math.inf).all()) and bool(hit[..., 11].isnan().all())
        assert bool(miss.isfinite().all())
        rest = [c for c in range(64) if c not in (7, 9, 11)]
        assert float((hit[..., rest].double() - want[0::2][..., rest]).abs().max()) < 0.05
        b.k_dev.view(b.n_slots, 16, 64)[s, 2, 0] = math.nan  # a NaN logit: nothing of it can be trusted
        b.run(partial=partial, plan=False)
        assert bool(b.out[0::2].isnan().all()) and bool(b.lse[0::2].isnan().all()) and bool(b.out[1::2].isfinite().all())


def test_other_partials_that_are_empty_hold_no_numbers():
    """A side without tokens has no weight, whatever else it holds."""
    b = Batch(10, BF16, 128, 32, 4, 2, [100], [0, 0, -1, -1])
    b.other[2][:] = 0.0
    b.other[0][:] = math.nan
    b.other[1][:] = math.nan
    b.run().check(other=False)


def test_the_partial_in_place_and_two_levels():
    """Prefixes of prefixes: two calls, the second joining its result with the first one's where that lies."""
    for dtype in (BF16, F32):
        low = Batch(11, dtype, 128, 32, 8, 2, [150, 90], _of(2, 12), other=False)
        top = Batch(12, dtype, 128, 32, 8, 2, [700], [0] * 12, other=False)
        top.q = low.q
        low.run(partial=True, result=False)
        o, m, l = low.o, low.m, low.l
        out = torch.empty(12, 16, 128, dtype=dtype, device="cuda")
        B.prefix_plan(top.p, 1, top.blocks, top.of_dev, top.len_dev, top.plan)
        B.shared_prefix_attn(top.p, 1, top.blocks, top.plan, top.q.cuda(), top.k_dev, top.v_dev, top.n_slots, top.table.cuda(), o, m, l, o, m, l,
                             out, None, top.ws)
        a, la, va, ea = low.want()
        b, lb, vb, eb = top.want()
        lse = torch.logaddexp(la, lb)
        wa, wb = (la - lse).exp()[..., None], (lb - lse).exp()[..., None]
        err = (ea + eb + 8 * U + (2.0 ** -15 if dtype == BF16 else 0.0))[..., None]
        off = (o.double().cpu() - (wa * a + wb * b)).abs()
        assert bool((off <= 4 * err * (wa * va + wb * vb) + 1e-30).all())
        assert bool(((m.double() + l.double().log()).cpu() - lse).abs().le(4 * (ea + eb) + 16 * U * lse.abs()).all())
        assert bool((out.double().cpu() - o.double().cpu()).abs().le(2.0 ** -8 * o.double().cpu().abs() + 1e-30).all())


def test_a_plan_of_another_problem_has_no_prefixes():
    b = Batch(13, BF16, 128, 32, 4, 2, [500], [0] * 6)
    B.prefix_plan(b.p, 1, b.blocks + 1, b.of_dev, b.len_dev, b.plan)
    b.run(plan=False)
    o_b, m_b, l_b = b.other
    want = torch.where(l_b[..., None] > 0, o_b, torch.zeros_like(o_b))
    assert bool(((b.out.cpu().float() - want).abs() <= 2.0 ** -8 * want.abs() + 8 * U).all())
    b.plan.zero_()
    b.run(plan=False)
    assert bool(((b.out.cpu().float() - want).abs() <= 2.0 ** -8 * want.abs() + 8 * U).all())


@pytest.mark.parametrize("dtype,n", [(BF16, 4), (BF16, 40), (F32, 6)])
def test_captured_and_on_a_side_stream(dtype, n):
    """Plan and attention captured once; prefixes, lengths, queries and tables change between the replays.  The results have the
    bits of the eager calls."""
    b = Batch(14, dtype, 128, 32, 4, 2, [640, 320], [0] * n, other=False)
    q, table = b.q.cuda(), b.table.cuda()
    out, lse = torch.empty(n, 8, 128, dtype=dtype, device="cuda"), torch.empty(n, 8, device="cuda")
    ws, plan = B.alloc_workspace(b.p), B.alloc_prefix_plan(b.p, 2)

    def step():
        B.prefix_plan(b.p, 2, b.blocks, b.of_dev, b.len_dev, plan)
        for _ in range(2):
            B.shared_prefix_attn(b.p, 2, b.blocks, plan, q, b.k_dev, b.v_dev, b.n_slots, table, None, None, None, None, None, None, out, lse, ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    gen = torch.Generator(device="cuda").manual_seed(1)
    for turn in range(4):
        b.of_dev.copy_(torch.randint(-1, 2, (n,), generator=gen, device="cuda"))
        b.len_dev.copy_(torch.randint(1, 641, (2,), generator=gen, device="cuda").clamp(max=torch.tensor([640, 320], device="cuda")))
        q.copy_(torch.randn(n, 8, 128, generator=gen, device="cuda"))
        b.k_dev.nan_to_num_(0.0), b.v_dev.nan_to_num_(0.0)
        graph.replay()
        torch.cuda.synchronize()
        b.q, b.of, b.lens = q.cpu(), b.of_dev.tolist(), b.len_dev.tolist()
        b.k, b.v = b.k_dev.cpu(), b.v_dev.cpu()
        b.run().check()
        assert torch.equal(b.out, out) and torch.equal(b.lse, lse), turn


def test_two_calls_at_once():
    """One plan, two layers on two streams, each with a workspace of its own."""
    a, c = (Batch(s, BF16, 128, 32, 8, 2, [3000], [0] * 24, other=False) for s in (15, 16))
    a.run().check()
    c.run().check()
    want = a.out.clone(), c.out.clone()
    streams = [torch.cuda.Stream() for _ in range(2)]
    q, table = [x.q.cuda() for x in (a, c)], [x.table.cuda() for x in (a, c)]
    torch.cuda.synchronize()
    for _ in range(5):
        for i, x in enumerate((a, c)):
            x.out.zero_()
            streams[i].wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(streams[i]):
                B.shared_prefix_attn(x.p, 1, x.blocks, a.plan, q[i], x.k_dev, x.v_dev, x.n_slots, table[i], None, None, None, None, None, None,
                                     x.out, x.lse, x.ws)
        torch.cuda.synchronize()
        assert torch.equal(a.out, want[0]) and torch.equal(c.out, want[1])


def test_rows_of_a_long_pool():
    """Slots whose tiles lie beyond 4 GiB of the pool."""
    S, d, Hkv = 64, 128, 1
    n_slots = 300_000   # 16 KiB each: 4.9 GB
    k = torch.zeros(n_slots, S, d, dtype=BF16, device="cuda")
    v = torch.zeros(n_slots, S, d, dtype=BF16, device="cuda")
    for n in (2, 40):
        b = Batch(17, BF16, d, S, 4, Hkv, [300], [0] * n, other=False)
        far = torch.arange(n_slots - b.n_slots, n_slots)
        k[far], v[far] = b.k.cuda(), b.v.cuda()
        b.table = torch.where(b.table >= 0, b.table + n_slots - b.n_slots, b.table)
        small = b.k, b.v
        b.k_dev, b.v_dev, b.n_slots = k, v, n_slots
        b.run()
        b.table = torch.where(b.table >= 0, b.table - (n_slots - len(small[0])), b.table)
        b.check()


def test_both_marshallers_pass_the_same():
    """A recorded call (ctypes) does what the call itself does (the extension module)."""
    b = Batch(18, BF16, 128, 32, 4, 2, [200, 77], _of(2, 6)).run(partial=True)
    eager = [t.clone() for t in (b.out, b.lse, b.o, b.m, b.l)]
    q, table, other = b.q.cuda(), b.table.cuda(), [t.cuda() for t in b.other]
    for t in (b.out, b.lse, b.o, b.m, b.l):
        t.zero_()
    b.plan.zero_()
    calls = [B.prepare(B.prefix_plan, b.p, 2, b.blocks, b.of_dev, b.len_dev, b.plan),
             B.prepare(B.shared_prefix_attn, b.p, 2, b.blocks, b.plan, q, b.k_dev, b.v_dev, b.n_slots, table, *other, b.o, b.m, b.l, b.out,
                       b.lse, b.ws)]
    for c in calls:
        c()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(eager, (b.out, b.lse, b.o, b.m, b.l)))


def test_graphs_that_share_a_workspace():
    """Two captured batches with one workspace, replayed in turn."""
    a, c = (Batch(s, BF16, 128, 32, 8, 2, [1500, 40], _of(2, 14), other=False) for s in (19, 20))
    a.run().check()
    c.run().check()
    want = [(x.out.clone(), x.lse.clone()) for x in (a, c)]
    ws = a.ws
    graphs, keep = [], []
    for x in (a, c):
        q, table, graph = x.q.cuda(), x.table.cuda(), torch.cuda.CUDAGraph()
        keep.append((q, table))
        with torch.cuda.graph(graph):
            B.shared_prefix_attn(x.p, 2, x.blocks, x.plan, q, x.k_dev, x.v_dev, x.n_slots, table, None, None, None, None, None, None, x.out, x.lse, ws)
        graphs.append(graph)
    for turn in range(4):
        for x in (a, c):
            x.out.zero_(), x.lse.zero_()
        for g in graphs if turn % 2 else graphs[::-1]:
            g.replay()
        torch.cuda.synchronize()
        for x, (out, lse) in zip((a, c), want):
            assert torch.equal(x.out, out) and torch.equal(x.lse, lse), turn


@pytest.mark.parametrize("n", [3, 30])
def test_neighbours_are_left_alone(n):
    b = Batch(21, BF16, 64, 16, 4, 1, [130, 17], _of(2, n), other=False)
    sizes = dict(out=n * 4 * 64, lse=n * 4, o=n * 4 * 64, m=n * 4, l=n * 4)
    bufs = {k: torch.full((v + 128,), 7.0, dtype=b.dtype if k == "out" else F32, device="cuda") for k, v in sizes.items()}
    at = {k: bufs[k][64:64 + v] for k, v in sizes.items()}
    plan = torch.full((b.plan.numel() + 1024,), 0x5a, dtype=torch.uint8, device="cuda")
    inner = plan[512:512 + b.plan.numel()]
    B.prefix_plan(b.p, 2, b.blocks, b.of_dev, b.len_dev, inner)
    B.shared_prefix_attn(b.p, 2, b.blocks, inner, b.q.cuda(), b.k_dev, b.v_dev, b.n_slots, b.table.cuda(), None, None, None, at["o"], at["m"],
                         at["l"], at["out"], at["lse"], b.ws)
    torch.cuda.synchronize()
    b.out, b.lse, b.o, b.m, b.l = (at[k].view(n, 4, -1).squeeze(-1) if sizes[k] == n * 4 else at[k].view(n, 4, 64) for k in ("out", "lse", "o", "m", "l"))
    b.check()
    for k, v in sizes.items():
        assert bool((bufs[k][:64] == 7.0).all()) and bool((bufs[k][64 + v:] == 7.0).all()), k
    assert bool((plan[:512] == 0x5a).all()) and bool((plan[512 + b.plan.numel():] == 0x5a).all())


def test_many_prefixes():
    """As many as a plan takes, most of them nobody's."""
    P, n = 2048, 70
    lens = [(7 * i) % 45 for i in range(P)]
    Batch(22, BF16, 64, 16, 2, 1, lens, [(29 * b) % P for b in range(n)], other=False).run().check()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_long_prefix_in_many_splits(dtype):
    """Windows of units, and of a wave's list entries, one after the other; blocks without a slot in between."""
    for n, G in ((1, 2), (20, 8)):
        Batch(23, dtype, 64, 16, G, 1, [70_003], [0] * n, p_host=0.4, other=False).run().check()


def test_many_prefixes_that_somebody_has():
    """More prefixes than the planning workgroup has threads, more sequences than that too."""
    P, n = 1500, 1700
    lens = [(13 * i) % 37 for i in range(P)]
    Batch(24, BF16, 64, 16, 1, 1, lens, [(11 * b) % P if b % 5 else -1 for b in range(n)], other=False).run().check()
