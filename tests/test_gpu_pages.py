"""Forking, freeing, reserving and compacting pages against a cache kept block by block on the CPU: tables, lengths, digests,
tiles, counts and lists bit for bit, through random sequences of calls and at the ends of their ranges."""
import numpy as np
import pytest
import torch

from paper_2603_27138_amd import binding as B
from tests.pages_oracle import Book

pytestmark = pytest.mark.gpu


class Cache:
    """Device arrays and their image on the CPU."""

    def __init__(self, rng, Bn, Hkv, S, d, dtype, mb, n_slots, ctx, digest_kind=0, paired=False, share=0.7, G=2, spread=None):
        self.S, self.Bn, self.Hkv, self.mb, self.n_slots = S, Bn, Hkv, mb, n_slots
        code = B.F32 if dtype == torch.float32 else B.BF16
        bits = np.uint32 if dtype == torch.float32 else np.uint16
        draw = lambda *shape: rng.integers(0, 1 << 12, shape).astype(bits)  # noqa: E731  (small numbers: finite floats)
        table = np.full((Bn, Hkv, mb), -1, np.int32)
        slots = iter(rng.permutation(spread or n_slots).tolist())
        for b in range(Bn):
            nb = min((max(0, ctx[b]) + S - 1) // S, mb)
            for g in range(Hkv):
                for j in range(nb):
                    if rng.random() < share:
                        table[b, g, j] = next(slots, -1)
        elem = (d,) if digest_kind else (2, d)
        digest = draw(Bn, Hkv, mb, *elem) if not digest_kind else rng.integers(0, 1 << 12, (Bn, Hkv, mb, d)).astype(np.uint32)
        pools = [draw(n_slots, S * d) for _ in range(2)]
        self.book = Book(S, np.array(ctx, np.int32), table, digest, *pools)
        dev = lambda x: torch.from_numpy(x.view(np.int16) if x.dtype == np.uint16 else x.view(np.int32)).cuda()  # noqa: E731
        self.ctx, self.table, self.digest = dev(self.book.ctx.copy()), dev(self.book.table.copy()), dev(digest)
        if paired:
            self.pool = torch.stack([dev(p) for p in pools], 1).contiguous()
            self.k_pool, self.v_pool, stride = self.pool.view(-1)[:], self.pool.view(-1)[S * d:], 2 * S * d
        else:
            self.pool, stride = None, 0
            self.k_pool, self.v_pool = (dev(p) for p in pools)
        self.p = B.make_problem(Bn, G * Hkv, Hkv, d, S, code, mb, 1, self.ctx, digest_kind=digest_kind, tile_stride=stride)
        self.pages = B.alloc_pages(n_slots)
        self.pages.fill_(-0x11111111)
        B.pages_init(self.p, self.ctx, self.table, n_slots, self.pages)
        self.check("init")

    def cache(self):
        return self.ctx, self.digest, self.table, self.k_pool, self.v_pool, self.n_slots, self.pages

    def check(self, what):
        bk = self.book
        assert np.array_equal(self.ctx.cpu().numpy(), bk.ctx), what
        assert np.array_equal(self.table.cpu().numpy(), bk.table), what
        assert np.array_equal(self.pages[:self.n_slots].cpu().numpy(), bk.refs), what
        assert np.array_equal(self.digest.cpu().numpy().view(bk.digest.dtype), bk.digest), what
        pools = (self.pool[:, 0], self.pool[:, 1]) if self.pool is not None else (self.k_pool, self.v_pool)
        for dev, cpu in zip(pools, (bk.k_pool, bk.v_pool)):
            assert np.array_equal(dev.cpu().numpy().view(cpu.dtype), cpu), what

    def fork(self, src, dst, deep=False):
        i32 = dict(dtype=torch.int32, device="cuda")
        status = torch.full((len(src),), 77, **i32)
        B.fork_sequences(self.p, torch.tensor(src, **i32), torch.tensor(dst, **i32), deep, *self.cache(), status)
        want = self.book.fork(src, dst, deep)
        assert status.cpu().tolist() == want.tolist(), (src, dst, deep)
        self.check(("fork", src, dst, deep))
        return want

    def free(self, seq):
        B.free_sequences(self.p, torch.tensor(seq, dtype=torch.int32, device="cuda"), self.ctx, self.table, self.n_slots, self.pages)
        self.book.free(seq)
        self.check(("free", seq))

    def reserve(self):
        new = torch.full((self.Bn, self.Hkv), 77, dtype=torch.int32, device="cuda")
        short = torch.full((1,), 77, dtype=torch.int32, device="cuda")
        B.reserve_blocks(self.p, self.ctx, self.n_slots, self.pages, new, short)
        want, missing = self.book.reserve()
        assert np.array_equal(new.cpu().numpy(), want) and short.item() == missing
        self.check("reserve")
        return new, want

    def advance(self):
        """The next token's blocks and lengths, as append_token would leave them (its own tests look at the rest)."""
        _, want = self.reserve()
        for b in range(self.Bn):
            t = self.book.ctx[b]
            if 0 <= t < self.mb * self.S:
                if t % self.S == 0:
                    self.book.table[b, :, t // self.S] = want[b]
                self.book.ctx[b] = t + 1
        self.ctx.copy_(torch.from_numpy(self.book.ctx))
        self.table.copy_(torch.from_numpy(self.book.table))

    def compact(self):
        where = torch.full((self.n_slots,), 77, dtype=torch.int32, device="cuda")
        live = torch.full((1,), 77, dtype=torch.int32, device="cuda")
        B.compact_pool(self.p, self.table, self.k_pool, self.v_pool, self.n_slots, self.pages, where, live)
        want, n = self.book.compact()
        assert np.array_equal(where.cpu().numpy(), want) and live.item() == n
        self.check("compact")


SHAPES = [  # Hkv, S, d, dtype, digest_kind, paired pools
    (1, 16, 64, torch.bfloat16, 0, False), (2, 32, 128, torch.bfloat16, 0, False), (3, 16, 64, torch.float32, 0, True),
    (2, 64, 128, torch.float32, 0, False), (2, 64, 64, torch.bfloat16, 1, False), (1, 32, 128, torch.bfloat16, 1, True),
]


@pytest.mark.parametrize("seed", range(3))
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"h{s[0]}-S{s[1]}-d{s[2]}-{str(s[3])[6:]}-{s[4]}{s[5]}")
def test_random_calls(shape, seed):
    Hkv, S, d, dtype, kind, paired = shape
    rng = np.random.default_rng([seed, S, d, Hkv])
    Bn, mb = 7, 5
    ctx = [int(rng.integers(1, mb * S)), -1, int(rng.integers(1, mb * S)), -1, 0, -1, S]
    # room for about half of what the calls ask for
    c = Cache(rng, Bn, Hkv, S, d, dtype, mb, int(rng.integers(12, 40)) * Hkv, ctx, kind, paired)
    for _ in range(12):
        do = rng.choice(["fork", "deep", "free", "advance", "compact"], p=[0.35, 0.15, 0.2, 0.15, 0.15])
        if do in ("fork", "deep"):
            n = int(rng.integers(1, 4))
            c.fork(rng.integers(0, Bn, n).tolist(), rng.integers(0, Bn, n).tolist(), bool(do == "deep"))
        elif do == "free":
            c.free(rng.integers(-1, Bn + 1, int(rng.integers(1, 4))).tolist())
        elif do == "advance":
            c.advance()
        else:
            c.compact()


@pytest.mark.parametrize("deep", [False, True])
def test_lengths(deep):
    """Parents of every kind of length: none, empty, one token, a block less one, a block, one more, all blocks, the last not full."""
    S, mb, rng = 16, 3, np.random.default_rng(4)
    lens = [-1, 0, 1, S - 1, S, S + 1, mb * S - 1, mb * S]
    c = Cache(rng, 2 * len(lens), 2, S, 64, torch.bfloat16, mb, 200, lens + [-1] * len(lens), share=1.0)
    n = len(lens)
    assert (c.fork(list(range(n)), list(range(n, 2 * n)), deep) == 0).all()
    c.advance()
    c.free(list(range(0, 2 * n, 2)))
    c.compact()
    c.free(list(range(1, 2 * n, 2)))
    assert not c.book.refs.any()
    c.compact()


def test_refused_forks_change_nothing():
    rng = np.random.default_rng(5)
    c = Cache(rng, 6, 2, 16, 64, torch.bfloat16, 3, 64, [40, 33, -1, -1, -1, 7])
    big = 2 ** 31 - 1
    # out of range, onto itself, onto a sequence with tokens, onto a parent, the same child twice
    assert c.fork([0, -1, 6, 0], [6, 2, 2, -1]).tolist() == [-1, -1, -1, -1]
    assert c.fork([0, big, -big - 1], [0, 2, 3]).tolist() == [-1, -1, -1]
    assert c.fork([0, 0, 1], [1, 5, 2]).tolist() == [-1, -1, 0]
    assert c.fork([0, 3], [3, 4]).tolist() == [-1, 0]   # 3 is a parent, with nothing to give
    assert c.fork([0, 1], [3, 3], True).tolist() == [0, -1]


def test_no_slots_left():
    rng = np.random.default_rng(6)
    S = 16
    c = Cache(rng, 4, 2, S, 64, torch.bfloat16, 4, 11, [3 * S + 5, -1, -1, 0], share=1.0)  # holds eight of eleven slots
    assert c.fork([0, 0], [1, 2]).tolist() == [0, 1]     # three are left for four tails
    new, want = c.reserve()
    assert (want == -1).all()
    c.free([1])
    c.reserve()
    c.free([2, 3, 0])
    c.fork([0], [1], True)


def test_pool_without_slots():
    rng = np.random.default_rng(7)
    c = Cache(rng, 3, 1, 16, 64, torch.bfloat16, 2, 0, [20, -1, -1])
    assert c.fork([0], [1]).tolist() == [0]
    c.advance()
    c.compact()
    c.free([0, 1, 2])


@pytest.mark.parametrize("n_slots", [1, 31, 32, 33, 64, 1000, 33000, 70001])
def test_slots_over_many_words(n_slots):
    """Takers and holes that lie in one word, at its ends, and beyond the words that one trip looks at."""
    rng = np.random.default_rng(n_slots)
    Bn, mb, S = 4, 64, 16
    c = Cache(rng, Bn, 2, S, 64, torch.bfloat16, mb, n_slots, [mb * S - 3, 17, -1, -1], share=1.0)
    # everything below a high slot is held by others
    if n_slots > 40:
        held = torch.zeros(n_slots, dtype=torch.bool)
        held[:n_slots - 300] = torch.from_numpy(rng.random(max(0, n_slots - 300)) < 0.999)
        extra = np.flatnonzero(held.numpy() & (c.book.refs == 0))
        words = -(-n_slots // 64) * 64
        c.book.refs[extra] = 1
        c.pages[:n_slots].copy_(torch.from_numpy(c.book.refs))
        bits = np.zeros(-(-n_slots // 32) * 32, np.uint8)
        bits[:n_slots] = c.book.refs > 0
        used = np.packbits(bits.reshape(-1, 32), axis=1, bitorder="little").view(np.int32).ravel()
        c.pages[words:words + len(used)].copy_(torch.from_numpy(used.copy()))
    c.fork([0, 1], [2, 3], True)
    c.free([0])
    c.compact()
    c.fork([2], [0])
    c.compact()


def test_entries_that_name_no_slot():
    """Entries outside the pool are blocks on the host to a fork, and left alone by a compaction; a slot that nobody holds stays free."""
    rng = np.random.default_rng(8)
    c = Cache(rng, 3, 2, 16, 64, torch.bfloat16, 4, 40, [50, -1, -1], share=1.0)
    c.table[0, 0, 1] = c.book.table[0, 0, 1] = 40
    c.table[0, 1, 2] = c.book.table[0, 1, 2] = 2 ** 31 - 1
    c.table[0, 1, 0] = c.book.table[0, 1, 0] = -7
    B.pages_init(c.p, c.ctx, c.table, c.n_slots, c.pages)
    c.book.init()
    c.fork([0], [1])
    c.fork([0], [2], True)
    c.free([1])
    c.compact()
    unheld = int(np.flatnonzero(c.book.refs == 0)[0])
    c.table[2, 0, 0] = c.book.table[2, 0, 0] = unheld
    c.free([2])


def test_entries_beyond_the_last_block():
    """They are no blocks to begin with; an entry that a caller leaves behind there (a sequence cut short) is given back with the rest."""
    rng = np.random.default_rng(12)
    c = Cache(rng, 3, 2, 16, 64, torch.bfloat16, 5, 40, [40, -1, 16], share=1.0)
    c.table[0, :, 3:] = c.book.table[0, :, 3:] = 39
    c.table[1] = c.book.table[1] = 5
    B.pages_init(c.p, c.ctx, c.table, c.n_slots, c.pages)
    c.book.init()
    c.check("init")
    c.ctx[0] = c.book.ctx[0] = 20
    c.fork([0], [1])
    c.free([0, 1])
    assert c.book.refs.sum() == 2


def test_shared_slots_given_back_together():
    """Forks of two parents freed in lists that mix them, and a slot that several entries of one sequence name."""
    rng = np.random.default_rng(13)
    c = Cache(rng, 30, 1, 16, 64, torch.bfloat16, 4, 64, [50, 64] + [-1] * 28, share=1.0)
    c.fork([0, 1] * 10, list(range(2, 22)))
    c.fork([0] * 5, list(range(22, 27)))
    c.free([2, 3, 4, 5, 6, 7, 8, 9, 10, 25, 11, 2, 3])
    c.free([0])
    c.free(list(range(30)))
    assert not c.book.refs.any()
    c.table[4] = c.book.table[4] = 7
    c.ctx[4] = c.book.ctx[4] = 64
    B.pages_init(c.p, c.ctx, c.table, c.n_slots, c.pages)
    c.book.init()
    c.fork([4], [5])
    c.free([4])
    c.free([5])


@pytest.mark.parametrize("n", [40, 1500])
def test_long_lists(n):
    """More forks than one round of the plan looks at, children listed twice within and across rounds."""
    rng = np.random.default_rng(n)
    rows = 2 * n + 3
    c = Cache(rng, rows, 1, 16, 64, torch.bfloat16, 3, 3000, [33, 20, -1] + [-1] * (2 * n), share=1.0)
    dst = list(range(3, 3 + n))
    dst[n // 3], dst[-1] = 5, 3
    src = rng.integers(0, 2, n).tolist()
    status = c.fork(src, dst)
    assert (status == -1).sum() == 2
    c.free(rng.integers(0, rows, n).tolist())
    c.compact()


def test_empty_lists_and_a_side_stream():
    rng = np.random.default_rng(9)
    c = Cache(rng, 4, 2, 32, 128, torch.bfloat16, 4, 64, [100, -1, -1, 31])
    c.fork([], [])
    c.free([])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.fork([0, 3], [1, 2])
        c.free([0])
        c.compact()
    torch.cuda.current_stream().wait_stream(side)
    c.check("after")


def test_captured_steps():
    """A step of sampling (old answers freed, new ones forked, blocks reserved, tokens appended) captured once and replayed, with
    eager work between the replays, leaves what the eager calls leave."""
    S, d, Hkv, n, mb = 16, 64, 2, 5, 6
    gen = torch.Generator(device="cuda").manual_seed(3)
    rows = n + 2
    i32 = dict(dtype=torch.int32, device="cuda")

    def fresh():
        g = torch.Generator(device="cuda").manual_seed(3)
        x = dict(ctx=torch.tensor([-1] * n + [4 * S, 2 * S + 3], **i32), table=torch.full((rows, Hkv, mb), -1, **i32), slots=80)
        x["table"][n, :, :4] = torch.arange(8, **i32).view(2, 4)
        x["table"][n + 1, :, :3] = 8 + torch.arange(6, **i32).view(2, 3)
        x["digest"] = torch.randn(rows, Hkv, mb, 2, d, generator=g, device="cuda").bfloat16()
        x["k"], x["v"] = (torch.randn(80, S, d, generator=g, device="cuda").bfloat16() for _ in range(2))
        x["p"] = B.make_problem(rows, Hkv, Hkv, d, S, B.BF16, mb, 1, x["ctx"])
        x["answers"] = B.make_problem(n, Hkv, Hkv, d, S, B.BF16, mb, 1, x["ctx"])
        x["pages"] = B.alloc_pages(80)
        B.pages_init(x["p"], x["ctx"], x["table"], 80, x["pages"])
        x["new"], x["short"], x["status"] = torch.zeros(n, Hkv, **i32), torch.zeros(1, **i32), torch.zeros(n, **i32)
        x["src"], x["dst"] = torch.tensor([n, n + 1, n, n + 1, n], **i32), torch.arange(n, **i32)
        x["kn"], x["vn"] = torch.zeros(n, Hkv, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, Hkv, d, dtype=torch.bfloat16, device="cuda")
        return x

    def step(x):
        cache = (x["ctx"], x["digest"], x["table"], x["k"], x["v"], 80, x["pages"])
        B.free_sequences(x["p"], x["dst"], x["ctx"], x["table"], 80, x["pages"])
        B.fork_sequences(x["p"], x["src"], x["dst"], False, *cache, x["status"])
        B.reserve_blocks(x["answers"], x["ctx"], 80, x["pages"], x["new"], x["short"])
        B.append_token(x["answers"], x["ctx"], x["kn"], x["vn"], x["new"], x["digest"], x["table"], x["k"], x["v"], 80)

    eager, captured = fresh(), fresh()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(captured)
    for turn in range(4):
        kn, vn = (torch.randn(n, Hkv, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
        parents = torch.randint(n, rows, (n,), generator=gen, **i32)
        for x in (eager, captured):
            x["kn"].copy_(kn)
            x["vn"].copy_(vn)
            x["src"].copy_(parents)
        step(eager)
        graph.replay()
        torch.cuda.synchronize()
        for key in ("ctx", "table", "digest", "k", "v", "new", "short", "status"):
            assert torch.equal(eager[key], captured[key]), (turn, key)
        assert torch.equal(eager["pages"][:80], captured["pages"][:80])
    assert eager["status"].tolist() == [0] * n and eager["short"].item() == 0


def test_tiles_beyond_four_gib():
    """Slots whose tiles lie beyond 4 GiB of a pool: copied by a deep fork, moved by a compaction."""
    S, d, Hkv, n_slots = 64, 128, 1, 150_000   # 32 KiB a tile: 4.9 GB a pool
    i32 = dict(dtype=torch.int32, device="cuda")
    k, v = (torch.zeros(n_slots, S, d, device="cuda") for _ in range(2))
    table, ctx = torch.full((3, Hkv, 4), -1, **i32), torch.tensor([4 * S, -1, -1], **i32)
    far = torch.tensor([n_slots - 1, n_slots - 7, 140_000, 139_999], **i32)
    table[0, 0] = far
    tiles = [torch.randn(4, S, d, device="cuda") for _ in range(2)]
    for pool, t in zip((k, v), tiles):
        pool[far.long()] = t
    digest = torch.zeros(3, Hkv, 4, 2, d, device="cuda")
    p = B.make_problem(3, 1, Hkv, d, S, B.F32, 4, 1, ctx)
    pages = B.alloc_pages(n_slots)
    B.pages_init(p, ctx, table, n_slots, pages)
    held = pages[:n_slots].clone()
    filler = torch.full((1, 1, n_slots), -1, **i32)   # everything but the last slots is somebody's
    filler[0, 0, :n_slots - 20] = torch.arange(n_slots - 20, **i32)
    words = -(-n_slots // 64) * 64
    pages[:n_slots - 20] += 1
    pages[words:words + (n_slots - 20) // 32] = -1
    status = torch.empty(1, **i32)
    B.fork_sequences(p, torch.tensor([0], **i32), torch.tensor([1], **i32), True, ctx, digest, table, k, v, n_slots, pages, status)
    assert status.item() == 0 and int(table[1].min()) >= 149_900
    for pool, t in zip((k, v), tiles):
        assert torch.equal(pool[table[1, 0].long()], t)
    pages[:n_slots] = held
    pages[:n_slots].index_add_(0, table[1, 0].long(), torch.ones(4, **i32))
    bits = (pages[:n_slots] > 0).cpu().numpy().astype(np.uint8)
    bits = np.concatenate([bits, np.zeros(-len(bits) % 32, np.uint8)])
    pages[words:words + len(bits) // 32] = torch.from_numpy(np.packbits(bits.reshape(-1, 32), axis=1, bitorder="little").view(np.int32).ravel().copy()).cuda()
    slot_map, live = torch.empty(n_slots, **i32), torch.empty(1, **i32)
    B.compact_pool(p, table, k, v, n_slots, pages, slot_map, live)
    assert live.item() == 8 and int(table.max()) == 7
    for pool, t in zip((k, v), tiles):
        assert torch.equal(pool[table[0, 0].long()], t) and torch.equal(pool[table[1, 0].long()], t)


def test_neighbours_are_left_alone():
    """What lies around the outputs stays as it is."""
    rng = np.random.default_rng(14)
    c = Cache(rng, 5, 2, 16, 64, torch.bfloat16, 3, 37, [40, 33, -1, -1, 16], share=1.0)
    i32 = dict(dtype=torch.int32, device="cuda")
    guard = lambda n: torch.full((n + 32,), 0x5a5a5a5a, **i32)  # noqa: E731
    bufs = {name: guard(n) for name, n in dict(status=2, new=10, short=1, where=37, live=1).items()}
    of = lambda name, n: bufs[name][16:16 + n]  # noqa: E731
    B.fork_sequences(c.p, torch.tensor([0, 1], **i32), torch.tensor([2, 3], **i32), False, *c.cache(), of("status", 2))
    B.reserve_blocks(c.p, c.ctx, c.n_slots, c.pages, of("new", 10), of("short", 1))
    B.compact_pool(c.p, c.table, c.k_pool, c.v_pool, c.n_slots, c.pages, of("where", 37), of("live", 1))
    torch.cuda.synchronize()
    for name, b in bufs.items():
        n = b.numel() - 32
        assert bool((b[:16] == 0x5a5a5a5a).all()) and bool((b[16 + n:] == 0x5a5a5a5a).all()), name
        assert not bool((b[16:16 + n] == 0x5a5a5a5a).any()), name


def test_both_marshallers_pass_the_same():
    """Recorded calls (ctypes) leave what the calls themselves leave (the extension module)."""
    states = []
    for recorded in (False, True):
        rng = np.random.default_rng(15)
        c = Cache(rng, 6, 2, 16, 64, torch.bfloat16, 4, 60, [50, 32, -1, -1, -1, 20], share=1.0)
        i32 = dict(dtype=torch.int32, device="cuda")
        keep = dict(src=torch.tensor([0, 1], **i32), dst=torch.tensor([2, 3], **i32), gone=torch.tensor([0, 5], **i32),
                    status=torch.empty(2, **i32), new=torch.empty(6, 2, **i32), short=torch.empty(1, **i32), where=torch.empty(60, **i32),
                    live=torch.empty(1, **i32))
        calls = [(B.pages_init, (c.p, c.ctx, c.table, 60, c.pages)),
                 (B.fork_sequences, (c.p, keep["src"], keep["dst"], True, *c.cache(), keep["status"])),
                 (B.free_sequences, (c.p, keep["gone"], c.ctx, c.table, 60, c.pages)),
                 (B.compact_pool, (c.p, c.table, c.k_pool, c.v_pool, 60, c.pages, keep["where"], keep["live"])),
                 (B.reserve_blocks, (c.p, c.ctx, 60, c.pages, keep["new"], keep["short"]))]
        for fn, args in calls:
            B.prepare(fn, *args)() if recorded else fn(*args)
        torch.cuda.synchronize()
        states.append([c.ctx, c.table, c.digest, c.k_pool, c.v_pool, c.pages[:60], *list(keep.values())])
    assert all(torch.equal(x, y) for x, y in zip(*states))


@pytest.mark.parametrize("dtype,d,S", [(torch.bfloat16, 64, 16), (torch.float32, 64, 16)])
def test_rows_of_many_blocks(dtype, d, S):
    """Rows beyond 4096 blocks, with and without a slot, as long as a sequence can be and a few blocks shorter; freed slots that lie side by
    side, and taken again."""
    rng = np.random.default_rng(31)
    mb = 4101
    c = Cache(rng, 6, 1, S, d, dtype, mb, 5 * mb, [mb * S, (mb - 7) * S + 3, -1, -1, -1, -1], share=0.5, G=1)
    assert (c.fork([0, 1, 0], [2, 3, 4], True) == 0).all()
    c.free([2, 4])
    c.fork([1, 3], [2, 4], True)
    c.free([1])
    c.compact()
    c.fork([0], [5])
