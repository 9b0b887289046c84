"""What the entry points for pages and shared prefixes refuse, before anything is launched (so without a GPU)."""
import ctypes

import pytest

from paper_2603_27138_amd import binding as B

X, ODD, BIG = ctypes.c_void_p(0x10000), ctypes.c_void_p(0x10004), 1 << 40


def _problem(**kw):
    base = dict(B=4, Hq=8, Hkv=2, d=128, S=32, dtype=B.BF16, max_blocks=64, k=8, sm_scale=0.0, ctx_len=0x1000)
    base.update(kw)
    return B.Problem(**base)


def _call(name, p, **kw):
    """The entry point with arguments that it would take (aligned addresses that are never looked at), but for kw."""
    order = {
        "scout_pages_init": "p ctx table n_slots pages pages_bytes stream",
        "reserve_blocks": "p ctx n_slots pages pages_bytes new_slot n_short stream",
        "fork_sequences": "p n src dst deep ctx digest table k v n_slots pages pages_bytes status stream",
        "free_sequences": "p n src ctx table n_slots pages pages_bytes stream",
        "compact_pool": "p table k v n_slots pages pages_bytes slot_map n_live stream",
        "scout_prefix_plan": "p n_prefix blocks of len plan plan_bytes stream",
        "shared_prefix_attn": "p n_prefix blocks plan plan_bytes q k v n_slots ptable o_b m_b l_b o m l out lse ws ws_bytes stream",
    }[name].split()
    numbers = dict(n_slots=10, pages_bytes=BIG, plan_bytes=BIG, ws_bytes=BIG, n=2, deep=0, n_prefix=2, blocks=16, stream=None)
    args = []
    for a in order:
        v = kw[a] if a in kw else ctypes.byref(p) if a == "p" and p is not None else None if a == "p" else numbers.get(a, X)
        args.append(v)
    return getattr(B.lib(), name)(*args)


ALL = ["scout_pages_init", "reserve_blocks", "fork_sequences", "free_sequences", "compact_pool", "scout_prefix_plan", "shared_prefix_attn"]


@pytest.mark.parametrize("name", ALL)
@pytest.mark.parametrize("kw,code", [(dict(Hq=7), -1), (dict(B=-1), -1), (dict(dtype=3), -1), (dict(ctx_len=None), -1), (dict(d=96), -2),
                                     (dict(S=8), -2), (dict(Hq=64, Hkv=2), -2), (dict(B=70000), -2), (dict(tile_stride=100), -1)])
def test_bad_problems(name, kw, code):
    assert _call(name, _problem(**kw)) == code
    assert _call(name, None) == -1


@pytest.mark.parametrize("name,kw,code", [
    ("scout_pages_init", dict(ctx=None), -1), ("scout_pages_init", dict(table=None), -1), ("scout_pages_init", dict(n_slots=-1), -1),
    ("scout_pages_init", dict(n_slots=(1 << 29) + 1), -2), ("scout_pages_init", dict(pages=None), -3),
    ("scout_pages_init", dict(pages=ODD), -3), ("scout_pages_init", dict(pages_bytes=1000), -3),
    ("reserve_blocks", dict(ctx=None), -1), ("reserve_blocks", dict(new_slot=None), -1), ("reserve_blocks", dict(n_short=None), -1),
    ("reserve_blocks", dict(pages=None), -3), ("reserve_blocks", dict(n_slots=-1), -1), ("reserve_blocks", dict(pages_bytes=0), -3),
    *[("fork_sequences", {a: None}, -1) for a in ("src", "dst", "ctx", "digest", "table", "k", "v", "status")],
    *[("fork_sequences", {a: ODD}, -1) for a in ("digest", "k", "v")],
    ("fork_sequences", dict(n=-1), -1), ("fork_sequences", dict(n=5), -1), ("fork_sequences", dict(deep=2), -1),
    ("fork_sequences", dict(n_slots=-1), -1), ("fork_sequences", dict(pages=None), -3), ("fork_sequences", dict(pages_bytes=64), -3),
    *[("free_sequences", {a: None}, -1) for a in ("src", "ctx", "table")],
    ("free_sequences", dict(n=-1), -1), ("free_sequences", dict(n=5), -1), ("free_sequences", dict(pages=ODD), -3),
    *[("compact_pool", {a: None}, -1) for a in ("table", "k", "v", "slot_map", "n_live")],
    ("compact_pool", dict(k=ODD), -1), ("compact_pool", dict(pages_bytes=64), -3), ("compact_pool", dict(n_slots=-5), -1),
    ("scout_prefix_plan", dict(of=None), -1), ("scout_prefix_plan", dict(len=None), -1), ("scout_prefix_plan", dict(n_prefix=-1), -1),
    ("scout_prefix_plan", dict(n_prefix=2049), -2), ("scout_prefix_plan", dict(blocks=0), -1), ("scout_prefix_plan", dict(blocks=(1 << 20) + 1), -2),
    ("scout_prefix_plan", dict(plan=None), -3), ("scout_prefix_plan", dict(plan=ODD), -3), ("scout_prefix_plan", dict(plan_bytes=100), -3),
    *[("shared_prefix_attn", {a: None}, -1) for a in ("q", "k", "v", "ptable", "o_b", "m_b", "l_b", "o", "m", "l")],
    *[("shared_prefix_attn", {a: ODD}, -1) for a in ("q", "k", "v", "o_b", "o", "out")],
    ("shared_prefix_attn", dict(out=None), -1),                                  # lse without out
    ("shared_prefix_attn", dict(out=None, lse=None, o=None, m=None, l=None), -1),  # nothing to write
    ("shared_prefix_attn", dict(n_prefix=-1), -1), ("shared_prefix_attn", dict(n_prefix=5000), -2), ("shared_prefix_attn", dict(blocks=0), -1),
    ("shared_prefix_attn", dict(blocks=(1 << 20) + 1), -2), ("shared_prefix_attn", dict(n_slots=-1), -1),
    ("shared_prefix_attn", dict(plan=None), -3), ("shared_prefix_attn", dict(plan=ODD), -3), ("shared_prefix_attn", dict(plan_bytes=100), -3),
    ("shared_prefix_attn", dict(ws=None), -3), ("shared_prefix_attn", dict(ws=ctypes.c_void_p(0x10010)), -3),
    ("shared_prefix_attn", dict(ws_bytes=100), -3),
])
def test_bad_arguments(name, kw, code):
    assert _call(name, _problem(), **kw) == code


@pytest.mark.parametrize("name,problem,kw", [
    # more workgroups than a launch can have
    ("fork_sequences", dict(B=65535, Hq=1, Hkv=1, max_blocks=16384), dict(n=65535, deep=1)),
    ("fork_sequences", dict(B=65535, Hq=1, Hkv=1, max_blocks=16384), dict(n=65535, deep=0)),
    ("scout_prefix_plan", dict(B=1, Hq=8192, Hkv=8192), dict(n_prefix=2048)),
    ("shared_prefix_attn", dict(B=1, Hq=8192, Hkv=8192), dict(n_prefix=2048)),
])
def test_more_than_a_launch_holds(name, problem, kw):
    assert _call(name, _problem(**problem), **kw) == -2


def test_sizes():
    n = ctypes.c_size_t(0)
    L = B.lib()
    assert L.scout_pages_bytes(-1, ctypes.byref(n)) == -1 and L.scout_pages_bytes(5, None) == -1
    assert L.scout_pages_bytes((1 << 29) + 1, ctypes.byref(n)) == -2
    sizes = [B.pages_bytes(s) for s in (0, 1, 1000, 100000, 1 << 29)]
    assert sizes == sorted(sizes) and sizes[0] > 0 and all(s % 4 == 0 for s in sizes) and sizes[-1] > 4 << 29
    p = _problem()
    assert L.scout_prefix_plan_bytes(ctypes.byref(p), -1, ctypes.byref(n)) == -1
    assert L.scout_prefix_plan_bytes(ctypes.byref(p), 2049, ctypes.byref(n)) == -2
    assert L.scout_prefix_plan_bytes(ctypes.byref(p), 1, None) == -1 and L.scout_prefix_plan_bytes(None, 1, ctypes.byref(n)) == -1
    assert 0 < B.prefix_plan_bytes(p, 0) <= B.prefix_plan_bytes(p, 7) <= B.prefix_plan_bytes(p, 2048)
    assert B.prefix_plan_bytes(_problem(ctx_len=None), 3) > 0


def test_nothing_to_do():
    p = _problem(B=0)
    assert _call("scout_prefix_plan", p) == 0 and _call("shared_prefix_attn", p) == 0
    assert _call("fork_sequences", p, n=0) == 0 and _call("free_sequences", p, n=0) == 0
    assert _call("fork_sequences", _problem(), n=0) == 0 and _call("free_sequences", _problem(), n=0) == 0


@pytest.mark.parametrize("name", ["shared_prefix_attn", "scout_prefix_plan", "fork_sequences", "free_sequences"])
def test_a_selection_per_query_head_changes_nothing(name):
    """The cache has a row per KV head whatever the selection: such a problem is taken as any other."""
    assert _call(name, _problem(B=0, per_head=1), n=0) == 0
