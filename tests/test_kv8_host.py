"""8-bit pools and query/key norms, what needs no GPU: layout, plans, refusals."""
import ctypes

import numpy as np
import pytest

import kv8_ref as R
from paper_2312_05516_amd import binding as pv
from paper_2312_05516_amd import workloads as wl

OK, INVALID, UNSUPPORTED, RANGE, WORKSPACE = 0, 1, 2, 3, 4
A = 4096  # an address that is aligned; nothing is launched in these tests


def _plan(make=pv.plan_create_kv8, ctx=(5, 40), new=(3, 1), heads=(4, 2, 64), max_pages=8,
          dtype="f16", pages=64):
    return make(pv.pool_desc(pages, heads[1], heads[2], dtype), heads[0], ctx, new, max_pages)


@pytest.mark.parametrize("d", [64, 128])
def test_offsets_are_the_documented_layout(d):
    desc = pv.pool_desc(3, 5, d, "bf16")
    assert pv.kv8_pool_bytes(desc) == 3 * 5 * 16 * d and pv.kv8_scale_bytes(desc) == 15
    b = wl.custom([16], [16], num_q_heads=5, num_kv_heads=5, head_dim=d, dtype="bf16", pool_pages=3)
    p = R.Pools(b)
    seen = set()
    for page, head, slot, dim in [(0, 0, 0, 0), (2, 4, 15, d - 1), (1, 3, 6, 17), (1, 0, 13, 40)]:
        for at, which in ((pv.kv8_k_offset(desc, page, head, slot, dim), "k"),
                          (pv.kv8_v_offset(desc, page, head, slot, dim), "v")):
            getattr(p, which)[:] = 0
            getattr(p, which)[at] = 9
            codes = p.slots(which, page, head)
            assert codes[slot, dim] == 9 and (codes != 0).sum() == 1
    for slot in range(16):
        for dim in range(d):
            seen.add(("k", pv.kv8_k_offset(desc, 1, 2, slot, dim)))
            seen.add(("v", pv.kv8_v_offset(desc, 1, 2, slot, dim)))
    assert len(seen) == 2 * 16 * d
    for bad in [(3, 0, 0, 0), (0, 5, 0, 0), (0, 0, 16, 0), (0, 0, 0, d), (-1, 0, 0, 0)]:
        assert pv.kv8_k_offset(desc, *bad) == -1 and pv.kv8_v_offset(desc, *bad) == -1
    assert pv.kv8_pool_bytes(pv.pool_desc(3, 5, 96, "f16")) == 0
    assert pv.kv8_scale_bytes(pv.pool_desc(0, 5, 64, "f16")) == 0


def test_definition_of_codes():
    """The tests' own definition against torch's conversion to the type."""
    import torch
    x = np.concatenate([np.linspace(-448, 448, 20001), 2.0 ** np.linspace(-14, 8, 3001)])
    x = x.astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(R.one_nan(R.encode(x.astype(np.float64))), R.one_nan(want))
    codes = np.arange(256, dtype=np.uint8)
    vals = torch.from_numpy(codes).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(R.decode(codes), vals, equal_nan=True)
    for dtype, (lo, hi) in R.E_RANGE.items():  # every code times a scale is a value of the type
        import helpers as H
        for e in (lo, hi):
            most = 240.0 if e == hi else 448.0
            x = R.VALUES[R.VALUES <= most] * 2.0 ** e
            assert np.array_equal(H.bits_to_f64(H.f64_to_bits(x, dtype), dtype), x)


def test_plans_for_8_bit_pools():
    p = _plan()
    assert pv.plan_is_kv8(p) and not pv.plan_is_kv8(_plan(pv.plan_create))
    assert pv._lib.pv_plan_is_kv8(None) == -1
    assert pv.plan_total_q(p) == 4
    # the same kernels as for 16-bit pools: long prompts, prompts, generation steps
    for ctx, new, kind in (((20000,) * 8, (512,) * 8, 3), ((900, 300), (100, 90), 1), ((900, 300), (1, 1), 0)):
        q = _plan(ctx=ctx, new=new, heads=(64, 8, 128), max_pages=2000, pages=20000)
        assert [pv.plan_num_work_items(q, k) > 0 for k in (0, 1, 3)] == [kind == k for k in (0, 1, 3)]
        assert pv.plan_kernel_variants(q) == {0: 2 + 32, 1: 0, 3: 16}[kind]
    for ctx, variants in (((900,) * 33, 2), ((900,) * 32, 2 + 32), ((250,) * 32, 2), ((250, 256), 2 + 32)):
        q = _plan(ctx=ctx, new=(1,) * len(ctx), heads=(64, 8, 128), max_pages=60, pages=2000)
        assert pv.plan_kernel_variants(q) == variants
    for bad, status in (((pv.pool_desc(4, 2, 96, "f16"), 4, [1], [1], 4), UNSUPPORTED),
                        ((pv.pool_desc(4, 2, 64, "f16"), 3, [1], [1], 4), INVALID),
                        ((pv.pool_desc(4, 2, 64, "f16"), 4, [-1], [1], 4), INVALID),
                        ((pv.pool_desc(4, 2, 64, "f16"), 4, [64], [1], 4), RANGE)):
        with pytest.raises(pv.PvError) as e:
            pv.plan_create_kv8(*bad)
        assert e.value.status == status


def test_page_table_with_one_writer_a_page():
    p = _plan(ctx=(5, 21), new=(30, 3))  # pages 0..2, of which 0..2 are written; 0..1, of which 1 is
    ok = np.full((2, 8), -1, np.int32)
    ok[0, :3], ok[1, :2] = (3, 4, 5), (6, 7)
    assert pv.plan_check_page_table(p, ok) == OK
    shared = ok.copy()
    shared[1, 0] = 4  # read by one request, written by the other
    assert pv.plan_check_page_table(p, shared) == OK
    both = ok.copy()
    both[1, 1] = 5    # other slots of a page that the first request writes
    assert pv.plan_check_page_table(p, both) == INVALID
    assert pv.plan_check_page_table(p, both, check_append_unique=False) == OK
    twice = ok.copy()
    twice[0, 2] = 4
    assert pv.plan_check_page_table(p, twice) == INVALID
    out = ok.copy()
    out[1, 1] = 64
    assert pv.plan_check_page_table(p, out) == RANGE


def _pool(**change):
    f = {"k": A, "v": A, "k_scales": A + 1, "v_scales": A + 3} | change
    return ctypes.byref(pv._Kv8Ptrs(*(f[n] for n in ("k", "v", "k_scales", "v_scales"))))


def _call(name, p, pool=None, **change):
    """Status of an entry point with good arguments but for `change`."""
    a = {"q": A, "out": A, "k": A, "v": A, "qw": A, "kw": A, "eps": 1e-6, "cs": A, "max_pos": 4096,
         "style": 0, "pt": A, "scale": 0.1, "ws": A, "bytes": 1 << 40} | change
    pool = _pool() if pool is None else pool
    h = p.handle if p is not None else None
    if name == "append":
        return pv._lib.pv_kv8_append_planned(h, a["k"], a["v"], a["pt"], pool, None)
    if name == "read":
        return pv._lib.pv_kv8_read_planned(h, pool, a["pt"], a["k"], a["v"], None)
    if name == "attend":
        return pv._lib.pv_kv8_multi_token_paged_attn_planned(h, a["q"], pool, a["pt"], a["scale"],
                                                             a["out"], a["ws"], a["bytes"], None)
    args = (h, a["q"], a["out"], a["k"], a["v"], a["qw"], a["kw"], a["eps"], a["cs"], a["max_pos"],
            a["style"], a["pt"])
    if name == "norm8":
        return pv._lib.pv_kv8_norm_rope_append_planned(*args, pool, None)
    assert name == "norm16"
    return pv._lib.pv_norm_rope_kv_append_planned(*args, A, A, None)


EIGHT = ["append", "read", "attend", "norm8"]


@pytest.mark.parametrize("name", EIGHT + ["norm16"])
def test_calls_without_a_plan_of_their_kind_are_refused(name):
    assert _call(name, None) == INVALID
    assert _call(name, _plan(pv.plan_create if name in EIGHT else pv.plan_create_kv8)) == INVALID
    # nor one whose lists are on no device
    assert _call(name, _plan(pv.plan_create_kv8 if name in EIGHT else pv.plan_create)) == INVALID


def test_16_bit_calls_refuse_plans_for_8_bit_pools():
    p = _plan()
    lib = pv._lib
    assert lib.pv_kv_append_planned(p.handle, A, A, A, A, A, None) == INVALID
    assert lib.pv_rope_kv_append_planned(p.handle, A, A, A, A, A, 4096, 0, A, A, A, None) == INVALID
    assert lib.pv_multi_token_paged_attn_planned(p.handle, A, A, A, A, 0.1, A, A, 1 << 40, None) == INVALID
    assert lib.pv_multi_token_paged_attn_noalloc(p.handle, A, A, A, A, 0.1, A, None) == INVALID


@pytest.mark.parametrize("name", EIGHT + ["norm16"])
def test_bad_arguments_are_refused(name):
    p = _plan(pv.plan_create_kv8 if name in EIGHT else pv.plan_create)
    names = {"append": ["k", "v", "pt"], "read": ["k", "v", "pt"], "attend": ["q", "out", "pt"]}
    for n in names.get(name, ["k", "v", "pt", "cs"]):
        assert _call(name, p, **{n: None}) == INVALID
        if n != "pt":
            assert _call(name, p, **{n: A + 8}) == INVALID
    if name in EIGHT:
        for n in ("k", "v", "k_scales", "v_scales"):
            assert _call(name, p, pool=_pool(**{n: None})) == INVALID
        assert _call(name, p, pool=_pool(k=A + 8)) == INVALID
        assert _call(name, p, pool=_pool(v=A + 1)) == INVALID
        assert _call(name, p, pool=ctypes.POINTER(pv._Kv8Ptrs)()) == INVALID
    if name.startswith("norm"):
        for eps in (0.0, -1e-6, float("nan"), float("inf")):
            assert _call(name, p, eps=eps) == INVALID
        assert _call(name, p, style=2) == INVALID and _call(name, p, style=-1) == INVALID
        assert _call(name, p, out=None) == INVALID and _call(name, p, q=None) == INVALID
        assert _call(name, p, qw=A + 2) == INVALID and _call(name, p, kw=A + 8) == INVALID
        assert _call(name, p, max_pos=40) == RANGE   # positions 5..7 and 40
    if name == "attend":
        for scale in (float("nan"), float("inf")):
            assert _call(name, p, scale=scale) == INVALID
        long = _plan(ctx=(100000,), new=(1,), heads=(8, 1, 128), max_pages=6251, pages=6300)
        assert pv.plan_workspace_bytes(long) > 0
        for ws in ({"ws": None}, {"bytes": 16}, {"ws": A + 16}):
            assert _call(name, long, **ws) == WORKSPACE


@pytest.mark.parametrize("name", EIGHT + ["norm16"])
def test_batches_without_new_tokens_launch_nothing(name):
    for ctx, new in (((), ()), ((5, 7), (0, 0))):
        p = _plan(pv.plan_create_kv8 if name in EIGHT else pv.plan_create, ctx=ctx, new=new)
        assert _call(name, p) == OK


def test_pool_of_tensors_that_are_not_contiguous_is_refused():
    import torch
    t = torch.zeros(64, 2, dtype=torch.uint8)
    with pytest.raises(ValueError):
        pv.Kv8Pool(t[:, 0], t, t, t)


def test_generated_code_of_the_256_row_kernel_over_8_bit_pools():
    """As test_isa_check has it for 16-bit pools: pinned matrix-core instructions, no operand written
    right in front of one, no spills."""
    import os
    from paper_2312_05516_amd import build as pv_build
    from paper_2312_05516_amd import isa_check
    for src in pv_build.ISA_CHECKED_KV8:
        if not os.path.exists(pv_build.isa_path(src)):
            pv_build.build(verbose=False)
        with open(pv_build.isa_path(src)) as f:
            text = f.read()
        pinned, hazards = isa_check.pinned_mfma_hazards(text)
        assert pinned >= 64 and hazards == []
        spills = isa_check.spill_counts(text)
        assert len(spills) == 2 and all(n == 0 for n in spills.values()), spills


def test_tiles_over_long_contexts_have_room_for_their_page_ids(monkeypatch):
    """The 256-row kernel keeps the page ids of an item in LDS, 8192 of them, however the list is cut."""
    monkeypatch.setenv("PV_TILE_MIN_KEYS", "64")
    for ctx in ((300000,), (400000, 20), (131072 - 256,), (131072,), (1000000,) * 3):
        p = _plan(ctx=ctx, new=(256,) * len(ctx), heads=(8, 1, 128), max_pages=70000, pages=200000)
        items = [pv.plan_work_item(p, 3, i) for i in range(pv.plan_num_work_items(p, 3))]
        assert len(items) >= 8 * len(ctx) and all(0 < int(w[5]) - int(w[4]) <= 8192 * 16 for w in items)


@pytest.mark.parametrize("seed", range(12))
def test_work_items_cover_every_row_and_key_once(seed):
    """Of random batches, short and long, in every kernel's list; parts of a row meet, and the merge knows
    them all."""
    rng = np.random.default_rng(seed)
    heads = [(8, 1, 128), (4, 4, 64), (16, 2, 128), (64, 8, 128)][seed % 4]
    n = int(rng.integers(1, 30))
    ctx = rng.integers(0, [50, 3000, 30000][seed % 3], n)
    new = np.where(rng.random(n) < 0.5, 1, rng.integers(0, 600, n))
    p = pv.plan_create_kv8(pv.pool_desc(70000, heads[1], heads[2], "bf16"), heads[0], ctx, new, 2000)
    group = heads[0] // heads[1]
    rows = {(r, h): [[] for _ in range(int(new[r]) * group)] for r in range(n) for h in range(heads[1])}
    parts = 0
    for kind, most in ((0, 16), (1, 128), (3, 256)):
        for i in range(pv.plan_num_work_items(p, kind)):
            r, h, first, count, lo, hi, at, of = (int(x) for x in pv.plan_work_item(p, kind, i))
            assert 0 < count <= most and (kind != 3 or count == 256)
            assert lo < hi and lo % 32 == 0 and 0 <= at < of and (of > 1 or lo == 0)
            parts += of > 1
            for row in range(first, first + count):
                rows[r, h][row].append((lo, hi))
    merged = sum(int(pv.plan_work_item(p, 2, i)[7]) for i in range(pv.plan_num_work_items(p, 2)))
    assert merged == parts
    for (r, h), each in rows.items():
        for row, spans in enumerate(each):
            spans.sort()
            assert spans and spans[0][0] == 0 and all(a[1] == b[0] for a, b in zip(spans, spans[1:]))
            assert spans[-1][1] >= ctx[r] + row // group + 1  # and sees its own token
