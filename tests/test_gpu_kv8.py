"""8-bit pools on the GPU against the definition in 64 bits (kv8_ref): append and reading back bit for
bit, attention within a bound that counts the roundings."""
import numpy as np
import pytest

import helpers as H
import kv8_ref as R
from paper_2312_05516_amd import workloads as wl

pytestmark = pytest.mark.gpu


def _batch(ctx, new, heads=(4, 2, 128), dtype="bf16", seed=5, **kw):
    return wl.custom(ctx, new, num_q_heads=heads[0], num_kv_heads=heads[1], head_dim=heads[2],
                     dtype=dtype, seed=seed, **kw)


def _new_rows(b, seed, std=1.0):
    return [R.random_bits((b.total_q, b.num_kv_heads, b.head_dim), b.dtype, seed + i, std)
            for i in range(2)]


def _check_append(b, before, k, v):
    want = before.copy()
    R.append(want, k, v)
    run, dev = R.Run(b), R.to_dev(before)
    run.append(dev, k, v)
    got = R.from_dev(dev, b)
    got.same_as(want)
    return run, dev, want


# ------------------------------------------------------------------ append
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads", [(4, 2, 128), (3, 3, 64), (7, 1, 64), (8, 8, 128)])
@pytest.mark.parametrize("fill", ["nan", "random"])
def test_append_is_the_definition_bit_for_bit(dtype, heads, fill):
    # begun and half-filled pages, one token to several pages, an empty request, ends inside a page
    b = _batch([0, 3, 16, 31, 250, 9, 12, 0], [1, 1, 16, 33, 6, 0, 4, 70], heads, dtype)
    before = R.Pools(b, fill, seed=3)
    if fill == "nan":  # half-filled pages hold something
        R.append(before, *[R.random_bits((int(b.ctx_lens.sum()), b.num_kv_heads, b.head_dim), dtype,
                                         70 + i) for i in range(2)],
                 np.zeros_like(b.ctx_lens), b.ctx_lens)
    _check_append(b, before, *_new_rows(b, 11))


@pytest.mark.parametrize("dtype,d", [("f16", 64), ("bf16", 128)])
def test_a_history_token_by_token(dtype, d):
    """45 appends of one token, each in a size of its own, so that scales grow inside pages."""
    rng = np.random.default_rng(8)
    b0 = _batch([0], [45], (2, 2, d), dtype)
    want = R.Pools(b0)
    dev = R.to_dev(want)
    k, v = _new_rows(b0, 21)
    size = 2.0 ** rng.integers(-6, 7, (45, 2, 1))
    k, v = (H.f64_to_bits(H.bits_to_f64(x, dtype) * size, dtype) for x in (k, v))
    changes = 0
    for t in range(45):
        before = want.k_scales.copy()
        b = wl.Batch(**{**b0.__dict__, "ctx_lens": np.array([t], np.int32),
                        "q_lens": np.array([1], np.int32)})
        R.append(want, k[t:t + 1], v[t:t + 1], [t], [1])
        changes += t % 16 > 0 and int((before != want.k_scales).any())
        R.Run(b).append(dev, k[t:t + 1], v[t:t + 1])
    R.from_dev(dev, b0).same_as(want)
    assert changes >= 3  # pages whose scale grew with a later token


@pytest.mark.parametrize("heads,dtype", [((40, 40, 128), "f16"), ((11, 11, 64), "bf16"),
                                         ((8, 1, 128), "bf16"), ((35, 35, 64), "f16")])
@pytest.mark.parametrize("std", [1e-2, 1.0, 50.0])
def test_one_token_to_every_request(heads, dtype, std):
    """A batch of generation steps: pages begun, scales kept (1e-2), grown here and there and everywhere."""
    ctx = [0, 1, 5, 15, 16, 31, 47, 100]
    b = _batch(ctx, [1] * len(ctx), heads, dtype)
    before = R.Pools(b)
    R.append(before, *[R.random_bits((int(b.ctx_lens.sum()), heads[1], heads[2]), dtype, 60 + i)
                       for i in range(2)], np.zeros_like(b.ctx_lens), b.ctx_lens)
    k, v = _new_rows(b, 62, std)
    inf = 0x7C00 if dtype == "f16" else 0x7F80
    k[2, 0, 3], v[3, 0, 60], k[4, -1] = inf, inf | 1, 0
    k[6, 0, 9] = v[5, -1, 63] = inf - 1  # the largest finite value
    _check_append(b, before, k, v)


@pytest.mark.parametrize("heads,dtype", [((40, 40, 128), "f16"), ((7, 7, 64), "bf16")])
def test_batches_of_many_rows(heads, dtype):
    """More than 64 MiB of rows: the streaming hint, and several heads a wavefront when read back."""
    new = [2000, 1, 1400, 17] if heads[2] == 128 else [37000, 1, 450, 17]
    b = _batch([0, 9, 4, 100], new, heads, dtype)
    assert b.total_q * heads[1] * heads[2] * 4 > 64 << 20
    k, v = _new_rows(b, 71)
    run, dev = R.Run(b), R.to_dev(R.Pools(b, "random", seed=2))
    run.append(dev, k, v)
    p = R.from_dev(dev, b)
    for got, new_rows in zip(run.read(dev), (k, v)):
        # the rows come back within half a step of a code: 2^-4 of the value, or 2^-10 of the block's scale,
        # which is at most 2^(1 - 448's exponent 8) * its largest value, at most 2^3 here
        x, y = (H.bits_to_f64(t, dtype) for t in (got, new_rows))
        assert (np.abs(x - y) <= np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10 * 2.0 ** -4)).all()
    for r, lo in ((0, 1984), (2, 4), (3, 100)):  # some pages against the definition
        n = min(16, int(b.kv_lens[r]) - lo)
        kk, vv = R.rows(p, r, lo, lo + n)
        at = int(b.q_start[r]) + lo - int(b.ctx_lens[r])
        back = run.read(dev)
        assert np.array_equal(kk, H.bits_to_f64(back[0][at:at + n], dtype))
        assert np.array_equal(vv, H.bits_to_f64(back[1][at:at + n], dtype))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_extreme_values(dtype):
    """Zeros, the type's least and largest values, infinities, NaN, and values next to a scale's end."""
    b = _batch([5, 0, 4], [11, 48, 9], (1, 1, 64), dtype)
    before = R.Pools(b)
    R.append(before, *[R.random_bits((9, 1, 64), dtype, 40 + i, 1e-3) for i in range(2)],
             [0, 0, 0], [5, 0, 4])
    k, v = _new_rows(b, 31)
    inf, one = (0x7C00, 0x3C00) if dtype == "f16" else (0x7F80, 0x3F80)
    for x in (k, v):
        flat = x.reshape(-1, 64)
        flat[0] = 0                                   # begins at slot 5: the scale stays
        flat[2, ::7] = inf - 1                        # the largest finite value: the largest scale
        flat[3, 1::9] = 0x8000 | (inf - 1)
        flat[11:27] &= 0x8000                         # a page of zeros, of either sign
        flat[27:43] &= 0x8007                         # a page of the type's smallest values
        flat[43, 5], flat[44, 6], flat[45, 7] = inf, 0x8000 | inf, inf | 1
        flat[46] = one
        flat[59:] = inf                               # nothing finite
    sevens = H.f64_to_bits(np.array([1.75, 1.75 * (1 + 2.0 ** -7), -1.75]), dtype)
    k.reshape(-1, 64)[47:50, 0] = sevens
    _check_append(b, before, k, v)


def test_a_scale_that_grows_past_everything():
    """Codes under a far larger scale become zero."""
    b = _batch([7], [2], (1, 1, 128), "bf16")
    before = R.Pools(b)
    R.append(before, *[R.random_bits((7, 1, 128), "bf16", 50 + i, 1e-36) for i in range(2)], [0], [7])
    _, _, want = _check_append(b, before, *_new_rows(b, 51, 1e37))
    assert (R.one_nan(want.slots("k", int(b.page_table[0, 0]), 0))[:7] == 0).all()


# ------------------------------------------------------------------ reading back
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads", [(4, 2, 128), (3, 3, 64)])
def test_read_returns_code_times_scale(dtype, heads):
    b = _batch([0, 3, 16, 0, 250, 9], [1, 1, 40, 31, 6, 0], heads, dtype)
    p = R.Pools(b, "random", seed=6)
    lo, hi = R.E_RANGE[dtype]
    p.k_scales[:4] = lo + 127
    run, dev = R.Run(b), R.to_dev(p)
    k, v = (H.bits_to_f64(x, dtype) for x in run.read(dev))
    for r in range(b.num_reqs):
        c, n, s = int(b.ctx_lens[r]), int(b.q_lens[r]), int(b.q_start[r])
        want = R.rows(p, r, c, c + n)
        for got, w in zip((k, v), want):
            assert np.array_equal(got[s:s + n], w, equal_nan=True)
    R.from_dev(dev, b).same_as(p)


def test_what_was_read_back_appends_to_the_same_values():
    b = _batch([0, 0], [77, 5], (2, 2, 128), "bf16")
    k, v = _new_rows(b, 61)
    run, dev = R.Run(b), R.to_dev(R.Pools(b))
    run.append(dev, k, v)
    first = run.read(dev)
    run.append(dev, *first)
    for a, z in zip(first, run.read(dev)):
        assert np.array_equal(a, z)


# ------------------------------------------------------------------ attention
def _check_attention(b, p, q, scale=None, table=None):
    scale = b.scale if scale is None else scale
    got = R.Run(b, table).attend(R.to_dev(p), q, scale)
    want, bound = R.attention(b, H.bits_to_f64(q, b.dtype), p, scale, table)
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (int(bad.sum()), float(np.max(np.abs(got - want) / bound)))
    return got


GROUPS = [((4, 2, 128), "bf16"), ((8, 1, 128), "f16"), ((3, 3, 64), "f16"), ((7, 1, 64), "bf16"),
          ((24, 2, 64), "bf16"), ((40, 2, 128), "f16")]


@pytest.mark.parametrize("heads,dtype", GROUPS)
def test_generation_steps(heads, dtype):
    # the first token of all, ends at every place of a page, of a block of 64 keys, several blocks
    ctx = [0, 1, 14, 15, 16, 62, 63, 64, 127, 255, 256, 300, 511, 700]
    b = _batch(ctx, [1] * len(ctx), heads, dtype)
    _check_attention(b, *R.filled(b, 100))


@pytest.mark.parametrize("heads,dtype", GROUPS)
def test_generation_steps_of_many_requests(heads, dtype):
    """More items than CUs have four wavefronts each, fewer have eight."""
    ctx = [0, 1, 14, 15, 16, 62, 63, 64, 127, 255, 256, 300, 511, 700]
    ctx = ctx * (257 // (len(ctx) * heads[1]) + 1)
    b = _batch(ctx, [1] * len(ctx), heads, dtype)
    run = R.Run(b)
    assert run.pv.plan_kernel_variants(run.plan) == 2
    _check_attention(b, *R.filled(b, 102))


@pytest.mark.parametrize("heads,dtype", GROUPS)
def test_prompts(heads, dtype):
    b = _batch([0, 0, 5, 130, 64, 33, 1], [1, 17, 33, 70, 200, 0, 129], heads, dtype)
    _check_attention(b, *R.filled(b, 110))


@pytest.mark.parametrize("heads,dtype", GROUPS)
def test_prompts_beside_generation_steps(heads, dtype):
    b = _batch([400, 31, 0, 290, 77, 900], [1, 90, 3, 1, 140, 1], heads, dtype)
    _check_attention(b, *R.filled(b, 120))


@pytest.mark.parametrize("new", [1, 5, 60])
@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (64, "f16")])
def test_long_contexts_are_cut_and_merged(new, d, dtype):
    b = _batch([9001, 130], [new, new], (4, 1, d), dtype)
    run = R.Run(b)
    assert run.pv.plan_num_work_items(run.plan, 2) > 0
    _check_attention(b, *R.filled(b, 130))


@pytest.mark.parametrize("ctx,new,heads", [([700] * 200, 1, (8, 1, 128)), ([2500] * 9, 40, (8, 1, 128))])
def test_distance_from_64_bits_of_lists_that_are_hardly_cut(ctx, new, heads):
    """Probabilities are rounded once: to about sqrt(2) times the error of the result's own rounding
    (1.66e-3 in bf16), whatever the number of parts."""
    b = _batch(ctx, [new] * len(ctx), heads, "bf16")
    p, q = R.filled(b, 140)
    got = _check_attention(b, p, q)
    want, _ = R.attention(b, H.bits_to_f64(q, b.dtype), p, b.scale)
    assert np.linalg.norm(got - want) / np.linalg.norm(want) < 1.5 * 1.66e-3


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("ctx,new,heads", [
    ([900, 70, 300], [70, 128, 33], (8, 2, 128)),    # tiles that end at every place of a block, rests
    ([0, 1, 31], [256, 300, 64], (4, 1, 128)),       # first prompts
    ([4097, 15], [256, 257], (2, 2, 128)),
    ([5000, 9000], [64, 1], (8, 1, 128)),            # cut into parts, and a generation step beside
])
def test_long_prompts_in_tiles_of_256_rows(monkeypatch, ctx, new, heads, dtype):
    monkeypatch.setenv("PV_TILE_MIN_KEYS", "64")
    b = _batch(ctx, new, heads, dtype)
    run = R.Run(b)
    assert run.pv.plan_num_work_items(run.plan, 3) > 0
    p, q = R.filled(b, 135)
    for scale in (b.scale, 0.0, -1.2):
        _check_attention(b, p, q, scale=scale)


@pytest.mark.parametrize("scale", [0.0, -0.07, 1.5])
@pytest.mark.parametrize("heads,dtype", [((8, 1, 128), "bf16"), ((3, 3, 64), "f16")])
def test_scales(scale, heads, dtype):
    b = _batch([30, 200, 64], [70, 1, 20], heads, dtype)
    _check_attention(b, *R.filled(b, 150), scale=scale)


def test_scores_of_any_size_and_blocks_of_any_scale():
    """Pages a million times apart in size, in K and in V."""
    b = _batch([300, 90], [1, 50], (4, 2, 128), "bf16")
    lens = b.kv_lens.astype(np.int64)
    rng = np.random.default_rng(3)
    p = R.Pools(b)
    k, v = (H.bits_to_f64(R.random_bits((int(lens.sum()), 2, 128), "bf16", 160 + i), "bf16")
            for i in range(2))
    page = np.concatenate([np.arange(n) // 16 for n in lens])
    size = 2.0 ** rng.integers(-12, 8, (2, 40))
    R.append(p, H.f64_to_bits(k * size[0][page][:, None, None], "bf16"),
             H.f64_to_bits(v * size[1][page][:, None, None], "bf16"), np.zeros_like(lens), lens)
    _check_attention(b, p, R.random_bits((b.total_q, 4, 128), "bf16", 162))


@pytest.mark.parametrize("group,tiles,d", [(1, "0", 128), (1, "0", 64), (4, "0", 128), (16, "0", 64),
                                           (16, "64", 128)])
def test_nan_and_infinity_stay_in_their_rows(monkeypatch, group, tiles, d):
    """A NaN among cached values reaches the rows that see it, and no others; one behind the end of a
    sequence reaches nobody (every unused slot of `filled` is NaN).  In all three kernels."""
    monkeypatch.setenv("PV_TILE_MIN_KEYS", tiles)
    b = _batch([40, 40], [30, 1], (2 * group, 2, d), "f16")
    p, q = R.filled(b, 170)
    page = int(b.page_table[0, 3])  # positions 48..63 of the first request; its rows see 40 + i
    codes = p.slots("v", page, 1)
    codes[2, 17] = 0x7F
    p.put("v", page, 1, codes)
    got = R.Run(b).attend(R.to_dev(p), q)
    nan = np.isnan(got)
    assert nan[10:30, group:, 17].all()
    nan[10:30, group:, 17] = False
    assert not nan.any()
    k = p.slots("k", page, 0)  # and one among the keys, of the other head: the whole rows that see it
    k[9, 5] = 0xFF
    p.put("k", page, 0, k)
    got = R.Run(b).attend(R.to_dev(p), q)
    assert np.isnan(got[17:30, :group]).all() and not np.isnan(got[:17, :group]).any()
    assert not np.isnan(got[30]).any()


@pytest.mark.parametrize("new", [1, 40])
def test_page_order_and_shared_pages_change_nothing(new):
    b = _batch([200, 200, 90], [new, new, new], (8, 2, 128), "bf16")
    p, q = R.filled(b, 180)
    got = R.Run(b).attend(R.to_dev(p), q)
    order = np.random.default_rng(1).permutation(b.num_pages)
    moved = p.copy()
    for src, dst in enumerate(order):
        for h in range(2):
            for which in "kv":
                moved.put(which, dst, h, p.slots(which, src, h))
            for s in ("k_scales", "v_scales"):
                getattr(moved, s)[dst * 2 + h] = getattr(p, s)[src * 2 + h]
    table = np.where(b.page_table >= 0, order[b.page_table], -1)
    assert np.array_equal(got, R.Run(b, table).attend(R.to_dev(moved), q))
    shared = b.page_table.copy()
    shared[1, :12] = shared[0, :12]  # whole pages of the first request's history
    _check_attention(b, p, q, table=shared)


def test_pages_swapped_out_and_in():
    """A block of head size 128 has the bytes of a 16-bit block of head size 64, so the page copy moves 8-bit
    pages under a description of those; scales are a byte for each block beside them."""
    import torch
    b = _batch([200, 90], [1, 40], (8, 2, 128), "bf16")
    p, q = R.filled(b, 190)
    run, dev = R.Run(b), R.to_dev(p)
    want = run.attend(dev, q)
    half = run.pv.pool_desc(b.num_pages, 2, 64, "bf16")
    src = torch.arange(b.num_pages, dtype=torch.int32, device="cuda")
    staging = torch.empty(b.num_pages * 2 * 2 * 2048, dtype=torch.uint8, pin_memory=True)
    run.pv.pages_gather(half, dev.k, dev.v, src, b.num_pages, staging)
    torch.cuda.synchronize()
    order = np.random.default_rng(2).permutation(b.num_pages).astype(np.int32)
    back = R.to_dev(R.Pools(b, "random", seed=13))
    to = torch.from_numpy(order).cuda()
    run.pv.pages_scatter(half, staging, to, b.num_pages, back.k, back.v)
    for n in ("k_scales", "v_scales"):
        getattr(back, n).view(b.num_pages, 2)[to.long()] = getattr(dev, n).view(b.num_pages, 2)
    table = np.where(b.page_table >= 0, order[b.page_table], -1)
    assert np.array_equal(want, R.Run(b, table).attend(back, q))


def test_offsets_past_32_bits():
    """Pools of 4.3 GB: pages whose codes lie behind 2^32."""
    import torch
    from paper_2312_05516_amd import binding as pv
    heads, d, pages = 40, 128, 52600
    b = _batch([40, 100], [3, 20], (heads, heads, d), "bf16", pool_pages=60)
    assert pages * heads * 16 * d > 2 ** 32
    small, q = R.filled(b, 190)
    k, v = _new_rows(b, 191)
    want = small.copy()
    R.append(want, k, v)
    far = pages - b.num_pages
    big = [torch.zeros(pages * heads * 16 * d, dtype=torch.uint8, device="cuda") for _ in "kv"]
    scales = [torch.zeros(pages * heads, dtype=torch.uint8, device="cuda") for _ in "kv"]
    for t, s, src, ssrc in ((big[0], scales[0], small.k, small.k_scales),
                            (big[1], scales[1], small.v, small.v_scales)):
        t[far * heads * 16 * d:] = torch.from_numpy(src).cuda()
        s[far * heads:] = torch.from_numpy(ssrc).cuda()
    dev = pv.Kv8Pool(*big, *scales)
    run = R.Run(b, np.where(b.page_table >= 0, b.page_table + far, -1))
    run.append(dev, k, v)
    tail = R.Pools(b)
    tail.k, tail.v = (t[far * heads * 16 * d:].cpu().numpy() for t in big)
    tail.k_scales, tail.v_scales = (s[far * heads:].cpu().numpy() for s in scales)
    tail.same_as(want)
    for t in big:
        assert not bool(t[:far * heads * 16 * d].any())
    for got, which in zip(run.read(dev), "kv"):
        x = [R.rows(want, r, int(b.ctx_lens[r]), int(b.kv_lens[r]))["kv".index(which)] for r in range(2)]
        assert np.array_equal(H.bits_to_f64(got, "bf16"), np.concatenate(x))
    got = run.attend(dev, q)
    o, bound = R.attention(b, H.bits_to_f64(q, "bf16"), want, b.scale)
    assert (np.abs(got - o) <= bound).all()


# ------------------------------------------------------------------ together, streams, graphs
def test_turns_of_a_conversation():
    """Prompt, a few generated tokens, another prompt: append and attention as a server calls them."""
    heads, dtype = (8, 2, 128), "bf16"
    whole = _batch([0, 0], [260, 40], heads, dtype)
    want = R.Pools(whole)
    dev = R.to_dev(want)
    ctx = np.array([0, 0], np.int32)
    for turn, new in enumerate([(100, 17), (1, 1), (1, 1), (1, 0), (90, 5), (1, 1)]):
        new = np.array(new, np.int32)
        b = wl.Batch(**{**whole.__dict__, "ctx_lens": ctx.copy(), "q_lens": new,
                        "q_start": np.array([0, new[0]], np.int32)})
        k, v = _new_rows(b, 200 + 3 * turn, 1.0 + turn)
        q = R.random_bits((b.total_q, heads[0], heads[2]), dtype, 202 + 3 * turn)
        R.append(want, k, v, b.ctx_lens, b.q_lens)
        run = R.Run(b)
        run.append(dev, k, v)
        got = run.attend(dev, q)
        o, bound = R.attention(b, H.bits_to_f64(q, dtype), want, b.scale)
        assert (np.abs(got - o) <= bound).all()
        R.from_dev(dev, b).same_as(want)
        ctx += new


def test_another_stream_and_timing():
    import torch
    b = _batch([300, 20], [1, 60], (8, 2, 128), "bf16")
    p, q = R.filled(b, 210)
    run, dev = R.Run(b), R.to_dev(p)
    base = run.attend(dev, q)
    run.pv.plan_enable_timing(run.plan)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = run.attend(dev, q)
    assert np.array_equal(got, base)
    assert max(run.pv.plan_kernel_ms(run.plan, k) for k in (0, 1)) > 0


def test_one_plan_on_two_streams_at_once():
    """Two layers at a time: pools, results and workspaces of their own, lists and page table shared."""
    import torch
    b = _batch([7000, 300, 20], [1, 1, 60], (8, 2, 128), "bf16")
    run = R.Run(b)
    layers = [(R.to_dev(p), q) for p, q in (R.filled(b, 212), R.filled(b, 214))]
    want = [run.attend(dev, q) for dev, q in layers]
    assert not np.array_equal(*want)
    streams = [torch.cuda.Stream() for _ in layers]
    args = [(H.to_dev_bits(q, "bf16"), torch.empty_like(run.ws)) for _, q in layers]
    outs = [[torch.empty_like(q) for _ in range(8)] for q, _ in args]
    torch.cuda.synchronize()
    for i in range(8):
        for (dev, _), (q, ws), out, stream in zip(layers, args, outs, streams):
            run.pv.kv8_multi_token_paged_attn_planned(run.plan, q, dev, run.table, b.scale, out[i], ws,
                                                      stream=stream)
    torch.cuda.synchronize()
    for w, out in zip(want, outs):
        for o in out:
            assert np.array_equal(H.bits_to_f64(H.from_dev_bits(o), "bf16"), w)


@pytest.mark.parametrize("ctx,new", [([300, 20], [1, 60]), ([7000], [1])])
def test_captured_and_replayed(ctx, new):
    """Append, attention and reading back in one graph; replays with other rows in the same buffers."""
    import torch
    b = _batch(ctx, new, (8, 2, 128), "bf16")
    p, q0 = R.filled(b, 220)
    run, dev = R.Run(b), R.to_dev(p)
    k0, v0 = _new_rows(b, 221)
    q, k, v = (H.to_dev_bits(x, "bf16") for x in (q0, k0, v0))
    out, kr, vr = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)

    def step():
        run.pv.kv8_append_planned(run.plan, k, v, run.table, dev)
        run.pv.kv8_multi_token_paged_attn_planned(run.plan, q, dev, run.table, b.scale, out, run.ws)
        run.pv.kv8_read_planned(run.plan, dev, run.table, kr, vr)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(4):
        for t, seed in ((q, 230), (k, 240), (v, 250)):
            t.copy_(H.to_dev_bits(R.random_bits(tuple(t.shape), "bf16", seed + turn), "bf16"))
        start = R.from_dev(dev, b)
        out.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (out, kr, vr)]
        after = R.from_dev(dev, b)
        for n in ("k", "v", "k_scales", "v_scales"):
            getattr(dev, n).copy_(torch.from_numpy(getattr(start, n)))
        step()
        torch.cuda.synchronize()
        for a, z in zip(got, (out, kr, vr)):
            assert torch.equal(a, z)
        R.from_dev(dev, b).same_as(after)
