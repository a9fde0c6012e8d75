"""8-bit pools: what lies behind the last token of a page, under the largest scale, and the rotary append
without weights."""
import numpy as np
import pytest

import helpers as H
import kv8_ref as R
import test_gpu_kv8 as T
import test_gpu_norm_rope as N
from paper_2312_05516_amd import workloads as wl

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("code", [0x7E, 0xFE, 0x7F])
@pytest.mark.parametrize("group,tiles,d", [(1, "0", 128), (1, "0", 64), (4, "0", 128), (16, "0", 64),
                                           (16, "64", 128)])
def test_codes_behind_the_last_token_under_the_largest_scale(monkeypatch, group, tiles, d, code):
    """448 * 2^8 is past f16: such codes are infinities where they are widened, and nobody may see them.
    In all three kernels."""
    monkeypatch.setenv("PV_TILE_MIN_KEYS", tiles)
    b = T._batch([40, 37, 0], [30, 1, 19], (2 * group, 2, d), "f16")
    lens = b.kv_lens.astype(np.int64)
    k, v = (H.bits_to_f64(R.random_bits((int(lens.sum()), 2, d), "f16", 230 + i), "f16") for i in range(2))
    v = np.clip(v * 30000, -65504, 65504)
    v[::4, :, 0] = 65504  # some token of every page: the largest scale
    p = R.Pools(b)
    R.append(p, H.f64_to_bits(k, "f16"), H.f64_to_bits(v, "f16"), np.zeros_like(lens), lens)
    used = [int(b.page_table[r, i]) * 2 + h for r in range(3) for i in range((int(lens[r]) + 15) // 16)
            for h in range(2)]
    assert (p.v_scales[used] == 8 + 127).all()
    p.k[p.k == 0x7F] = code  # no token has a NaN: these are the places of none
    p.v[p.v == 0x7F] = code
    T._check_attention(b, p, R.random_bits((b.total_q, 2 * group, d), "f16", 232))


@pytest.mark.parametrize("style", ["interleaved", "half"])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads,ctx,new", [((6, 3, 128), (37, 0, 250, 8), (5, 33, 1, 0)),
                                           ((9, 3, 64), (3, 15, 16, 700), (1, 1, 1, 1)),
                                           ((70, 7, 128), (0, 9), (1700, 1))])
def test_without_weights_the_norms_call_is_the_rotary_append(heads, dtype, style, ctx, new):
    import torch
    from paper_2312_05516_amd import binding as pv
    b = wl.custom(ctx, new, num_q_heads=heads[0], num_kv_heads=heads[1], head_dim=heads[2], dtype=dtype,
                  seed=81)
    q, k, v, _ = N._inputs(b, 20)
    got = N._call16(b, q, k, v, (None, None), style)
    plan = pv.plan_create(pv.pool_desc(b.num_pages, b.num_kv_heads, b.head_dim, dtype), b.num_q_heads,
                          b.ctx_lens, b.q_lens, b.max_pages_per_req)
    pv.plan_upload(plan)
    q, k, v = (H.to_dev_bits(x, dtype) for x in (q, k, v))
    kp, vp = (torch.full((wl.pool_elems(b),), float("nan"), dtype=H._torch_dtype(dtype), device="cuda")
              for _ in "kv")
    out = torch.empty_like(q)
    pv.rope_kv_append_planned(plan, q, out, k, v, torch.from_numpy(N._table(b)).cuda(), style,
                              torch.from_numpy(b.page_table).cuda(), kp, vp)
    assert np.array_equal(H.from_dev_bits(out), got[0])
    assert np.array_equal(H.from_dev_bits(kp), got[3][0]) and np.array_equal(H.from_dev_bits(vp), got[3][1])
