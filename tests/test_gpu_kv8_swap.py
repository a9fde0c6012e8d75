"""Pages of 8-bit pools through the page copy, under the description of a 16-bit pool whose pages have the
same bytes: half the head size, or half the heads."""
import numpy as np
import pytest

import kv8_ref as R
from paper_2312_05516_amd import binding as pv
from paper_2312_05516_amd import workloads as wl


def _same_bytes(pages, kv_heads, head_dim, dtype):
    return (pv.pool_desc(pages, kv_heads, 64, dtype) if head_dim == 128
            else pv.pool_desc(pages, kv_heads // 2, 64, dtype))


@pytest.mark.parametrize("kv_heads,head_dim", [(5, 128), (8, 128), (6, 64), (2, 64)])
def test_descriptions_have_the_same_bytes(kv_heads, head_dim):
    desc = pv.pool_desc(7, kv_heads, head_dim, "bf16")
    assert pv.pool_bytes(_same_bytes(7, kv_heads, head_dim, "bf16")) == pv.kv8_pool_bytes(desc)


@pytest.mark.gpu
@pytest.mark.parametrize("heads,dtype", [((5, 5, 128), "bf16"), ((6, 6, 64), "f16"), ((8, 2, 64), "bf16")])
def test_some_pages_swapped_out_and_into_others(heads, dtype):
    import torch
    hq, h, d = heads
    b = wl.custom([200, 90, 5], [1, 40, 3], num_q_heads=hq, num_kv_heads=h, head_dim=d, dtype=dtype, seed=6)
    p, q = R.filled(b, 195)
    run, dev = R.Run(b), R.to_dev(p)
    want = run.attend(dev, q)
    desc = _same_bytes(b.num_pages, h, d, dtype)
    used = np.unique(b.page_table[b.page_table >= 0]).astype(np.int32)
    free = np.random.default_rng(4).permutation(b.num_pages).astype(np.int32)[:len(used)]
    src, to = (torch.from_numpy(x).cuda() for x in (used, free))
    staging = torch.empty(len(used) * h * 2 * 16 * d, dtype=torch.uint8, pin_memory=True)
    pv.pages_gather(desc, dev.k, dev.v, src, len(used), staging)
    torch.cuda.synchronize()
    before = R.Pools(b, "random", seed=14)
    back = R.to_dev(before)
    pv.pages_scatter(desc, staging, to, len(used), back.k, back.v)
    for n in ("k_scales", "v_scales"):
        getattr(back, n).view(-1, h)[to.long()] = getattr(dev, n).view(-1, h)[src.long()]
    moved = np.full(b.num_pages, -1, np.int32)
    moved[used] = free
    assert np.array_equal(want, R.Run(b, np.where(b.page_table >= 0, moved[b.page_table], -1)).attend(back, q))
    expect = before  # pages that nothing was swapped into keep their bytes
    for a, z in zip(used, free):
        for i in range(h):
            for which in "kv":
                expect.put(which, int(z), i, p.slots(which, int(a), i))
            for n in ("k_scales", "v_scales"):
                getattr(expect, n)[z * h + i] = getattr(p, n)[a * h + i]
    R.from_dev(back, b).same_as(expect)
