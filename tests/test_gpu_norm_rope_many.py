"""Norms, rotation and append into 16-bit pools over batches of more than 32 MiB of rows, which several
heads a workgroup work on (with head size 128, V in workgroups of its own): every result, and every element
of the pools that no new token belongs to."""
import numpy as np
import pytest

import test_gpu_norm_rope as N
from paper_2312_05516_amd import workloads as wl

pytestmark = pytest.mark.gpu


def _check(b, q, k, v, w, style, in_place=False):
    rows = (b.num_q_heads if q is not None else 0) + 2 * b.num_kv_heads
    assert b.total_q * rows * b.head_dim * 2 > 32 << 20
    assert (b.q_lens > 1).any()  # one token a request: a kernel of its own
    q_out, k_rows, v_rows, pools = N._call16(b, q, k, v, w, style, in_place=in_place)
    if q is not None:
        N._close(q_out, q, w[0], b, style)
    N._close(k_rows, k, w[1], b, style)
    assert np.array_equal(v_rows, v)
    nan = wl.nan_pattern(b.dtype)  # the pools' values before the call; no new row holds it
    for pool in pools:
        assert (pool == nan).sum() == pool.size - b.total_q * b.num_kv_heads * b.head_dim
    return q_out, pools


@pytest.mark.parametrize("style", ["interleaved", "half"])
@pytest.mark.parametrize("heads,dtype,new", [
    ((70, 7, 128), "bf16", (1100, 1, 500, 77)),   # 7 KV heads: no multiple of two or four a workgroup
    ((22, 11, 128), "f16", (2500, 1, 500, 77)),
    ((33, 11, 64), "f16", (3700, 1, 1200, 77)),
])
def test_both_weights_or_one(heads, dtype, new, style):
    b = wl.custom([0, 9, 4, 100], new, num_q_heads=heads[0], num_kv_heads=heads[1], head_dim=heads[2],
                  dtype=dtype, seed=79)
    q, k, v, w = N._inputs(b, 16)
    q_out, pools = _check(b, q, k, v, w, style)
    again = _check(b, q, k, v, w, style, in_place=True)
    assert np.array_equal(again[0], q_out) and all(map(np.array_equal, again[1], pools))
    _check(b, q, k, v, (w[0], None), style)
    _check(b, q, k, v, (None, w[1]), style)


@pytest.mark.parametrize("style", ["interleaved", "half"])
@pytest.mark.parametrize("heads,dtype", [((41, 41, 128), "f16"), ((41, 41, 64), "bf16")])
def test_keys_and_values_alone(heads, dtype, style):
    new = (1100, 1, 500, 77) if heads[2] == 128 else (2200, 1, 1000, 77)
    b = wl.custom([0, 9, 4, 100], new, num_q_heads=heads[0], num_kv_heads=heads[1], head_dim=heads[2],
                  dtype=dtype, seed=80)
    _, k, v, w = N._inputs(b, 18)
    _check(b, None, k, v, (None, w[1]), style)
