"""The arrays of an 8-bit pool in the binding: every call takes the addresses that they have then."""
import pytest
import torch

from paper_2312_05516_amd import binding as pv

PLAN = 4096  # no plan: the library's entry points are replaced by one that keeps what it is given


class _Plan:
    handle = PLAN


def _calls(monkeypatch):
    """The four calls that take a pool, each returning the addresses it hands to the library."""
    t = torch.zeros(4)
    cs = torch.zeros(4, 4)
    got = []

    def keep(name):
        def entry(*args):
            at = [a._obj for a in args if isinstance(getattr(a, "_obj", None), pv._Kv8Ptrs)]
            assert len(at) == 1
            got.append((name, at[0].k, at[0].v, at[0].k_scales, at[0].v_scales))
            return 0
        return entry

    for n in ("pv_kv8_append_planned", "pv_kv8_read_planned", "pv_kv8_norm_rope_append_planned",
              "pv_kv8_multi_token_paged_attn_planned"):
        monkeypatch.setattr(pv._lib, n, keep(n))

    def run(pool):
        got.clear()
        pv.kv8_append_planned(_Plan, t, t, t, pool, stream=1)
        pv.kv8_read_planned(_Plan, pool, t, t, t, stream=1)
        pv.kv8_norm_rope_append_planned(_Plan, t, t, t, t, t, t, 1e-6, cs, "half", t, pool, stream=1)
        pv.kv8_multi_token_paged_attn_planned(_Plan, t, pool, t, 0.1, t, None, stream=1)
        assert len({g[0] for g in got}) == 4
        assert len({g[1:] for g in got}) == 1
        return got[0][1:]

    return run


@pytest.mark.parametrize("name", ["k", "v", "k_scales", "v_scales"])
def test_addresses_are_those_of_the_call(monkeypatch, name):
    run = _calls(monkeypatch)
    arrays = {n: torch.zeros(64, dtype=torch.uint8) for n in ("k", "v", "k_scales", "v_scales")}
    pool = pv.Kv8Pool(**arrays)

    def now():
        return tuple(getattr(pool, n).data_ptr() for n in arrays)

    first = run(pool)
    assert first == now()
    getattr(pool, name).set_(torch.zeros(128, dtype=torch.uint8))  # another storage, the old one freed
    assert run(pool) == now() != first
    second = now()
    setattr(pool, name, torch.zeros(256, dtype=torch.uint8))       # another tensor
    assert run(pool) == now() != second
    setattr(pool, name, torch.zeros(8, 2, dtype=torch.uint8)[:, 0])
    with pytest.raises(ValueError):
        run(pool)


def test_strided_views_of_the_same_address_are_refused(monkeypatch):
    run = _calls(monkeypatch)
    arrays = {n: torch.zeros(64, dtype=torch.uint8) for n in ("k", "v", "k_scales", "v_scales")}
    pool = pv.Kv8Pool(**arrays)
    run(pool)
    pool.v = arrays["v"][::2]
    with pytest.raises(ValueError):
        run(pool)
    pool.v = arrays["v"]
    assert run(pool) == tuple(a.data_ptr() for a in arrays.values())


def test_addresses_as_numbers_and_arrays(monkeypatch):
    import numpy as np
    run = _calls(monkeypatch)
    n = np.zeros(64, np.uint8)
    pool = pv.Kv8Pool(4096, n, 8192, torch.zeros(4))
    assert run(pool) == (4096, n.ctypes.data, 8192, pool.v_scales.data_ptr())
    pool.k = 12288
    assert run(pool)[0] == 12288
    with pytest.raises(TypeError):
        pv.Kv8Pool("k", n, n, n)
