"""8-bit appends of more than 64 MiB of rows, whose loads have the streaming hint, bit for bit: codes and
scales of every page, those that no new token belongs to among them."""
import numpy as np
import pytest

import helpers as H
import kv8_ref as R
import test_gpu_kv8 as T

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,dtype,new", [((40, 40, 128), "f16", (2000, 1, 1400, 17)),
                                             ((10, 10, 128), "bf16", (9000, 1, 4300, 17)),
                                             ((7, 7, 64), "bf16", (37000, 1, 450, 17))])
def test_append_of_many_rows_is_the_definition(heads, dtype, new):
    b = T._batch([0, 9, 4, 100], new, heads, dtype, pool_pages=2600)
    assert b.total_q * heads[1] * heads[2] * 4 > 64 << 20
    used = {int(p) for r in range(4) for p in b.page_table[r, :(int(b.kv_lens[r]) + 15) // 16]}
    assert len(used) < b.num_pages
    before = R.Pools(b, "random", seed=2)
    k, v = T._new_rows(b, 73)
    # the partly filled pages begin with rows of three sizes: one keeps the page's scale, two make it grow
    for x in (k, v):
        for r, size in ((1, 2.0 ** -5), (2, 2.0 ** 6), (3, 1.0)):
            at = int(b.q_start[r])
            first = slice(at, at + min(12, int(b.q_lens[r])))
            x[first] = H.f64_to_bits(H.bits_to_f64(x[first], dtype) * size, dtype)
    run, dev, want = T._check_append(b, before, k, v)
    grown = [r for r in (1, 2, 3) if (want.k_scales != before.k_scales)[
        [int(b.page_table[r, int(b.ctx_lens[r]) // 16]) * heads[1] + h for h in range(heads[1])]].any()]
    assert 2 in grown and 3 in grown
    for r in (0, 2):  # and reading them back
        c, n, at = int(b.ctx_lens[r]), int(b.q_lens[r]), int(b.q_start[r])
        for got, x in zip(run.read(dev), R.rows(want, r, c, c + n)):
            assert np.array_equal(H.bits_to_f64(got[at:at + n], dtype), x, equal_nan=True)
