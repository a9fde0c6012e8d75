"""Plain numpy definition, in 64 bits, of what the 8-bit pool calls and the query/key norms compute, and
the GPU plumbing of their tests.  Written from the header's text; it calls nothing of the library."""
from __future__ import annotations

import numpy as np

import helpers as H
from paper_2312_05516_amd import workloads as wl

E_RANGE = {"f16": (-15, 8), "bf16": (-117, 120)}
HALF_STEP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}  # of a rounding, relative to the value

_c = np.arange(127)
VALUES = np.where(_c >= 8, (1 + _c % 8 / 8) * 2.0 ** (_c // 8 - 7), _c % 8 / 8 * 2.0 ** -6)
_ALL = np.concatenate([VALUES, [np.nan], -VALUES, [np.nan]])
_MID = (VALUES[1:] + VALUES[:-1]) / 2


def decode(codes: np.ndarray) -> np.ndarray:
    return _ALL[codes]


def encode(x: np.ndarray, most: float = 448.0) -> np.ndarray:
    """Nearest code, ties to even; what is not finite becomes NaN (0x7F)."""
    a = np.minimum(np.abs(np.nan_to_num(x, nan=0.0, posinf=0.0, neginf=0.0)), most)
    i = np.searchsorted(_MID, a)
    tie = (i < 126) & (a == _MID[np.minimum(i, 125)]) & (i % 2 == 1)
    code = (i + tie) | np.where(np.signbit(x), 0x80, 0)
    return np.where(np.isfinite(x), code, 0x7F).astype(np.uint8)


def one_nan(codes: np.ndarray) -> np.ndarray:
    """Both codes of NaN as one, and both of zero: the sign of either means nothing."""
    c = np.where(codes == 0xFF, 0x7F, codes)
    return np.where(c == 0x80, 0, c)


def needed(amax: float, dtype: str) -> int:
    lo, hi = E_RANGE[dtype]
    for e in range(lo, hi + 1):
        if amax <= 448.0 * 2.0 ** e:
            return e
    raise AssertionError("a value past the 16-bit type")


class Pools:
    """k, v: flat codes; k_scales, v_scales: [pages * heads] bytes."""

    def __init__(self, b: wl.Batch, fill="nan", seed=0):
        rng = np.random.default_rng(seed)
        n, t = wl.pool_elems(b), b.num_pages * b.num_kv_heads
        self.b = b
        if fill == "nan":
            self.k, self.v = (np.full(n, 0x7F, np.uint8) for _ in "kv")
            self.k_scales, self.v_scales = (np.full(t, 255, np.uint8) for _ in "kv")
        else:
            self.k, self.v = (rng.integers(0, 256, n).astype(np.uint8) for _ in "kv")
            lo, hi = E_RANGE[b.dtype]
            self.k_scales, self.v_scales = (
                rng.integers(max(lo, -9), min(hi, -5), t).astype(np.int64).astype(np.int16)
                .__add__(127).astype(np.uint8) for _ in "kv")

    def copy(self):
        c = Pools.__new__(Pools)
        c.b = self.b
        for n in ("k", "v", "k_scales", "v_scales"):
            setattr(c, n, getattr(self, n).copy())
        return c

    def k_block(self, page, head):
        """View of a block as [slot / 4, dim / 16, slot % 4, dim % 16]."""
        b = self.b
        at = (page * b.num_kv_heads + head) * 16 * b.head_dim
        return self.k[at:at + 16 * b.head_dim].reshape(4, b.head_dim // 16, 4, 16)

    def v_block(self, page, head):
        b = self.b
        at = (page * b.num_kv_heads + head) * 16 * b.head_dim
        return self.v[at:at + 16 * b.head_dim].reshape(b.head_dim, 16)

    def slots(self, which, page, head):
        """Codes of a block as [slot, dim] (a copy)."""
        if which == "k":
            return self.k_block(page, head).transpose(0, 2, 1, 3).reshape(16, -1).copy()
        return self.v_block(page, head).T.copy()

    def put(self, which, page, head, codes):
        d = self.b.head_dim
        if which == "k":
            self.k_block(page, head)[:] = codes.reshape(4, 4, d // 16, 16).transpose(0, 2, 1, 3)
        else:
            self.v_block(page, head)[:] = codes.T

    def same_as(self, other):
        for n in ("k", "v"):
            assert np.array_equal(one_nan(getattr(self, n)), one_nan(getattr(other, n))), n
        assert np.array_equal(self.k_scales, other.k_scales)
        assert np.array_equal(self.v_scales, other.v_scales)


def append(p: Pools, k_new: np.ndarray, v_new: np.ndarray, ctx=None, qn=None, table=None):
    """k_new, v_new: bit patterns [N, Hkv, D].  Changes p."""
    b = p.b
    ctx = b.ctx_lens if ctx is None else ctx
    qn = b.q_lens if qn is None else qn
    table = b.page_table if table is None else table
    top = E_RANGE[b.dtype][1]
    row = 0
    for r in range(len(ctx)):
        t, end = int(ctx[r]), int(ctx[r]) + int(qn[r])
        while t < end:
            stop = min(end, (t // 16 + 1) * 16)
            page, s0 = int(table[r, t // 16]), t % 16
            for h in range(b.num_kv_heads):
                for which, new, scales in (("k", k_new, p.k_scales), ("v", v_new, p.v_scales)):
                    x = H.bits_to_f64(new[row:row + stop - t, h], b.dtype)
                    at = page * b.num_kv_heads + h
                    e = needed(np.abs(x[np.isfinite(x)]).max(initial=0.0), b.dtype)
                    codes = p.slots(which, page, h)
                    if s0 > 0:
                        old = int(scales[at]) - 127
                        if e > old:
                            codes[:s0] = encode(decode(codes[:s0]) * 2.0 ** (old - e))
                        e = max(e, old)
                    with np.errstate(invalid="ignore"):
                        codes[s0:s0 + stop - t] = encode(x * 2.0 ** -e, 240.0 if e == top else 448.0)
                    p.put(which, page, h, codes)
                    scales[at] = e + 127
            row += stop - t
            t = stop
    assert row == k_new.shape[0]


def rows(p: Pools, r: int, lo: int, hi: int, table=None):
    """Values of positions lo..hi-1 of request r: (K, V) [hi - lo, Hkv, D] float64."""
    b = p.b
    table = b.page_table if table is None else table
    k, v = (np.zeros((hi - lo, b.num_kv_heads, b.head_dim)) for _ in "kv")
    for h in range(b.num_kv_heads):
        for lp in range(lo // 16, (hi + 15) // 16):
            page = int(table[r, lp])
            at = page * b.num_kv_heads + h
            a, z = max(lo, lp * 16), min(hi, lp * 16 + 16)
            for which, out, s in (("k", k, p.k_scales), ("v", v, p.v_scales)):
                out[a - lo:z - lo, h] = (decode(p.slots(which, page, h))[a % 16:a % 16 + z - a]
                                         * 2.0 ** (int(s[at]) - 127))
    return k, v


def attention(b: wl.Batch, q: np.ndarray, p: Pools, scale: float, table=None):
    """(result [N, Hq, D], bound on the error of a right kernel) in float64; q: float64 values.

    Bound, u the half step of the 16-bit type, w = sum_t P_t |V_t|: the result is rounded once (u * |o|),
    the probabilities are rounded once, in the sum over V and in their own (2 * u * w); scores are sums
    of D products in fp32 (D * 2^-24 * sum |q k| each at the most), which moves a probability by twice
    that, relative; 2^-16 * w covers exponentials, sums over keys and the final division in fp32."""
    G = b.num_q_heads // b.num_kv_heads
    u = HALF_STEP[b.dtype]
    out = np.zeros((b.total_q, b.num_q_heads, b.head_dim))
    bound = np.zeros_like(out)
    for r in range(b.num_reqs):
        c, n, s0 = int(b.ctx_lens[r]), int(b.q_lens[r]), int(b.q_start[r])
        if n == 0:
            continue
        K, V = rows(p, r, 0, c + n, table)
        seen = np.arange(c + n)[None] <= c + np.arange(n)[:, None]
        for hq in range(b.num_q_heads):
            Q, Kh, Vh = q[s0:s0 + n, hq], K[:, hq // G], V[:, hq // G]
            s = np.where(seen, (Q @ Kh.T) * scale, -np.inf)
            size = (np.where(seen, (np.abs(Q) @ np.abs(Kh).T), 0.0) * abs(scale)).max(axis=1)
            P = np.exp(s - s.max(axis=1, keepdims=True))
            P /= P.sum(axis=1, keepdims=True)
            o, w = P @ Vh, P @ np.abs(Vh)
            out[s0:s0 + n, hq] = o
            bound[s0:s0 + n, hq] = u * (np.abs(o) + 2 * w) + w * (
                2.0 ** -16 + 2 * b.head_dim * 2.0 ** -24 * size[:, None])
    return out, bound


def norm_rotate(x: np.ndarray, weight, eps: float, table: np.ndarray, pos: np.ndarray, style: str):
    """x: float64 [N, heads, D]; weight: float64 [D] or None; table: float32 [max_pos, D]."""
    d = x.shape[2]
    if weight is not None:
        x = x * weight / np.sqrt((x * x).mean(axis=2, keepdims=True) + eps)
    c, s = (table[pos].astype(np.float64)[:, None, i:i + d // 2] for i in (0, d // 2))
    y = np.empty_like(x)
    a, b = ((slice(0, d // 2), slice(d // 2, d)) if style == "half"
            else (slice(0, d, 2), slice(1, d, 2)))
    y[:, :, a] = x[:, :, a] * c - x[:, :, b] * s
    y[:, :, b] = x[:, :, b] * c + x[:, :, a] * s
    return y


def positions(b: wl.Batch) -> np.ndarray:
    return np.concatenate([np.arange(c, c + n) for c, n in zip(b.ctx_lens, b.q_lens)]).astype(np.int64)


# ---------------------------------------------------------------------------------------------
def to_dev(p: Pools):
    """(Kv8Pool, the four device tensors)"""
    import torch
    from paper_2312_05516_amd import binding as pv
    t = [torch.from_numpy(a).cuda() for a in (p.k, p.v, p.k_scales, p.v_scales)]
    return pv.Kv8Pool(*t)


def from_dev(dev, b) -> Pools:
    p = Pools.__new__(Pools)
    p.b = b
    for n in ("k", "v", "k_scales", "v_scales"):
        setattr(p, n, getattr(dev, n).cpu().numpy().copy())
    return p


class Run:
    """A batch on the device: plan for 8-bit pools, page table, workspace."""

    def __init__(self, b: wl.Batch, table=None):
        import torch
        from paper_2312_05516_amd import binding as pv
        self.b, self.pv = b, pv
        self.desc = pv.pool_desc(b.num_pages, b.num_kv_heads, b.head_dim, b.dtype)
        self.plan = pv.plan_create_kv8(self.desc, b.num_q_heads, b.ctx_lens, b.q_lens,
                                       b.max_pages_per_req)
        lists = torch.empty(pv.plan_device_bytes(self.plan), dtype=torch.uint8, device="cuda")
        pv.plan_upload_to(self.plan, lists)
        self.lists = lists
        t = b.page_table if table is None else table
        self.table = torch.from_numpy(np.ascontiguousarray(t, dtype=np.int32)).cuda()
        self.ws = torch.empty(max(pv.plan_workspace_bytes(self.plan), 256), dtype=torch.uint8,
                              device="cuda")

    def append(self, dev, k_new, v_new):
        k, v = H.to_dev_bits(k_new, self.b.dtype), H.to_dev_bits(v_new, self.b.dtype)
        self.pv.kv8_append_planned(self.plan, k, v, self.table, dev)

    def read(self, dev):
        import torch
        b = self.b
        k, v = (torch.full((b.total_q + 2, b.num_kv_heads, b.head_dim), 7.0,
                           dtype=H._torch_dtype(b.dtype), device="cuda") for _ in "kv")
        self.pv.kv8_read_planned(self.plan, dev, self.table, k, v)
        assert bool((k[b.total_q:] == 7.0).all()) and bool((v[b.total_q:] == 7.0).all())
        return H.from_dev_bits(k[:b.total_q]), H.from_dev_bits(v[:b.total_q])

    def attend(self, dev, q_bits, scale=None):
        """Result as float64 [N, Hq, D]; rows behind the last one must stay as they were."""
        import torch
        b = self.b
        q = H.to_dev_bits(q_bits, b.dtype)
        out = torch.full((b.total_q + 2, b.num_q_heads, b.head_dim), 7.0,
                         dtype=H._torch_dtype(b.dtype), device="cuda")
        self.pv.kv8_multi_token_paged_attn_planned(self.plan, q, dev, self.table,
                                                   b.scale if scale is None else scale, out, self.ws)
        assert bool((out[b.total_q:] == 7.0).all())
        return H.bits_to_f64(H.from_dev_bits(out[:b.total_q]), b.dtype)


def random_bits(shape, dtype, seed, std=1.0):
    return wl.as_u16(wl.random_values(shape, dtype, seed, std))


def filled(b: wl.Batch, seed: int, std=None):
    """Pools that hold every request's cached and new tokens (appended whole by the definition; all else
    NaN), heads of different sizes, and the queries."""
    p = Pools(b)
    lens = b.kv_lens.astype(np.int64)
    std = 2.0 ** np.linspace(-1, 1, b.num_kv_heads) if std is None else std
    k, v = (H.f64_to_bits(H.bits_to_f64(random_bits((int(lens.sum()), b.num_kv_heads, b.head_dim),
                                                    b.dtype, seed + i), b.dtype)
                          * np.reshape(std, (1, -1, 1)), b.dtype) for i in range(2))
    append(p, k, v, np.zeros_like(lens), lens)
    return p, random_bits((b.total_q, b.num_q_heads, b.head_dim), b.dtype, seed + 2)
