"""Performance cases of the operators around the 8-bit KV cache and of the query/key norms.

The operators, each a call of a serving program on one batch:

* ``attend``  multi-token paged attention over K/V pools of 8-bit codes;
* ``append``  new K/V rows are quantised into those pools;
* ``read``    K/V rows of the requests are read back from them as 16-bit values;
* ``norm``    queries and keys are normalised per head and rotated, keys and values stored, in
              the 16-bit pools or (``into8``) in the 8-bit pools.

The 8-bit pools.  A code is an e4m3 value (sign, 4 exponent bits, 3 of mantissa, no infinity); a
block is one page (16 tokens) of one KV head, K and V apart, with a scale 2^e held as the byte e + 127.

    K(page p, head h, slot s, dim d) at byte (p*Hkv+h)*16*D + (s/4)*4*D + (d/16)*64 + (s%4)*16 + d%16
    V(page p, head h, slot s, dim d) at byte (p*Hkv+h)*16*D + d*16 + s

New rows in slots s0.. of a page set e = max(the least e with max |x| <= 448 * 2^e, the page's e if
s0 > 0); where that is more than the page's e, the codes in front of s0 are rounded anew.

Lengths come from the case alone (``lens``), values and page numbers from the seed of ``prepare``.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

PAGE = 16
EPS = 1e-6
# exponents of a scale: every code * 2^e is a value of the 16-bit type
E_RANGE = {"f16": (-15, 8), "bf16": (-117, 120)}

MHA = (40, 40, 128)    # 13B-shaped layer
GQA = (64, 8, 128)     # 70B-shaped layer
GQA_D64 = (32, 8, 64)  # the other head size the library has


def _case(name, op, heads, dtype, requests, ctx, new, *, single=0.0, lens=1, style="", into8=False):
    """ctx, new = (fewest, most) cached and new tokens of a request; `single` = share of the requests
    that bring one token whatever `new` says."""
    c = {"op": op, "dtype": dtype, "q_heads": heads[0], "kv_heads": heads[1], "head_dim": heads[2],
         "requests": requests, "ctx_lo": ctx[0], "ctx_hi": ctx[1], "new_lo": new[0], "new_hi": new[1],
         "single": single, "lens": lens}
    if name:
        c["name"] = name
    if op == "norm":
        c |= {"style": style, "into8": into8}
    return c


def listed():
    return [
        # one user alone generates a token over a short chat: the smallest call, launches count
        _case("one_step", "attend", GQA_D64, "f16", 1, (700, 700), (1, 1)),
        # an ordinary generation batch, grouped heads
        _case("steps_gqa", "attend", GQA, "bf16", 64, (100, 6000), (1, 1)),
        # a large generation batch, every query head with K/V of its own (2.4 GB of codes)
        _case("steps_mha", "attend", MHA, "f16", 96, (500, 4000), (1, 1)),
        # new turns beside generation steps
        _case("mixed_gqa", "attend", GQA, "bf16", 48, (16, 2500), (16, 250), single=0.6),
        # prompts over long histories, bound by the matrix cores: the most arithmetic
        _case("long_history", "attend", GQA, "bf16", 4, (19000, 25000), (512, 512)),
        # a token for each of 256 running requests goes into its page, mostly mid-page
        _case("append_steps", "append", GQA, "bf16", 256, (1, 200), (1, 1)),
        # first prompts of a 40-head model are stored
        _case("append_prompts", "append", MHA, "f16", 8, (0, 40), (300, 1500)),
        # one short chat is read back
        _case("read_chat", "read", GQA, "bf16", 1, (0, 0), (611, 611)),
        # long histories are read back
        _case("read_histories", "read", GQA, "bf16", 8, (0, 0), (2000, 16000)),
        # generation steps of a model with normalised queries and keys, 16-bit pools
        _case("norm_steps", "norm", GQA, "bf16", 64, (20, 4000), (1, 1), style="half"),
        # its prompts, 16-bit pools
        _case("norm_prompts", "norm", MHA, "f16", 6, (0, 700), (200, 1200), style="interleaved"),
        # its prompts into the 8-bit pools (and read back, as the next layer of a tier does)
        _case("norm_into8", "norm", GQA, "bf16", 8, (0, 700), (100, 1000), style="half", into8=True),
    ]


# A drawn case stays below these: bytes and operations of the largest listed ones, and the values
# that the plain form of attention holds at once
_MOST_BYTES, _MOST_FLOPS = 2.2e9, 1.4e12
_MOST_KEYS, _MOST_SCORES = 2.2e9, 3.3e9


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        op = rng.choice(["attend", "attend", "attend", "append", "read", "norm"])
        heads = rng.choice([MHA, GQA, GQA, GQA_D64, (40, 10, 128), (16, 2, 128), (10, 10, 128),
                            (12, 12, 64), (7, 1, 64)])
        dtype = rng.choice(["f16", "bf16"])
        requests = log_int(1, 256)
        steps = rng.random() < 0.4
        ctx_lo = log_int(1, 20000 if op == "attend" else 2000) - 1
        new_lo = 1 if steps else log_int(1, 600)
        if op == "read":
            ctx_lo, new_lo = rng.choice([0, ctx_lo]), log_int(1, 16000)
        ctx = (ctx_lo, ctx_lo + log_int(1, 4000) - 1)
        new = (new_lo, new_lo if steps else new_lo + log_int(1, 900) - 1)
        case = _case("", op, heads, dtype, requests, ctx, new, lens=rng.randrange(1 << 20),
                     single=0.0 if steps or rng.random() < 0.5 else round(rng.random(), 2),
                     style=rng.choice(["half", "interleaved"]), into8=rng.random() < 0.5)
        w = work(case)
        if w["bytes"] / _MOST_BYTES + w["flops"] / _MOST_FLOPS > 1.0:
            continue
        cached, fresh = _lengths(case)
        longest = max(c + n for c, n in zip(cached, fresh))
        if op == "attend" and (
                requests * longest * heads[1] * heads[2] > _MOST_KEYS
                or requests * longest * heads[0] * max(fresh) > _MOST_SCORES):
            continue
        if requests * longest * heads[1] * heads[2] > 2 * _MOST_KEYS:
            continue
        return case


def _lengths(case):
    """Cached and new tokens of every request."""
    rng = random.Random(case["lens"])
    n = case["requests"]
    ctx = [rng.randint(case["ctx_lo"], case["ctx_hi"]) for _ in range(n)]
    new = [rng.randint(case["new_lo"], case["new_hi"]) for _ in range(n)]
    ones = set(rng.sample(range(n), min(n - 1, round(case["single"] * n))))
    return ctx, [1 if r in ones else new[r] for r in range(n)]


def work(case):
    ctx, new = _lengths(case)
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    total = sum(new)
    pages = sum((c + n + PAGE - 1) // PAGE for c, n in zip(ctx, new))
    touched = sum((c + n + PAGE - 1) // PAGE - c // PAGE for c, n in zip(ctx, new))
    if case["op"] == "attend":
        pairs = sum(n * c + n * (n + 1) // 2 for c, n in zip(ctx, new))
        return {"bytes": 2 * (sum(ctx) + total) * hkv * d + 2 * pages * hkv + 4 * pages
                + 2 * total * hq * d * 2, "flops": 4 * d * hq * pairs}
    rows16, rows8 = 2 * total * hkv * d * 2, 2 * total * hkv * d + 2 * touched * hkv
    if case["op"] != "norm":
        return {"bytes": rows16 + rows8 + 4 * touched, "flops": 0}
    nbytes = 2 * total * hq * d * 2 + rows16 + 4 * total * d + 4 * touched
    # into the 8-bit pools: the codes are written, and read back into rows
    return {"bytes": nbytes + (2 * rows8 + rows16 if case["into8"] else rows16), "flops": 0}


def _type(case):
    return torch.float16 if case["dtype"] == "f16" else torch.bfloat16


def _normal(shape, dtype, gen, std=1.0):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=gen)


def _head_std(n):
    """Heads differ in size: from a half to two."""
    return torch.exp2(torch.linspace(-1.0, 1.0, n, device="cuda"))[:, None]


def _power(e):
    """2^e as float32, for whole numbers -126 <= e <= 127."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _need(amax, dtype):
    """Least exponent e in the type's range with amax <= 448 * 2^e."""
    lo, hi = E_RANGE[dtype]
    m, x = torch.frexp(amax)
    e = torch.where(m <= 0.875, x - 9, x - 8)
    return torch.where(amax > 0, e, lo).clamp(lo, hi)


def _encode(x, e, dtype):
    """Codes (uint8) of the float32 values x under scales 2^e (broadcast)."""
    most = torch.where(e == E_RANGE[dtype][1], 240.0, 448.0)
    y = x * _power(-e)
    y = torch.where(torch.isfinite(y), torch.minimum(torch.maximum(y, -most), most),
                    torch.full_like(y, math.nan))
    return y.to(torch.float8_e4m3fn).view(torch.uint8)


def _decode(codes):
    return codes.view(torch.float8_e4m3fn).to(torch.float32)


def _k8(st):
    """The K pool as [page, head, slot / 4, dim / 16, slot % 4, dim % 16]; V as [page, head, dim, slot]."""
    p, h, d = st["pages"], st["case"]["kv_heads"], st["case"]["head_dim"]
    return st["k8"].view(p, h, 4, d // 16, 4, 16)


def _v8(st):
    return st["v8"].view(st["pages"], st["case"]["kv_heads"], st["case"]["head_dim"], PAGE)


def _fill8(st, gen):
    """Pools whose every page holds values of the heads' sizes, quantised page by page."""
    case, pages = st["case"], st["pages"]
    h, d = case["kv_heads"], case["head_dim"]
    n = pages * h * PAGE * d
    std = _head_std(h)[:, :, None]
    step = max(1, (1 << 28) // (h * PAGE * d))
    for name in ("k", "v"):
        codes = torch.empty(n, dtype=torch.uint8, device="cuda")
        scales = torch.empty(pages * h, dtype=torch.uint8, device="cuda")
        st[name + "8"], st[name + "_scales"] = codes, scales
        view = _k8(st) if name == "k" else _v8(st)
        for p in range(0, pages, step):
            m = min(step, pages - p)
            x = _normal((m, h, PAGE, d), torch.float32, gen).mul_(std).to(_type(case)).float()
            e = _need(x.abs().amax((2, 3)), case["dtype"])
            scales.view(pages, h)[p:p + m] = (e + 127).to(torch.uint8)
            c = _encode(x, e[:, :, None, None], case["dtype"])
            if name == "k":
                view[p:p + m] = c.view(m, h, 4, 4, d // 16, 16).transpose(3, 4)
            else:
                view[p:p + m] = c.transpose(2, 3)


def _fill16(st, gen):
    case = st["case"]
    shape = (st["pages"], case["kv_heads"], PAGE * case["head_dim"])
    st["k16"], st["v16"] = (_normal(shape, _type(case), gen) for _ in "kv")


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    ctx, new = _lengths(case)
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    t, total = _type(case), sum(new)
    per_req = [(c + n + PAGE - 1) // PAGE for c, n in zip(ctx, new)]
    pages = sum(per_req) + max(4, sum(per_req) // 8)
    order = np.random.default_rng(seed).permutation(pages).astype(np.int32)
    table = np.zeros((len(ctx), max(per_req)), dtype=np.int32)
    at = 0
    for r, n in enumerate(per_req):
        table[r, :n] = order[at:at + n]
        at += n
    st = {"case": case, "pages": pages, "table": torch.from_numpy(table).cuda(),
          "eps": EPS, "scale": 1.0 / math.sqrt(d)}
    # where the new tokens lie: request and position of each, and the pages they fall into
    who = np.repeat(np.arange(len(new)), new)
    pos = np.concatenate([np.arange(c, c + n) for c, n in zip(ctx, new)])
    start = np.concatenate([[True], (who[1:] != who[:-1]) | (pos[1:] // PAGE != pos[:-1] // PAGE)])
    for name, x in (("who", who), ("pos", pos), ("block", np.cumsum(start) - 1),
                    ("first", np.flatnonzero(start)), ("ctx", np.array(ctx)), ("new", np.array(new))):
        st[name] = torch.from_numpy(np.ascontiguousarray(x, dtype=np.int64)).cuda()
    st["longest"], st["most_new"] = max(c + n for c, n in zip(ctx, new)), max(new)
    eight = case["op"] != "norm" or case["into8"]
    (_fill8 if eight else _fill16)(st, gen)
    if case["op"] in ("append", "norm"):
        std = _head_std(hkv)
        st["k_new"] = _normal((total, hkv, d), torch.float32, gen).mul_(std).to(t)
        st["v_new"] = _normal((total, hkv, d), torch.float32, gen).mul_(std).to(t)
    if case["op"] in ("attend", "norm"):
        st["q"] = _normal((total, hq, d), t, gen)
    if case["op"] == "norm":
        st["q_weight"] = (1.0 + 0.2 * _normal((d,), torch.float32, gen)).to(t)
        st["k_weight"] = (1.0 + 0.2 * _normal((d,), torch.float32, gen)).to(t)
        theta = 10000.0 ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device="cuda") / d)
        angle = torch.arange(st["longest"], dtype=torch.float64, device="cuda")[:, None] * theta
        st["cos_sin"] = torch.cat([angle.cos(), angle.sin()], 1).float().contiguous()
    if own:
        from paper_2312_05516_amd import binding as pv
        desc = pv.pool_desc(pages, hkv, d, case["dtype"])
        make = pv.plan_create_kv8 if eight else pv.plan_create
        st["plan"] = make(desc, hq, ctx, new, table.shape[1])
        pv.plan_upload(st["plan"])
        if eight:
            st["pool"] = pv.Kv8Pool(st["k8"], st["v8"], st["k_scales"], st["v_scales"])
        if "q" in st:
            st["out"] = torch.empty_like(st["q"])
        if case["op"] == "attend":
            st["ws"] = torch.empty(max(256, pv.plan_workspace_bytes(st["plan"])), dtype=torch.uint8,
                                   device="cuda")
        if case["op"] == "read" or eight and case["op"] == "norm":
            st["k_rows"], st["v_rows"] = (torch.empty((total, hkv, d), dtype=t, device="cuda")
                                          for _ in "kv")
    return st


def _pools8(st):
    return {"k": st["k8"].view(torch.float8_e4m3fn), "v": st["v8"].view(torch.float8_e4m3fn),
            "k_scales": st["k_scales"], "v_scales": st["v_scales"]}


def run(st):
    op = st["case"]["op"]
    if own:
        from paper_2312_05516_amd import binding as pv
        if op == "attend":
            pv.kv8_multi_token_paged_attn_planned(st["plan"], st["q"], st["pool"], st["table"],
                                                  st["scale"], st["out"], st["ws"])
            return {"out": st["out"]}
        if op == "append":
            pv.kv8_append_planned(st["plan"], st["k_new"], st["v_new"], st["table"], st["pool"])
            return _pools8(st)
        if op == "read":
            pv.kv8_read_planned(st["plan"], st["pool"], st["table"], st["k_rows"], st["v_rows"])
            return {"k": st["k_rows"], "v": st["v_rows"]}
        if not st["case"]["into8"]:
            pv.norm_rope_kv_append_planned(st["plan"], st["q"], st["out"], st["k_new"], st["v_new"],
                                           st["q_weight"], st["k_weight"], st["eps"], st["cos_sin"],
                                           st["case"]["style"], st["table"], st["k16"], st["v16"])
            return {"q": st["out"], "k": st["k16"], "v": st["v16"]}
        pv.kv8_norm_rope_append_planned(st["plan"], st["q"], st["out"], st["k_new"], st["v_new"],
                                        st["q_weight"], st["k_weight"], st["eps"], st["cos_sin"],
                                        st["case"]["style"], st["table"], st["pool"])
        pv.kv8_read_planned(st["plan"], st["pool"], st["table"], st["k_rows"], st["v_rows"])
        return {"q": st["out"], "k": st["k_rows"], "v": st["v_rows"]}
    if op == "attend":
        return {"out": _attend(st)}
    if op == "append":
        _append(st, st["k_new"], st["v_new"])
        return _pools8(st)
    if op == "read":
        return _read(st)
    q, k = (_norm_rope(st, st[x], st[x[0] + "_weight"]) for x in ("q", "k_new"))
    if st["case"]["into8"]:
        _append(st, k, st["v_new"])
        return {"q": q, **_read(st)}
    h, d = st["case"]["kv_heads"], st["case"]["head_dim"]
    page, slot = _places(st)
    st["k16"].view(-1, h, d // 8, PAGE, 8)[page, :, :, slot] = k.view(-1, h, d // 8, 8)
    st["v16"].view(-1, h, 2, d, 8)[page, :, slot // 8, :, slot % 8] = st["v_new"]
    return {"q": q, "k": st["k16"], "v": st["v16"]}


def _places(st):
    return st["table"][st["who"], st["pos"] // PAGE].long(), st["pos"] % PAGE


def _append(st, k_new, v_new):
    h, d, dtype = st["case"]["kv_heads"], st["case"]["head_dim"], st["case"]["dtype"]
    page, slot = _places(st)
    pages, s0 = page[st["first"]], slot[st["first"]]
    kept = (torch.arange(PAGE, device="cuda")[None] < s0[:, None])[:, None, :, None]
    k8, v8 = _k8(st), _v8(st)
    old_k = k8[pages].transpose(3, 4).reshape(-1, h, PAGE, d)
    old_v = v8[pages].transpose(2, 3)
    for name, rows, old in (("k", k_new.float(), old_k), ("v", v_new.float(), old_v)):
        size = torch.where(torch.isfinite(rows), rows.abs(), torch.zeros_like(rows)).amax(2)
        amax = torch.zeros((len(pages), h), device="cuda").index_reduce_(0, st["block"], size, "amax")
        scales = st[name + "_scales"].view(-1, h)
        before = scales[pages].to(torch.int32) - 127
        e = _need(amax, dtype)
        e = torch.where(s0[:, None] > 0, torch.maximum(e, before), e)
        again = _encode(_decode(old) * _power((before - e).clamp(min=-126)[:, :, None, None]),
                        torch.zeros_like(e)[:, :, None, None], dtype)
        codes = torch.where(kept & (e > before)[:, :, None, None], again, old)
        scales[pages] = (e + 127).to(torch.uint8)
        if name == "k":
            k8[pages] = codes.view(-1, h, 4, 4, d // 16, 16).transpose(3, 4)
        else:
            v8[pages] = codes.transpose(2, 3)
        new = _encode(rows, e[st["block"]][:, :, None], dtype)
        if name == "k":
            k8[page, :, slot // 4, :, slot % 4] = new.view(-1, h, d // 16, 16)
        else:
            v8[page, :, :, slot] = new


def _read(st):
    h, d = st["case"]["kv_heads"], st["case"]["head_dim"]
    page, slot = _places(st)
    t = _type(st["case"])
    k = _k8(st)[page, :, slot // 4, :, slot % 4].reshape(-1, h, d)
    v = _v8(st)[page, :, :, slot]
    e_k, e_v = (st[n].view(-1, h)[page].to(torch.int32)[:, :, None] - 127
                for n in ("k_scales", "v_scales"))
    return {"k": (_decode(k) * _power(e_k)).to(t), "v": (_decode(v) * _power(e_v)).to(t)}


def _norm_rope(st, x, weight):
    d = st["case"]["head_dim"]
    x = x.float()
    x = x * torch.rsqrt(x.square().mean(2, keepdim=True) + st["eps"]) * weight.float()
    c, s = st["cos_sin"][st["pos"]][:, None].split(d // 2, 2)
    if st["case"]["style"] == "half":
        a, b = x[:, :, :d // 2], x[:, :, d // 2:]
        y = torch.cat([a * c - b * s, b * c + a * s], 2)
    else:
        a, b = x[:, :, 0::2], x[:, :, 1::2]
        y = torch.stack([a * c - b * s, b * c + a * s], 3).flatten(2)
    return y.to(_type(st["case"]))


def _attend(st):
    case = st["case"]
    hq, h, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    g, n = hq // h, st["most_new"]
    table = st["table"].long()
    r, length = table.shape[0], table.shape[1] * PAGE
    key = torch.arange(length, device="cuda")
    gone = (key >= (st["ctx"] + st["new"])[:, None])[:, None, :, None]

    def rows(codes, order, scales):
        x = _decode(codes) * _power(scales.view(-1, h)[table].to(torch.int32) - 127).view(
            r, -1, h, *[1] * (codes.dim() - 3))
        return x.permute(order).reshape(r, h, length, d).masked_fill_(gone, 0.0)

    # the requests' queries side by side, padded to the longest
    i = torch.arange(n, device="cuda")[None].minimum(st["new"][:, None] - 1)
    at = torch.cumsum(st["new"], 0) - st["new"]
    q = st["q"].float()[at[:, None] + i].view(r, n, h, g, d).transpose(1, 2).reshape(r, h, n * g, d)
    s = torch.matmul(q, rows(_k8(st)[table], (0, 2, 1, 3, 5, 4, 6), st["k_scales"]).transpose(2, 3))
    s *= st["scale"]
    unseen = key > (st["ctx"][:, None] + i)[:, :, None]
    s.view(r, h, n, g, length).masked_fill_(unseen[:, None, :, None], -math.inf)
    s = s.sub_(s.amax(3, keepdim=True)).exp_()
    out = torch.matmul(s, rows(_v8(st)[table], (0, 2, 1, 4, 3), st["v_scales"]))
    out /= s.sum(3, keepdim=True)
    out = out.view(r, h, n, g, d).transpose(1, 2).reshape(r * n, hq, d)
    return out[st["who"] * n + st["pos"] - st["ctx"][st["who"]]].to(_type(case))


# The same in 64 bits, from the definitions: one request after another, codes by their table of values

def _values64():
    """The values of the codes 0..126: without a sign."""
    c = torch.arange(127, dtype=torch.float64)
    m, x = c % 8, (c / 8).floor()
    return torch.where(x > 0, (1 + m / 8) * 2.0 ** (x - 7), m / 8 * 2.0 ** -6).cuda()


def _code_values64(codes):
    v = _values64()
    v = torch.cat([v, torch.full((1,), math.nan, dtype=torch.float64, device="cuda")])
    return torch.cat([v, -v])[codes.long()]


def _nearest64(x, most):
    """Nearest code value, ties to the even code, no larger than `most`."""
    v = _values64()
    mid = (v[1:] + v[:-1]) / 2
    a = x.abs()
    i = torch.searchsorted(mid, a.contiguous())
    tie = (i < 126) & (a == mid[i.clamp(max=125)]) & (i % 2 == 1)
    return torch.sign(x) * v[i + tie.long()].clamp(max=most)


def _rows64(st, r, lo, hi, which):
    """Values of positions lo..hi-1 of request r: [positions, heads, dims]."""
    h, d = st["case"]["kv_heads"], st["case"]["head_dim"]
    t = torch.arange(lo, hi, device="cuda")
    page = st["table"][r].long()[t // PAGE]
    s, i = (t % PAGE)[:, None], torch.arange(d, device="cuda")
    if which == "k":
        inside = torch.div(s, 4, rounding_mode="floor") * 4 * d + i // 16 * 64 + s % 4 * 16 + i % 16
    else:
        inside = i * 16 + s
    tile = page[:, None] * h + torch.arange(h, device="cuda")
    codes = st[which + "8"][tile[:, :, None] * (PAGE * d) + inside[:, None]]
    e = st[which + "_scales"][tile].double() - 127
    return _code_values64(codes) * torch.exp2(e)[:, :, None]


def _exact_attend(st, ctx, new):
    case = st["case"]
    h, d = case["kv_heads"], case["head_dim"]
    g, at, outs = case["q_heads"] // h, 0, []
    for r, (c, n) in enumerate(zip(ctx, new)):
        k, v = (_rows64(st, r, 0, c + n, x).transpose(0, 1) for x in "kv")
        q = st["q"][at:at + n].double().view(n, h, g, d).permute(1, 2, 0, 3).reshape(h, g * n, d)
        at += n
        s = torch.matmul(q, k.transpose(1, 2).contiguous()) / math.sqrt(d)
        seen = torch.arange(c + n, device="cuda") <= c + torch.arange(n, device="cuda")[:, None]
        s = torch.where(seen.repeat(g, 1), s, -math.inf)
        o = torch.matmul(torch.softmax(s, 2), v.contiguous())
        outs.append(o.view(h, g, n, d).permute(2, 0, 1, 3).reshape(n, h * g, d))
    return torch.cat(outs)


def _exact_append(st, ctx, new, k_new, v_new):
    """Values (without their scales) of the pools' codes after the append, and of the new rows with
    their scales."""
    case = st["case"]
    h, d = case["kv_heads"], case["head_dim"]
    least, largest = E_RANGE[case["dtype"]]
    got = {}
    for which, fresh in (("k", k_new), ("v", v_new)):
        values, rows, at = _code_values64(st[which + "8"]).view(-1, PAGE * d), [], 0
        slot, dim = torch.arange(PAGE, device="cuda")[:, None], torch.arange(d, device="cuda")
        if which == "k":
            inside = slot // 4 * 4 * d + dim // 16 * 64 + slot % 4 * 16 + dim % 16
        else:
            inside = dim * 16 + slot
        for r, (c, n) in enumerate(zip(ctx, new)):
            for p in range(c // PAGE, (c + n - 1) // PAGE + 1):
                lo, hi = max(c, p * PAGE), min(c + n, (p + 1) * PAGE)
                x = fresh[at:at + hi - lo].double().transpose(0, 1)
                at += hi - lo
                tiles = int(st["table"][r, p]) * h + torch.arange(h, device="cuda")
                e = torch.ceil(torch.log2(x.abs().amax((1, 2)) / 448)).clamp(least, largest)
                e += (x.abs().amax((1, 2)) > 448 * torch.exp2(e)).double()  # a logarithm rounded down
                e -= ((x.abs().amax((1, 2)) <= 224 * torch.exp2(e)) & (e > least)).double()  # or up
                s0 = lo - p * PAGE
                if s0 > 0:
                    before = st[which + "_scales"][tiles].double() - 127
                    e = torch.maximum(e, before)
                    front = inside[:s0]
                    old = values[tiles[:, None, None], front]
                    values[tiles[:, None, None], front] = _nearest64(
                        old * torch.exp2(before - e)[:, None, None], 448.0)
                y = _nearest64(x * torch.exp2(-e)[:, None, None], 448.0)
                y = torch.where((e == largest)[:, None, None], y.clamp(-240, 240), y)
                values[tiles[:, None, None], inside[s0:s0 + hi - lo]] = y
                rows.append((y * torch.exp2(e)[:, None, None]).transpose(0, 1))
        got[which] = (values, torch.cat(rows))
    return got


def _exact_norm_rope(st, x, weight):
    case, d = st["case"], st["case"]["head_dim"]
    x = x.double()
    y = x * weight.double() / torch.sqrt((x * x).sum(2, keepdim=True) / d + st["eps"])
    z = torch.empty_like(y)
    turn = st["cos_sin"].double()[st["pos"]]
    for i in range(d // 2):
        a, b = (2 * i, 2 * i + 1) if case["style"] == "interleaved" else (i, i + d // 2)
        c, s = turn[:, None, i], turn[:, None, d // 2 + i]
        z[:, :, a], z[:, :, b] = y[:, :, a] * c - y[:, :, b] * s, y[:, :, b] * c + y[:, :, a] * s
    return z


def exact(case, seed):
    st = prepare(case, seed)
    ctx, new = _lengths(case)
    h, d = case["kv_heads"], case["head_dim"]
    pages = sum((c + n - 1) // PAGE - c // PAGE + 1 for c, n in zip(ctx, new))
    if case["op"] == "attend":
        return {"out": _exact_attend(st, ctx, new)}
    if case["op"] == "read":
        k, v = (torch.cat([_rows64(st, r, c, c + n, x) for r, (c, n) in enumerate(zip(ctx, new))])
                for x in "kv")
        return {"k": k, "v": v}
    if case["op"] == "append":
        if pages > 8000:  # one page after another: too long
            return None
        got = _exact_append(st, ctx, new, st["k_new"], st["v_new"])
        return {"k": got["k"][0], "v": got["v"][0], "k_scales": None, "v_scales": None}
    q, k = (_exact_norm_rope(st, st[x], st[x[0] + "_weight"]) for x in ("q", "k_new"))
    if case["into8"]:
        if pages > 8000:
            return {"q": q, "k": None, "v": None}
        got = _exact_append(st, ctx, new, k.to(_type(case)), st["v_new"])
        return {"q": q, "k": got["k"][1], "v": got["v"][1]}
    kp, vp = st["k16"].double().view(-1, h, PAGE * d), st["v16"].double().view(-1, h, PAGE * d)
    at = 0
    for r, (c, n) in enumerate(zip(ctx, new)):
        t = torch.arange(c, c + n, device="cuda")
        page, slot = st["table"][r].long()[t // PAGE], (t % PAGE)[:, None]
        dim = torch.arange(d, device="cuda")
        where = page[:, None, None], torch.arange(h, device="cuda")[None, :, None]
        kp[(*where, (dim // 8 * 128 + slot * 8 + dim % 8)[:, None])] = k[at:at + n]
        vp[(*where, (slot // 8 * 8 * d + dim * 8 + slot % 8)[:, None])] = st["v_new"][at:at + n].double()
        at += n
    return {"q": q, "k": kp, "v": vp}
