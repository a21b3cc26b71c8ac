"""The key/value store's operators as they are measured: writing a quantised cache and reading it back, decode attention
over such a cache, and decode attention for a batch that shares long prefixes.

A store holds the K and V rows of one layer, ``[batch][kv heads][capacity][128]``, as bf16 or as codes with bf16 scales:

  e4m3   8-bit floats, one power-of-two scale a row: the smallest 2^e with max|x| / 2^e <= 448
  int8   whole numbers -127..127, one scale a row: bf16(max|x| / 127)
  int4   whole numbers -7..7 (stored + 8 in a nibble), one scale for each 32 elements: bf16(max|x| / 7)

A scale is at least 2^-126; a code is the element over its scale, rounded to the nearest, ties to even. The four elements
32g + 4q .. 32g + 4q + 3 of an int4 row are the nibbles, lowest first, of its 16-bit word 4q + g.

Where ``own`` is false, ``run`` computes the operators with elementary torch operations in 32 bits; where it is true it makes
the calls of the package.
"""
import math

import numpy as np
import torch

own = False

D = 128
FORMATS = ("bf16", "e4m3", "int8", "int4")
GROUPS = {"bf16": 0, "e4m3": 1, "int8": 1, "int4": 4}         # scales a row
ROW_BYTES = {"bf16": 256, "e4m3": 130, "int8": 130, "int4": 72}   # codes and scales of a row
DTYPE = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8, "int4": torch.uint8}
# query heads / KV heads of the 7B shape, the eviction sweep, the 32B shape and the smallest test configuration
HEADS = ((28, 4), (32, 8), (64, 8), (8, 2))


# ------------------------------------------------------------------------------------------------ the cases
def listed():
    def store(name, **kw):
        return {"name": name, "op": "store", **kw}

    def attn(name, **kw):
        return {"name": name, "op": "attn", "prefixes": 0, "prefix": 0, "prefix_least": 0, **kw}

    return [
        # one decode step of the 7B shape: one token a sequence is written behind the tokens that are there
        store("write one token", fmt="e4m3", batch=32, h_q=28, h_kv=4, capacity=1152, tokens=1, least=1, packed=True),
        # a batch of prompts of different lengths, K and V as they lie in the output of a fused projection
        store("write ragged prompts", fmt="int8", batch=8, h_q=28, h_kv=4, capacity=4608, tokens=4097, least=129, packed=True),
        # long prompts that are kept in 4 bits
        store("write long prompts", fmt="int4", batch=4, h_q=32, h_kv=8, capacity=33024, tokens=32768, least=32768, packed=False),
        # one sequence that comes back from 4 bits, the eviction step's smallest cache
        {"name": "read one sequence", "op": "read", "fmt": "int4", "batch": 1, "h_q": 8, "h_kv": 2, "capacity": 640, "tokens": 640, "least": 640},
        # a whole batch that comes back, every sequence at its own length
        {"name": "read a batch", "op": "read", "fmt": "e4m3", "batch": 64, "h_q": 64, "h_kv": 8, "capacity": 2304, "tokens": 2304, "least": 1500},
        # decode steps: one sequence (latency), the 7B batch, the 32B batch, and few sequences at a very long context
        attn("attention, one sequence", fmt="e4m3", batch=1, h_q=28, h_kv=4, capacity=640, longest=639, least=639, append=True),
        attn("attention, 7B batch", fmt="int8", batch=32, h_q=28, h_kv=4, capacity=1152, longest=1151, least=1, append=True),
        attn("attention, 32B batch", fmt="e4m3", batch=128, h_q=64, h_kv=8, capacity=2304, longest=2303, least=2048, append=True),
        attn("attention, long context", fmt="int4", batch=2, h_q=32, h_kv=8, capacity=131072, longest=131071, least=100003, append=False),
        # several answers sampled for one question: the question's rows are shared, each answer has its own compressed cache
        attn("shared question, 8 answers", fmt="bf16", batch=8, h_q=28, h_kv=4, capacity=640, longest=600, least=0, append=True,
             prefixes=1, prefix=2049, prefix_least=2049),
        attn("shared document, 32 answers", fmt="bf16", batch=32, h_q=28, h_kv=4, capacity=1152, longest=1100, least=1024, append=True,
             prefixes=1, prefix=8192, prefix_least=8192),
        attn("4 documents, 128 answers", fmt="e4m3", batch=128, h_q=64, h_kv=8, capacity=2304, longest=2303, least=1024, append=True,
             prefixes=4, prefix=16384, prefix_least=9000),
    ]


def _between(rng, lo, hi):
    """A whole number of lo..hi, spread over its logarithm."""
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(("store", "store", "read", "attn", "attn", "attn", "prefix", "prefix", "prefix"))
    h_q, h_kv = rng.choice(HEADS)
    if op in ("store", "read"):
        case = {"op": op, "fmt": rng.choice(FORMATS[1:]), "batch": _between(rng, 1, 64), "h_q": h_q, "h_kv": h_kv}
        most = 32768 * 32 // (case["batch"] * h_kv) if op == "store" else 64 * 8 * 2304 // (case["batch"] * h_kv)
        case["tokens"] = _between(rng, 1, min(most, 32768))
        case["least"] = rng.choice((case["tokens"], _between(rng, 1, case["tokens"])))
        case["capacity"] = case["tokens"] + rng.choice((0, 1, 127))
        if op == "store":
            case["packed"] = rng.random() < 0.5
        return case
    if op == "attn":
        case = {"op": "attn", "fmt": rng.choice(FORMATS[1:]), "batch": _between(rng, 1, 128), "h_q": h_q, "h_kv": h_kv}
        longest = _between(rng, 1, min(131071, 128 * 8 * 2303 // (case["batch"] * h_kv)))
        case |= {"prefixes": 0, "prefix": 0, "prefix_least": 0}
    else:
        prefixes = rng.choice((1, 1, 2, 3, 4))
        case = {"op": "attn", "fmt": rng.choice(FORMATS), "batch": prefixes * _between(rng, 1, 128 // prefixes), "h_q": h_q, "h_kv": h_kv}
        longest = _between(rng, 1, 2303)
        prefix = _between(rng, 1, 16384)
        case |= {"prefixes": prefixes, "prefix": prefix, "prefix_least": rng.choice((prefix, _between(rng, 1, prefix)))}
    case |= {"longest": longest, "least": rng.choice((longest, rng.randint(0, longest))), "append": rng.random() < 0.7}
    case["capacity"] = longest + rng.choice((1, 16, 129))
    return case


def _lengths(least, most, n, at):
    """n lengths of least..most, the longest among them, the same ones for every seed."""
    got = np.random.RandomState(1000 * n + at).randint(least, most + 1, n) if n else np.zeros(0, np.int64)
    if n:
        got[(7 * at) % n] = most
    return got.astype(np.int64)


def _counts(case):
    return _lengths(case["least"], case["tokens"], case["batch"], case["tokens"] % 97)


def _lens(case):
    return _lengths(case["least"], case["longest"], case["batch"], case["longest"] % 89)


def _prefix_lens(case):
    return _lengths(case["prefix_least"], case["prefix"], case["prefixes"], case["prefix"] % 83)


def work(case):
    row = ROW_BYTES[case["fmt"]]
    if case["op"] in ("store", "read"):
        rows = 2 * int(_counts(case).sum()) * case["h_kv"]
        passes = 2 if case["op"] == "store" else 1   # a store case writes the rows and reads them back
        return {"bytes": passes * rows * (2 * D + row), "flops": passes * rows * 2 * D}
    g_rows = case["batch"] * case["h_q"]
    new = 1 if case["append"] else 0
    own_rows, plens = _lens(case), _prefix_lens(case)
    heads = case["h_kv"]
    b = 2 * heads * int(own_rows.sum()) * row + new * 2 * heads * case["batch"] * (2 * D + row)
    b += 2 * heads * int(plens.sum()) * 2 * D + g_rows * (2 * 2 * D + 4)
    keys = int(own_rows.sum()) + new * case["batch"]
    if case["prefixes"]:
        keys += int(plens.sum()) * (case["batch"] // case["prefixes"])
    return {"bytes": b, "flops": 4 * D * keys * case["h_q"]}


# ------------------------------------------------------------------------------------------------ the store's arithmetic
def _scale(amax, fmt):
    """Scales of fp32 maxima, in fp32 (every one a bf16 value)."""
    if fmt == "e4m3":
        m, e = torch.frexp(amax)                        # amax = m 2^e, 1/2 <= m < 1; 448 = 0.875 * 2^9
        e = torch.where(m <= 0.875, e - 9, e - 8)
        e = torch.where(amax > 0, e, torch.full_like(e, -126)).clamp(min=-126)
        return torch.ldexp(torch.ones_like(amax), e)
    s = (amax / (127.0 if fmt == "int8" else 7.0)).to(torch.bfloat16).float()
    return s.clamp(min=2.0 ** -126)


def _encode(x, fmt):
    """bf16 rows [..., 128] -> codes and bf16 scales [..., scales a row]."""
    if fmt == "bf16":
        return x, None
    x = x.float().unflatten(-1, (GROUPS[fmt], -1))
    s = _scale(x.abs().amax(-1, keepdim=True), fmt)
    q = (x / s).flatten(-2)
    s = s.squeeze(-1).to(torch.bfloat16)
    if fmt == "e4m3":
        return q.to(torch.float8_e4m3fn), s
    q = torch.round(q)
    if fmt == "int8":
        return q.to(torch.int8), s
    q = (q + 8).to(torch.uint8).unflatten(-1, (4, 8, 4)).transpose(-3, -2).flatten(-3).unflatten(-1, (64, 2))
    return q[..., 0] | (q[..., 1] << 4), s


def _decode(c, s, fmt, dtype=torch.float32):
    """The values that codes and scales stand for, in fp32 or fp64."""
    if fmt == "bf16":
        return c.to(dtype)
    if fmt == "int4":
        c = torch.stack((c & 15, c >> 4), -1).flatten(-2).unflatten(-1, (8, 4, 4)).transpose(-3, -2).flatten(-3)
        c = c.to(dtype) - 8
    return (c.to(dtype).unflatten(-1, (GROUPS[fmt], -1)) * s.to(dtype).unsqueeze(-1)).flatten(-2)


# ------------------------------------------------------------------------------------------------ inputs
def _rand(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)


def _keys(gen, *shape):
    """Keys as they come out of a projection: a few channels are much larger than the others."""
    channel = torch.exp(0.5 * _rand(gen, D))
    return (_rand(gen, *shape, D) * channel).to(torch.bfloat16)


def _filled(gen, case):
    """Codes and scales of a store whose rows have all been written, in pieces to save memory."""
    b, h, c, fmt = case["batch"], case["h_kv"], case["capacity"], case["fmt"]
    got = []
    for kind in ("k", "v"):
        parts = [_encode(_keys(gen, h, c) if kind == "k" else _rand(gen, h, c, D).to(torch.bfloat16), fmt) for _ in range(b)]
        codes = torch.stack([p[0].view(torch.uint8) if fmt == "e4m3" else p[0] for p in parts])
        got.append((codes.view(DTYPE[fmt]), None if fmt == "bf16" else torch.stack([p[1] for p in parts])))
    return got


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    b, h_q, h, c, fmt = case["batch"], case["h_q"], case["h_kv"], case["capacity"], case["fmt"]
    st = {"case": case}
    if case["op"] == "attn":
        (st["k"], st["k_scale"]), (st["v"], st["v_scale"]) = _filled(gen, case)
        st["length"] = torch.from_numpy(_lens(case)).to("cuda", torch.int32)
        st["q"] = _rand(gen, b, h_q, D).to(torch.bfloat16)
        st["k_new"] = _keys(gen, b, h) if case["append"] else None
        st["v_new"] = _rand(gen, b, h, D).to(torch.bfloat16) if case["append"] else None
        st["out"] = torch.zeros_like(st["q"])
        st["lse"] = torch.zeros((b, h_q), dtype=torch.float32, device="cuda")
        if case["prefixes"]:
            st["k_prefix"] = _keys(gen, case["prefixes"], h, case["prefix"])
            st["v_prefix"] = _rand(gen, case["prefixes"], h, case["prefix"], D).to(torch.bfloat16)
            st["prefix_lens"] = [int(n) for n in _prefix_lens(case)]
            st["prefix_lens_dev"] = torch.tensor(st["prefix_lens"], device="cuda")
        return st
    n = case["tokens"]
    counts = _counts(case)
    st["count"] = torch.from_numpy(counts).to("cuda", torch.int32)
    # the rows go behind the ones that are there, as far as the capacity lets them
    st["first"] = torch.from_numpy((c - counts) * 7 // 8).to("cuda", torch.int32)
    st["k_out"] = torch.zeros((b, n, h, D), dtype=torch.bfloat16, device="cuda")
    st["v_out"] = torch.zeros_like(st["k_out"])
    if case["op"] == "read":
        (st["k"], st["k_scale"]), (st["v"], st["v_scale"]) = _filled(gen, case)
        return st
    shape = (b, h, c, 64 if fmt == "int4" else D)
    for name in ("k", "v"):
        st[name] = torch.zeros(shape, dtype=torch.uint8, device="cuda").view(DTYPE[fmt])
        st[name + "_scale"] = torch.zeros((b, h, c, GROUPS[fmt]), dtype=torch.bfloat16, device="cuda")
    if case["packed"]:   # [tokens][all heads of q, k and v][128], k and v are views of it
        qkv = torch.randn((b, n, h_q + 2 * h, D), generator=gen, device="cuda", dtype=torch.bfloat16)
        st["k_in"], st["v_in"] = qkv[:, :, h_q:h_q + h], qkv[:, :, h_q + h:]
        st["k_in"] *= torch.exp(0.5 * _rand(gen, D))
    else:
        st["k_in"], st["v_in"] = _keys(gen, b, n, h), _rand(gen, b, n, h, D).to(torch.bfloat16)
    return st


# ------------------------------------------------------------------------------------------------ one pass
def _bytes(x):
    return x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x


def _plain_write(st, x, name):
    """Codes and scales of x [batch][tokens][kv heads][128] into the store's rows first .. first + count - 1."""
    case = st["case"]
    codes, scale = _encode(x, case["fmt"])
    for dst, src in ((_bytes(st[name]), _bytes(codes)), (st[name + "_scale"], scale)):
        if case["least"] == case["tokens"]:      # every sequence has all tokens: an indexed store
            rows = st["first"].long()[:, None] + torch.arange(case["tokens"], device="cuda")
            dst[torch.arange(case["batch"], device="cuda")[:, None], :, rows] = src
        else:                                    # else by the store's rows, each from its token or as it was
            t = torch.arange(case["capacity"], device="cuda") - st["first"].long()[:, None]
            here = (t >= 0) & (t < st["count"].long()[:, None])
            index = t.clamp(0, case["tokens"] - 1)[:, :, None, None].expand(-1, -1, *src.shape[2:])
            dst.copy_(torch.where(here[:, None, :, None], src.gather(1, index).transpose(1, 2), dst))


def _plain_read(st, name, out):
    case = st["case"]
    t = torch.arange(case["tokens"], device="cuda")
    rows = (st["first"].long()[:, None] + t).clamp(max=case["capacity"] - 1)
    at = torch.arange(case["batch"], device="cuda")[:, None]
    codes = _bytes(st[name])[at, :, rows].view(st[name].dtype)
    x = _decode(codes, st[name + "_scale"][at, :, rows], case["fmt"]).to(torch.bfloat16)
    here = (t < st["count"].long()[:, None])[:, :, None, None]
    out.copy_(x if case["least"] == case["tokens"] else torch.where(here, x, out))


def _plain_attn(st):
    case = st["case"]
    b, h_q, h, fmt = case["batch"], case["h_q"], case["h_kv"], case["fmt"]
    n = st["length"].long()
    if case["append"]:
        at = torch.arange(b, device="cuda")
        for name in ("k", "v"):
            codes, scale = _encode(st[name + "_new"], fmt)
            _bytes(st[name])[at, :, n] = _bytes(codes)
            if scale is not None:
                st[name + "_scale"][at, :, n] = scale
        n = n + 1
    most = case["longest"] + int(case["append"])

    def values(name):
        s = st[name + "_scale"]
        return _decode(st[name][:, :, :most], None if s is None else s[:, :, :most], fmt)

    q = st["q"].float().view(b, h, h_q // h, D)
    z = (q @ values("k").transpose(-1, -2)) / math.sqrt(D)
    z = z.masked_fill((torch.arange(most, device="cuda") >= n[:, None])[:, None, None, :], -math.inf)
    if case["prefixes"]:
        p = case["prefixes"]
        qp = q.view(p, b // p, h, h_q // h, D).transpose(1, 2).flatten(2, 3)              # [prefix][head][rows][128]
        zp = (qp @ st["k_prefix"].float().transpose(-1, -2)) / math.sqrt(D)
        zp = zp.masked_fill((torch.arange(case["prefix"], device="cuda") >= st["prefix_lens_dev"][:, None])[:, None, None, :], -math.inf)
        zp = zp.unflatten(2, (b // p, h_q // h)).transpose(1, 2).flatten(0, 1)
        z = torch.cat((z, zp), -1)
    m = z.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)      # nothing to attend to: out = 0, lse = -inf
    w = torch.exp(z - m)
    total = w.sum(-1, keepdim=True)
    o = w[..., :most] @ values("v")
    if case["prefixes"]:
        wp = w[..., most:].unflatten(0, (p, b // p)).transpose(1, 2).flatten(2, 3)
        op = wp @ st["v_prefix"].float()
        o = o + op.unflatten(2, (b // p, h_q // h)).transpose(1, 2).flatten(0, 1)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    st["out"].copy_(o.view(b, h_q, D))
    st["lse"].copy_((m + torch.log(total)).view(b, h_q))


def _store(st):
    """The handle that a program keeps over its buffers; made at the first pass."""
    if "store" not in st:
        import paper_2512_00504_b200 as gkv
        case = st["case"]
        st["store"] = gkv.KVStore(case["fmt"], batch=case["batch"], h_q=case["h_q"], h_kv=case["h_kv"], capacity=case["capacity"],
                                  buffers=(st["k"], st["v"], st["k_scale"], st["v_scale"]) if case["fmt"] != "bf16" else (st["k"], st["v"]),
                                  max_prefix=case.get("prefix", 0), n_prefix=case.get("prefixes", 0))
        if case.get("prefixes"):
            st["prefix"] = gkv.Prefix(st["k_prefix"], st["v_prefix"], st["prefix_lens"])
    return st["store"]


def run(state):
    st, case = state, state["case"]
    if case["op"] == "attn":
        if own:
            _store(st).attn(st["length"], st["q"], st["out"], k_new=st["k_new"], v_new=st["v_new"], prefix=st.get("prefix"),
                            lse=st["lse"], max_len=case["longest"])
        else:
            _plain_attn(st)
        got = {"out": st["out"], "lse": st["lse"]}
        if case["append"]:   # the store with its new rows
            got |= {name: st[name] for name in ("k", "v", "k_scale", "v_scale") if st[name] is not None and not (case["fmt"] == "int4" and "scale" not in name)}
        return got
    if case["op"] == "store":
        if own:
            _store(st).write(st["k_in"], st["v_in"], first=st["first"], count=st["count"])
        else:
            _plain_write(st, st["k_in"], "k")
            _plain_write(st, st["v_in"], "v")
    if own:
        _store(st).read(st["k_out"], st["v_out"], first=st["first"], count=st["count"])
    else:
        _plain_read(st, "k", st["k_out"])
        _plain_read(st, "v", st["v_out"])
    got = {"k_out": st["k_out"], "v_out": st["v_out"]}
    return got if case["op"] == "read" else got | {"k_scale": st["k_scale"], "v_scale": st["v_scale"]}


# ------------------------------------------------------------------------------------------------ in 64 bits
def _exact_code(x, fmt):
    """(codes as fp64 numbers, scales as fp64 numbers) of rows, from the definition."""
    x = x.double().unflatten(-1, (GROUPS[fmt], -1))
    a = x.abs().amax(-1, keepdim=True)
    least = 2.0 ** -126
    if fmt == "e4m3":
        s = torch.exp2(torch.ceil(torch.log2((a / 448).clamp(min=least))))
        y = x / s
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)      # spacing of 8-bit floats
        return torch.round(y / step) * step, s
    s = (a / (127 if fmt == "int8" else 7)).to(torch.bfloat16).double().clamp(min=least)
    return torch.round(x / s), s


def _exact_values(st, name, b, rows):
    """fp64 values of the first rows of sequence b of the store, without the plain form's helpers."""
    fmt, c = st["case"]["fmt"], st[name][b, :, :rows]
    if fmt == "bf16":
        return c.double()
    if fmt == "int4":
        x = torch.empty(c.shape[:-1] + (D,), dtype=torch.float64, device=c.device)
        for e in range(D):
            g, q, i = e // 32, (e % 32) // 4, e % 4
            x[..., e] = ((c[..., 8 * q + 2 * g + i // 2] >> (4 * (i % 2))) & 15).double() - 8
    else:
        x = c.double()
    s = st[name + "_scale"][b, :, :rows].double()
    return x * torch.repeat_interleave(s, D // GROUPS[fmt], dim=-1)


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "attn":
        return _exact_attn(case, st)
    got = {}
    counts, firsts = st["count"].tolist(), st["first"].tolist()
    for name in ("k", "v"):
        out = st[name + "_out"].double()
        scales = st[name + "_scale"].double() if case["op"] == "store" else None
        for b, (n, first) in enumerate(zip(counts, firsts)):
            if case["op"] == "store":
                code, s = _exact_code(st[name + "_in"][b, :n], case["fmt"])
                out[b, :n] = (code * s).flatten(-2)
                scales[b, :, first:first + n] = s.squeeze(-1).transpose(0, 1)
            else:
                out[b, :n] = _exact_values(st, name, b, first + n)[:, first:].transpose(0, 1)
        got[name + "_out"] = out
        if scales is not None:
            got[name + "_scale"] = scales
    return got


def _exact_attn(case, st):
    b, h_q, h, fmt = case["batch"], case["h_q"], case["h_kv"], case["fmt"]
    g = h_q // h
    out = torch.zeros((b, h_q, D), dtype=torch.float64, device="cuda")
    lse = torch.full((b, h_q), -math.inf, dtype=torch.float64, device="cuda")
    pre = {}
    for i, n in enumerate(_lens(case).tolist()):
        k, v = _exact_values(st, "k", i, n), _exact_values(st, "v", i, n)
        if case["append"]:
            if fmt == "bf16":
                kn, vn = st["k_new"][i].double(), st["v_new"][i].double()
            else:
                kn, vn = ((c * s).flatten(-2) for c, s in (_exact_code(st[x][i], fmt) for x in ("k_new", "v_new")))
            k, v = torch.cat((k, kn[:, None]), 1), torch.cat((v, vn[:, None]), 1)
        q = st["q"][i].double().view(h, g, D)
        z = torch.einsum("hgd,htd->hgt", q, k) / math.sqrt(D)
        if case["prefixes"]:
            p = i // (b // case["prefixes"])
            if p not in pre:
                pre = {p: (st["k_prefix"][p, :, :st["prefix_lens"][p]].double(), st["v_prefix"][p, :, :st["prefix_lens"][p]].double())}
            zp = torch.einsum("hgd,htd->hgt", q, pre[p][0]) / math.sqrt(D)
        else:
            zp = z[..., :0]
        if z.shape[-1] + zp.shape[-1] == 0:
            continue
        l = torch.logsumexp(torch.cat((z, zp), -1), -1, keepdim=True)
        o = torch.einsum("hgt,htd->hgd", torch.exp(z - l), v)
        if case["prefixes"]:
            o = o + torch.einsum("hgt,htd->hgd", torch.exp(zp - l), pre[p][1])
        out[i], lse[i] = o.reshape(h_q, D), l.reshape(h_q)
    got = {"out": out, "lse": lse}
    if case["append"]:
        got |= {name: None for name in ("k", "v", "k_scale", "v_scale") if st[name] is not None and not (fmt == "int4" and "scale" not in name)}
    return got
