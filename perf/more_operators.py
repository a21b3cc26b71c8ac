"""Paged key/value caches and rotary positions as they are measured: rotating q and k, appending rows to a paged cache with the
rotation on the way, and decode attention over the pages.

Rotation: a head's first ``rot`` elements are taken as pairs, (i, i + rot/2) or, interleaved, (2i, 2i + 1). Pair i of a token at
position p turns by p times the pair's frequency, and is multiplied by a factor (1 except for some long-context scalings).
Elements behind the first ``rot`` stay as they are. The gradient of the rotation is the same with the angle's sign changed.

A paged cache holds the K and V rows of one layer in pages of ``page`` rows a head, ``[pages][kv heads][page][128]`` (or, token
by token, ``[pages][page][kv heads][128]``); row r of sequence i is row r % page of page ``table[i][r // page]``. Rows are bf16 or
codes with bf16 scales:

  e4m3   8-bit floats, one power-of-two scale a row: the smallest 2^e with max|x| / 2^e <= 448
  int8   whole numbers -127..127, one scale a row: bf16(max|x| / 127)
  int4   whole numbers -7..7 (stored + 8 in a nibble), one scale for each 32 elements: bf16(max|x| / 7)

A scale is at least 2^-126; a code is the element over its scale, rounded to the nearest, ties to even. The four elements
32g + 4q .. 32g + 4q + 3 of an int4 row are the nibbles, lowest first, of its 16-bit word 4q + g. What is rotated on the way into
the pages or the attention is rounded to bf16, as the rotation by itself would leave it: keys are coded, and queries attend, as
they are then.

Where ``own`` is false, ``run`` computes the operators with elementary torch operations in 32 bits (angles in 64); where it is
true it makes the calls of the package.
"""
import math

import numpy as np
import torch

own = False

D = 128
FORMATS = ("bf16", "e4m3", "int8", "int4")
GROUPS = {"bf16": 0, "e4m3": 1, "int8": 1, "int4": 4}             # scales a row
ROW_BYTES = {"bf16": 256, "e4m3": 130, "int8": 130, "int4": 72}   # codes and scales of a row
CODE = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8, "int4": torch.uint8}
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
# query heads / KV heads of the 7B shape, the eviction sweep, the 32B shape and the smallest test configuration
HEADS = ((28, 4), (32, 8), (64, 8), (8, 2))
SCALINGS = ("none", "linear", "ntk", "wavelength", "yarn")


# ------------------------------------------------------------------------------------------------ the cases
def listed():
    def rotate(name, **kw):
        return {"name": name, "op": "rotate", "head": D, "rot": D, "interleaved": False, "scaling": "none", "transpose": False, "packed": True, **kw}

    def append(name, **kw):
        return {"name": name, "op": "append", "rot": D, "interleaved": False, "scaling": "none", "token_major": False, "packed": True, **kw}

    def attn(name, **kw):
        return {"name": name, "op": "attn", "rot": D, "interleaved": False, "scaling": "none", "token_major": False, "append": True, "packed": True, **kw}

    return [
        # q and k of one decode step of the 7B batch, as they lie in the output of a fused projection
        rotate("rotate, decode step", type="bf16", batch=32, tokens=1, h_q=28, h_kv=4, far=4096),
        # a prompt of odd length, far out in a scaled context
        rotate("rotate, prompt", type="bf16", batch=1, tokens=4097, h_q=64, h_kv=8, scaling="yarn", far=131072),
        # half of each head, neighbours as pairs, in 32 bits: a batch that is trained on
        rotate("rotate, half a head", type="fp32", batch=4, tokens=4096, h_q=32, h_kv=8, rot=64, interleaved=True, packed=False, far=4096),
        # the gradients of q and k that come back to the same batch
        rotate("rotate, gradient", type="bf16", batch=8, tokens=8192, h_q=28, h_kv=4, transpose=True, packed=False, far=8192),
        # one decode step of the 7B batch: a row a sequence
        append("append one token", fmt="e4m3", batch=32, h_q=28, h_kv=4, page=16, tokens=1, least=1, longest=1151),
        # a batch of prompts of different lengths; the quantised rows are read back as well
        append("append ragged prompts", fmt="int8", batch=8, h_q=28, h_kv=4, page=64, tokens=4097, least=129, longest=4224, scaling="wavelength"),
        # long prompts
        append("append long prompts", fmt="bf16", batch=4, h_q=32, h_kv=8, page=16, tokens=32768, least=32768, longest=32768, packed=False),
        # decode steps: one sequence (latency), the 7B batch with pages that end inside a tile, the 32B batch, few sequences at a
        # very long context, and a batch in which lengths differ a hundredfold
        attn("attention, one sequence", fmt="bf16", batch=1, h_q=28, h_kv=4, page=16, longest=639, least=639),
        attn("attention, 7B batch", fmt="e4m3", batch=32, h_q=28, h_kv=4, page=24, longest=1151, least=1, interleaved=True),
        attn("attention, 32B batch", fmt="bf16", batch=128, h_q=64, h_kv=8, page=64, longest=2303, least=2048),
        attn("attention, long context", fmt="int4", batch=2, h_q=32, h_kv=8, page=256, longest=131071, least=100003, append=False, scaling="yarn"),
        attn("attention, lengths apart", fmt="bf16", batch=16, h_q=28, h_kv=4, page=32, longest=65535, least=300, token_major=True, scaling="linear"),
    ]


def _between(rng, lo, hi):
    """A whole number of lo..hi, spread over its logarithm."""
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(("rotate", "append", "append", "attn", "attn", "attn"))
    h_q, h_kv = rng.choice(HEADS)
    case = {"op": op, "h_q": h_q, "h_kv": h_kv, "interleaved": rng.random() < 0.4, "scaling": rng.choice(SCALINGS), "packed": rng.random() < 0.6}
    if op == "rotate":
        head = rng.choice((64, 80, 128, 128, 256))
        most = 8 * 8192 * 32 * D // ((h_q + h_kv) * head)        # elements of the largest listed one
        case |= {"type": rng.choice(("bf16", "bf16", "fp16", "fp32")), "head": head, "rot": rng.choice((head, head // 2, head // 4)),
                 "batch": _between(rng, 1, 64), "transpose": rng.random() < 0.3, "far": rng.choice((4096, 131072, 1 << 20))}
        case["tokens"] = _between(rng, 1, most // case["batch"] // (2 if case["type"] == "fp32" else 1))
        return case
    case |= {"rot": rng.choice((D, D, 64, 32)), "token_major": rng.random() < 0.3, "page": rng.choice((16, 16, 32, 64, 128, 256, 1, 5, 24))}
    if op == "append":
        case |= {"fmt": rng.choice(FORMATS), "batch": _between(rng, 1, 64)}
        case["tokens"] = _between(rng, 1, min(32768, 4 * 32768 * 8 // 2 // (case["batch"] * h_kv)))
        case["least"] = rng.choice((case["tokens"], _between(rng, 1, case["tokens"])))
        case["longest"] = case["tokens"] + rng.choice((0, 1, 127))
        return case
    fmt = rng.choice(FORMATS)
    case |= {"fmt": fmt, "batch": _between(rng, 1, 128), "append": rng.random() < 0.7}
    if fmt in ("int8", "int4") and case["append"]:
        case["rot"] = 0      # whole-number codes of rotated keys may come out next to each other: those rows come as they are
    longest = _between(rng, 1, min(131071, 128 * 8 * 2303 // (case["batch"] * h_kv)))
    return case | {"longest": longest, "least": rng.choice((longest, rng.randint(0, longest)))}


def _lengths(least, most, n, at):
    """n lengths of least..most, the longest among them, the same ones for every seed."""
    got = np.random.RandomState(1000 * n + at).randint(least, most + 1, n)
    got[(7 * at) % n] = most
    return got.astype(np.int64)


def _counts(case):
    return _lengths(case["least"], case["tokens"], case["batch"], case["tokens"] % 97)


def _lens(case):
    if case["op"] == "append":
        return np.full(case["batch"], case["longest"])
    return _lengths(case["least"], case["longest"], case["batch"], case["longest"] % 89)


def work(case):
    if case["op"] == "rotate":
        n = case["batch"] * case["tokens"] * (case["h_q"] + case["h_kv"])
        return {"bytes": 2 * n * case["head"] * (4 if case["type"] == "fp32" else 2) + 4 * case["batch"] * case["tokens"], "flops": 3 * n * case["rot"]}
    row, heads = ROW_BYTES[case["fmt"]], case["h_kv"]
    if case["op"] == "append":
        rows = 2 * int(_counts(case).sum()) * heads
        back = 2 if case["fmt"] in ("int8", "int4") else 1       # these are read back as well
        return {"bytes": back * rows * (2 * D + row), "flops": rows * (2 * D + 3 * case["rot"] // 2)}
    new = 1 if case["append"] else 0
    rows = int(_lens(case).sum())
    b = 2 * heads * rows * row + new * 2 * heads * case["batch"] * (2 * D + row) + case["batch"] * case["h_q"] * (2 * 2 * D + 4)
    return {"bytes": b + 4 * rows // case["page"], "flops": 4 * D * (rows + new * case["batch"]) * case["h_q"]}


# ------------------------------------------------------------------------------------------------ frequencies
def frequencies(rot, scaling):
    """(radians a position of the rot/2 pairs, in 64 bits; factor of cos and sin), from the published definitions, for a
    context eight times the 4096 positions that the base 10000 was made for."""
    theta, factor, original = 1e4, 8.0, 4096.0
    f = theta ** (-np.arange(0, rot, 2, dtype=np.float64) / max(rot, 1))
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "ntk":
        return (theta * factor ** (rot / max(rot - 2, 1))) ** (-np.arange(0, rot, 2, dtype=np.float64) / max(rot, 1)), 1.0
    if scaling == "wavelength":      # long waves are stretched, short ones stay, between 1 and 4 turns in the original context it is blended
        turns = original * f / (2 * np.pi)
        keep = np.clip((turns - 1.0) / (4.0 - 1.0), 0, 1)
        return keep * f + (1 - keep) * f / factor, 1.0
    if scaling == "yarn":            # the blend runs over the pairs' numbers, between 32 turns and 1
        at = lambda turns: rot * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(theta))  # noqa: E731
        low, high = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), rot - 1)
        stretch = np.clip((np.arange(rot // 2) - low) / max(high - low, 0.001), 0, 1)
        return f * (1 - stretch) + f / factor * stretch, 0.1 * math.log(factor) + 1.0
    return f, 1.0


# ------------------------------------------------------------------------------------------------ the rows' arithmetic
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


def _decode(c, s, fmt):
    """The values that codes and scales stand for, in fp32."""
    if fmt == "bf16":
        return c.float()
    if fmt == "int4":
        c = torch.stack((c & 15, c >> 4), -1).flatten(-2).unflatten(-1, (8, 4, 4)).transpose(-3, -2).flatten(-3)
        c = c.float() - 8
    return (c.float().unflatten(-1, (GROUPS[fmt], -1)) * s.float().unsqueeze(-1)).flatten(-2)


# ------------------------------------------------------------------------------------------------ inputs
def _rand(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)


def _keys(gen, *shape):
    """Keys as they come out of a projection: a few channels are much larger than the others."""
    channel = torch.exp(0.5 * _rand(gen, D))
    return (_rand(gen, *shape, D) * channel).to(torch.bfloat16)


def _qkv(gen, case, *tokens):
    """q, k, v [..., heads, 128] in bf16: slices of one tensor, as a fused projection leaves them, or tensors of their own."""
    h_q, h = case["h_q"], case["h_kv"]
    if case["packed"]:
        qkv = torch.randn((*tokens, h_q + 2 * h, D), generator=gen, device="cuda", dtype=torch.bfloat16)
        qkv[..., h_q:h_q + h, :] *= torch.exp(0.5 * _rand(gen, D))
        return qkv[..., :h_q, :], qkv[..., h_q:h_q + h, :], qkv[..., h_q + h:, :]
    return _rand(gen, *tokens, h_q, D).to(torch.bfloat16), _keys(gen, *tokens, h), _rand(gen, *tokens, h, D).to(torch.bfloat16)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    b, h_q, h = case["batch"], case["h_q"], case["h_kv"]
    st = {"case": case}
    freq, st["factor"] = frequencies(case["rot"], case["scaling"])
    st["freq_host"], st["freq"] = freq, torch.from_numpy(freq).cuda()
    if case["op"] == "rotate":
        n, d, dtype = case["tokens"], case["head"], TYPES[case["type"]]
        if case["packed"]:
            qkv = torch.randn((b, n, h_q + 2 * h, d), generator=gen, device="cuda", dtype=dtype)
            st["q"], st["k"] = qkv[:, :, :h_q], qkv[:, :, h_q:h_q + h]
        else:
            st["q"], st["k"] = _rand(gen, b, n, h_q, d).to(dtype), _rand(gen, b, n, h, d).to(dtype)
        st["q_out"], st["k_out"] = (torch.zeros((b, n, heads, d), dtype=dtype, device="cuda") for heads in (h_q, h))
        start = torch.randint(0, max(1, case["far"] - n), (b, 1), generator=gen, device="cuda", dtype=torch.int32)
        st["pos"] = start + torch.arange(n, device="cuda", dtype=torch.int32)
        return st
    # the pool: every sequence has the pages that it needs, in no order; places that it does not need yet hold -1
    page, lens = case["page"], _lens(case)
    need = [-(-(int(n) + (1 if case["op"] == "attn" and case["append"] else 0)) // page) for n in lens]
    pages, width = sum(need) + 3, max(max(need), 1)
    order = np.random.RandomState(int(seed) % (1 << 31)).permutation(pages)
    table, at = np.full((b, width), -1, np.int32), 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    st["table"] = torch.from_numpy(table).cuda()
    fmt = case["fmt"]
    shape = (pages, page, h) if case["token_major"] else (pages, h, page)
    if case["op"] == "append":
        for name in ("k", "v"):
            st[name] = torch.zeros((*shape, 64 if fmt == "int4" else D), dtype=torch.uint8 if fmt != "bf16" else torch.bfloat16, device="cuda").view(CODE[fmt])
            st[name + "_scale"] = torch.zeros((*shape, GROUPS[fmt]), dtype=torch.bfloat16, device="cuda") if GROUPS[fmt] else None
        n, counts = case["tokens"], _counts(case)
        _, st["k_in"], st["v_in"] = _qkv(gen, case, b, n)
        st["count"] = torch.from_numpy(counts).to("cuda", torch.int32)
        st["first"] = torch.from_numpy((case["longest"] - counts) * 7 // 8).to("cuda", torch.int32)   # behind the rows that are there
        if fmt in ("int8", "int4"):
            st["k_out"], st["v_out"] = (torch.zeros((b, n, h, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        return st
    for name in ("k", "v"):      # pages that have all been written, made in pieces to save memory
        made = [_encode(_keys(gen, *x) if name == "k" else _rand(gen, *x, D).to(torch.bfloat16), fmt)
                for x in ((min(4096, pages - i), *shape[1:]) for i in range(0, pages, 4096))]
        st[name] = torch.cat([m[0].view(torch.uint8) if fmt == "e4m3" else m[0] for m in made]).view(CODE[fmt])
        st[name + "_scale"] = torch.cat([m[1] for m in made]) if GROUPS[fmt] else None
    st["length"] = torch.from_numpy(lens).to("cuda", torch.int32)
    st["q"], k_new, v_new = _qkv(gen, case, b)
    st["k_new"], st["v_new"] = (k_new, v_new) if case["append"] else (None, None)
    st["out"] = torch.zeros((b, h_q, D), dtype=torch.bfloat16, device="cuda")
    st["lse"] = torch.zeros((b, h_q), dtype=torch.float32, device="cuda")
    return st


# ------------------------------------------------------------------------------------------------ one pass
def _rotated(st, x, pos, transpose=False):
    """x [..., heads, dims] with pos [...], in fp32."""
    rot, x = st["case"]["rot"], x.float()
    if rot == 0:
        return x
    angle = (pos.double()[..., None] * st["freq"])[..., None, :]
    c, s = (torch.cos(angle) * st["factor"]).float(), (torch.sin(angle) * st["factor"]).float()
    s = -s if transpose else s
    if st["case"]["interleaved"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack((a * c - b * s, b * c + a * s), -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat((a * c - b * s, b * c + a * s), -1)
    return torch.cat((y, x[..., rot:]), -1)


def _bytes(x):
    return x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x


def _token_first(st, t):
    """Pages [pages][page][kv heads][...] whatever the order that they are kept in."""
    return t if st["case"]["token_major"] else t.transpose(1, 2)


def _put(st, x, name, row, here=None):
    """Codes and scales of x [batch][tokens][kv heads][128] into rows `row` [batch][tokens], where `here` says so."""
    page = st["case"]["page"]
    codes, scale = _encode(x, st["case"]["fmt"])
    at = torch.arange(len(row), device="cuda")[:, None].expand_as(row)
    if here is not None:
        at, row, codes, scale = at[here], row[here], _bytes(codes)[here], None if scale is None else scale[here]
    number = st["table"].long()[at, row // page]
    _token_first(st, _bytes(st[name]))[number, row % page] = _bytes(codes)
    if scale is not None:
        _token_first(st, st[name + "_scale"])[number, row % page] = scale


def _plain_append(st):
    case = st["case"]
    t = torch.arange(case["tokens"], device="cuda")
    row = st["first"].long()[:, None] + t
    here = None if case["least"] == case["tokens"] else t < st["count"].long()[:, None]
    _put(st, _rotated(st, st["k_in"], row).to(torch.bfloat16), "k", row, here)
    _put(st, st["v_in"], "v", row, here)
    if case["fmt"] not in ("int8", "int4"):
        return
    page, row = case["page"], row.clamp(max=case["longest"] - 1)
    number = st["table"].long()[torch.arange(len(row), device="cuda")[:, None], row // page]

    def back(name):
        c, s = (_token_first(st, st[n])[number, row % page] for n in (name, name + "_scale"))
        x = _decode(c, s, case["fmt"]).to(torch.bfloat16)
        out = st[name + "_out"]
        out.copy_(x if here is None else torch.where(here[:, :, None, None], x, out))

    back("k")
    back("v")


def _plain_attn(st):
    case = st["case"]
    b, h_q, h, fmt, page = case["batch"], case["h_q"], case["h_kv"], case["fmt"], case["page"]
    n = st["length"].long()
    pos = n if case["append"] else n - 1
    q = _rotated(st, st["q"], pos).to(torch.bfloat16).float()
    if case["append"]:
        _put(st, _rotated(st, st["k_new"], n).to(torch.bfloat16)[:, None], "k", n[:, None])
        _put(st, st["v_new"][:, None], "v", n[:, None])
        n = n + 1
    number = st["table"].long().clamp(min=0)
    most = number.shape[1] * page

    def values(name):      # [batch][kv heads][rows][128]
        c = _token_first(st, _bytes(st[name]))[number].flatten(1, 2).transpose(1, 2).view(CODE[fmt])
        s = st[name + "_scale"]
        return _decode(c, None if s is None else _token_first(st, s)[number].flatten(1, 2).transpose(1, 2), fmt)

    z = (q.reshape(b, h, h_q // h, D) @ values("k").transpose(-1, -2)) / math.sqrt(D)
    z = z.masked_fill((torch.arange(most, device="cuda") >= n[:, None])[:, None, None, :], -math.inf)
    m = z.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)      # nothing to attend to: out = 0, lse = -inf
    w = torch.exp(z - m)
    total = w.sum(-1, keepdim=True)
    o = w @ values("v")
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    st["out"].copy_(o.view(b, h_q, D))
    st["lse"].copy_((m + torch.log(total)).view(b, h_q))


def _handles(st):
    """The handles that a program keeps over its buffers; made at the first pass."""
    if "rotary" not in st:
        import paper_2512_00504_b200 as gkv
        case = st["case"]
        st["rotary"] = gkv.Rotary(st["freq_host"], head_dim=case.get("head", D), interleaved=case["interleaved"], factor=st["factor"],
                                  device="cuda") if case["rot"] else None
        if case["op"] != "rotate":
            buffers = [st[n] for n in ("k", "v", "k_scale", "v_scale") if st[n] is not None]
            st["store"] = gkv.PagedStore(case["fmt"], pages=len(st["k"]), page_size=case["page"], h_q=case["h_q"], h_kv=case["h_kv"],
                                         token_major=case["token_major"], buffers=buffers, max_batch=case["batch"])
    return st["rotary"], st.get("store")


def run(state):
    st, case = state, state["case"]
    if own:
        rotary, store = _handles(st)
    if case["op"] == "rotate":
        if own:
            rotary.apply(st["pos"], st["q"], st["k"], q_out=st["q_out"], k_out=st["k_out"], transpose=case["transpose"])
        else:
            st["q_out"].copy_(_rotated(st, st["q"], st["pos"], case["transpose"]))
            st["k_out"].copy_(_rotated(st, st["k"], st["pos"], case["transpose"]))
        return {"q_out": st["q_out"], "k_out": st["k_out"]}
    scales = {n: st[n] for n in ("k_scale", "v_scale") if st[n] is not None}
    if case["op"] == "append":
        if own:
            store.append(st["table"], st["k_in"], st["v_in"], first=st["first"], count=st["count"], rotary=rotary)
            if case["fmt"] in ("int8", "int4"):
                store.read(st["table"], st["k_out"], st["v_out"], first=st["first"], count=st["count"])
        else:
            _plain_append(st)
        # whole-number codes come as the values that they stand for
        return {n: st[n + "_out" if case["fmt"] in ("int8", "int4") else n] for n in ("k", "v")} | scales
    if own:
        store.attn(st["table"], st["length"], st["q"], st["out"], k_new=st["k_new"], v_new=st["v_new"], rotary=rotary, lse=st["lse"],
                   max_len=case["longest"])
    else:
        _plain_attn(st)
    got = {"out": st["out"], "lse": st["lse"]}
    if case["append"]:   # the pages with their new rows
        got |= scales | ({} if case["fmt"] == "int4" else {n: st[n] for n in ("k", "v")})
    return got


# ------------------------------------------------------------------------------------------------ in 64 bits
def _turn(case, freq, factor, x, pos, sign=1.0):
    """fp64 rows [tokens][heads][dims] turned, from the definition of a pair as a complex number."""
    x, rot = x.double().clone(), case["rot"]
    if rot == 0:
        return x
    first = torch.arange(rot // 2, device=x.device) * (2 if case["interleaved"] else 1)
    second = first + (1 if case["interleaved"] else rot // 2)
    z = torch.complex(x[..., first], x[..., second])
    z = z * torch.polar(torch.full((), factor, dtype=torch.float64, device=x.device), sign * pos.double()[:, None, None] * freq)
    x[..., first], x[..., second] = z.real, z.imag
    return x


def _exact_code(x, fmt):
    """(codes as fp64 numbers, scales as fp64 numbers) of rows, from the definition."""
    if fmt == "bf16":
        return x.double(), None
    x = x.double().unflatten(-1, (GROUPS[fmt], -1))
    a = x.abs().amax(-1, keepdim=True)
    least = 2.0 ** -126
    if fmt == "e4m3":
        s = torch.exp2(torch.ceil(torch.log2((a / 448).clamp(min=least))))
        y = x / s
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)      # spacing of 8-bit floats
        return (torch.round(y / step) * step).flatten(-2), s.squeeze(-1)
    s = (a / (127 if fmt == "int8" else 7)).to(torch.bfloat16).double().clamp(min=least)
    return torch.round(x / s).flatten(-2), s.squeeze(-1)


def _times(code, s, fmt):
    return code if s is None else code * torch.repeat_interleave(s, D // GROUPS[fmt], dim=-1)


def _exact_rows(st, name, i, rows):
    """fp64 values [kv heads][rows][128] of sequence i's first rows, page by page's definition."""
    case, fmt = st["case"], st["case"]["fmt"]
    r = torch.arange(rows, device="cuda")
    number, slot = st["table"][i, r // case["page"]].long(), r % case["page"]
    pick = (lambda t: t[number, slot]) if case["token_major"] else (lambda t: t[number, :, slot])
    c = pick(st[name].view(torch.uint8)).view(CODE[fmt]) if fmt == "e4m3" else pick(st[name])
    if fmt == "int4":
        e = torch.arange(D, device="cuda")
        g, q, k = e // 32, (e % 32) // 4, e % 4
        x = ((c[..., 8 * q + 2 * g + k // 2].long() >> (4 * (k % 2))) & 15).double() - 8
    else:
        x = c.double()
    return _times(x, pick(st[name + "_scale"]).double() if GROUPS[fmt] else None, fmt).transpose(0, 1)


def exact(case, seed):
    st = prepare(case, seed)
    freq, factor = (torch.from_numpy(x).cuda() if isinstance(x, np.ndarray) else x for x in frequencies(case["rot"], case["scaling"]))
    if case["op"] == "rotate":
        sign = -1.0 if case["transpose"] else 1.0
        return {n + "_out": torch.stack([_turn(case, freq, factor, x, p, sign) for x, p in zip(st[n], st["pos"])]) for n in ("q", "k")}
    fmt, page = case["fmt"], case["page"]
    if case["op"] == "append":
        whole = fmt in ("int8", "int4")
        got = {n: st[n + "_out"].double() if whole else st[n].double() for n in ("k", "v")}
        got |= {n: st[n].double() for n in ("k_scale", "v_scale") if st[n] is not None}
        for i, (n, first) in enumerate(zip(_counts(case).tolist(), st["first"].tolist())):
            r = first + torch.arange(n, device="cuda")
            number, slot = st["table"][i, r // page].long(), r % page
            at = (number, slot) if case["token_major"] else (number, slice(None), slot)
            for name in ("k", "v"):
                x = st[name + "_in"][i, :n]
                x = _turn(case, freq, factor, x, r).to(torch.bfloat16) if name == "k" else x
                code, s = _exact_code(x, fmt)
                if whole:
                    got[name][i, :n] = _times(code, s, fmt)
                else:
                    got[name][at] = code
                if s is not None:
                    got[name + "_scale"][at] = s
        return got
    b, h_q, h = case["batch"], case["h_q"], case["h_kv"]
    out = torch.zeros((b, h_q, D), dtype=torch.float64, device="cuda")
    lse = torch.full((b, h_q), -math.inf, dtype=torch.float64, device="cuda")
    for i, n in enumerate(_lens(case).tolist()):
        k, v = _exact_rows(st, "k", i, n), _exact_rows(st, "v", i, n)
        pos = torch.tensor([n if case["append"] else n - 1], device="cuda")
        q = _turn(case, freq, factor, st["q"][i][None], pos)[0].to(torch.bfloat16).double()
        if case["append"]:
            new = (_turn(case, freq, factor, st["k_new"][i][None], pos)[0].to(torch.bfloat16), st["v_new"][i])
            kn, vn = (_times(*_exact_code(x, fmt), fmt) for x in new)
            k, v = torch.cat((k, kn[:, None]), 1), torch.cat((v, vn[:, None]), 1)
        if k.shape[1] == 0:
            continue
        z = torch.einsum("hgd,htd->hgt", q.view(h, h_q // h, D), k) / math.sqrt(D)
        l = torch.logsumexp(z, -1, keepdim=True)
        out[i], lse[i] = torch.einsum("hgt,htd->hgd", torch.exp(z - l), v).reshape(h_q, D), l.reshape(h_q)
    got = {"out": out, "lse": lse}
    if case["append"]:
        got |= {n: None for n in ("k_scale", "v_scale") if st[n] is not None} | ({} if fmt == "int4" else {"k": None, "v": None})
    return got
