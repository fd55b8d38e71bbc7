"""Performance cases of the paged key/value cache: appending new tokens (with the position rotation), attention over the
cache and reading rows back.

Every case is one pass through one of these, on inputs that are resident on the GPU.  A cache is a pool of pages of
``page`` tokens; sequence b's token i lies in page ``table[b, i // page]``.  Head layouts and lengths are those of the
repository's workloads (32 query / 8 KV heads, d = 128; a few heads in fp32), or generic.

A case is a dict of plain values:
  kind    "append" (kv_append, and for a 4-bit cache kv_read of the rows that it wrote) | "read" (kv_read) | "attn" (kv_attn)
  dtype   "bf16" | "fp32": new tokens, outputs, and the cache where fmt is "plain"
  fmt     "plain" | "fp4": 4-bit codes with one power-of-two scale for 32 channels
  lens    tokens of each sequence in the cache, the new ones included, comma separated
  new     new tokens of each sequence; one number for all: a batch [B, H, n, d], else packed [H, total, d]
  Hq, Hkv, d, page
  rot     rotated channels, pairs   "half" (i, i + rot/2) | "even" (2i, 2i + 1),   base of the frequencies
  layout  "head" (q, k, v one head after the other) | "token" (one fused projection row [Hq + 2 Hkv, d] a token)
"""
import math

import torch

own = False


def _case(name, kind, lens, new, **kw):
    c = dict(name=name, kind=kind, dtype="bf16", fmt="plain", lens=lens, new=new, Hq=32, Hkv=8, d=128, page=64, rot=128,
             pairs="half", base=500000.0, layout="token")
    c.update(kw)
    return c


# lengths of serving batches: prompts and conversations of mixed length, most of them short
_BATCH32 = ",".join(str(200 + (i * i * 37) % 15877) for i in range(32))
_BATCH64 = ",".join(str(33 + (i * 2371) % 16384) for i in range(64))


def listed():
    return [
        # one sequence decodes one token: a launch's latency
        _case("append_one", "append", "8192", "1"),
        # a packed batch of prompts before their prefill: rotated q and k, and the pages
        _case("append_prompts", "append", "911,4097,16384,30001", "911,4097,16384,30001"),
        # a step of a batch of 64 conversations into a 4-bit cache
        _case("append_fp4_step", "append", _BATCH64, "1", fmt="fp4"),
        # a long document's chunk into a 4-bit cache, read back for the prefill that follows
        _case("append_fp4_chunk", "append", "30011", "16384", fmt="fp4", page=128),
        # one fp32 shard of few heads, neighbouring pairs, part of the channels rotated
        _case("append_fp32", "append", "4000,1777", "1500", dtype="fp32", Hq=8, Hkv=2, d=64, rot=32, pairs="even", page=16,
              layout="head", base=10000.0),
        # a cached prefix is read back from 4 bits
        _case("read_fp4", "read", "16384,9001", "9001", fmt="fp4"),
        # a short chat, one token: latency
        _case("attn_one_1k", "attn", "1000", "1"),
        # the 128k context, one token: few rows, one long axis
        _case("attn_one_128k", "attn", "131072", "1"),
        # a serving batch of 32 with mixed lengths
        _case("attn_batch", "attn", _BATCH32, "1", page=16),
        # the batch of 64 over a 4-bit cache
        _case("attn_fp4_batch", "attn", _BATCH64, "1", fmt="fp4"),
        # chunks of two prompts over what is cached of them, packed, from 4 bits
        _case("attn_fp4_chunk", "attn", "16384,5003", "1024,403", fmt="fp4"),
        # the largest: the next chunk of a long document over a plain cache
        _case("attn_chunk", "attn", "30011,8192", "2048,1000"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append"] * 3 + ["read"] + ["attn"] * 6)
    fmt = rng.choice(["plain", "fp4"])
    kw = dict(fmt=fmt, page=rng.choice([16, 32, 64, 128, 256]), layout=rng.choice(["head", "token"]))
    kw["Hq"], kw["Hkv"] = rng.choice([(32, 8), (32, 8), (16, 2), (8, 8), (12, 4), (32, 2)])
    kw["d"] = rng.choice([128, 128, 64])
    if fmt == "plain" and rng.random() < 0.3:
        kw.update(dtype="fp32", d=rng.choice([32, 64, 128]), Hq=8, Hkv=rng.choice([1, 2, 8]))
    kw["rot"] = rng.choice([kw["d"], kw["d"], kw["d"] // 2])
    kw["pairs"] = rng.choice(["half", "half", "even"])
    kw["base"] = rng.choice([10000.0, 500000.0])
    small = 4 if kw.get("dtype") == "fp32" else 1
    if kind == "attn":
        shape = rng.choice(["one", "few", "chunk"])
        if shape == "chunk":
            lens = [_log_int(rng, 600, 16000 // small) for _ in range(rng.choice([1, 2]))]
            new = [min(n, _log_int(rng, 20, 1500 // small)) for n in lens]
        else:
            B = _log_int(rng, 1, 64)
            lens = [_log_int(rng, 30, 200000 // small // max(B, 4)) for _ in range(B)]
            new = [1 if shape == "one" else min(rng.choice([2, 3, 5, 8]), min(lens))]
    elif rng.random() < 0.4:
        B = _log_int(rng, 1, 64)
        lens, new = [_log_int(rng, 30, 8000 // small) for _ in range(B)], [1]
    else:
        lens = [_log_int(rng, 100, 16000 // small) for _ in range(rng.choice([1, 2, 4]))]
        new = [max(1, int(n * rng.uniform(0.1, 1.0))) for n in lens]
    if rng.random() < 0.5 and len(set(new)) > 1:
        new = [min(new)]
    c = _case("", kind, ",".join(map(str, lens)), ",".join(map(str, new)), **kw)
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs
def _lens(c):
    return [int(x) for x in c["lens"].split(",")]


def _new(c):
    n = [int(x) for x in c["new"].split(",")]
    return n * (len(_lens(c)) if len(n) == 1 else 1)


def _packed(c):
    return "," in c["new"]


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _pool(c, pages, gen):
    """One pool of pages with values in it: rows of the type, or (codes, scales)."""
    H, d, page = c["Hkv"], c["d"], c["page"]
    if c["fmt"] == "plain":
        return torch.randn(pages, H, page, d, device="cuda", generator=gen, dtype=_dtype(c)), None
    codes = torch.randint(0, 256, (pages, H, page, d // 2), device="cuda", generator=gen, dtype=torch.uint8)
    scales = torch.randint(124, 128, (pages, H, d // 32, page), device="cuda", generator=gen, dtype=torch.uint8)
    return codes, scales


def _inputs(c, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    lens, new, page, d = _lens(c), _new(c), c["page"], c["d"]
    B, T = len(lens), sum(new)
    per = [-(-n // page) for n in lens]
    pages = sum(per) + 3
    order = torch.randperm(pages, device="cuda", generator=gen).to(torch.int32)
    table = torch.zeros(B, max(per), device="cuda", dtype=torch.int32)
    at = 0
    for b, n in enumerate(per):
        table[b, :n] = order[at:at + n]
        at += n
    s = dict(case=c, table=table, kv_len=torch.tensor(lens, device="cuda", dtype=torch.int32), T=T)
    s["kc"], s["ks"] = _pool(c, pages, gen)
    s["vc"], s["vs"] = _pool(c, pages, gen)
    ends = [0]
    for n in new:
        ends.append(ends[-1] + n)
    s["cu"] = torch.tensor(ends, device="cuda", dtype=torch.int32)
    if c["kind"] == "read":
        return s
    Hq, Hkv = c["Hq"], c["Hkv"]
    if c["kind"] == "attn":
        x = torch.randn(T, Hq, d, device="cuda", generator=gen).to(_dtype(c))
        s["q"] = x.transpose(0, 1) if c["layout"] == "token" else x.transpose(0, 1).contiguous()
    else:
        x = torch.randn(T, Hq + 2 * Hkv, d, device="cuda", generator=gen).to(_dtype(c))
        q, k, v = (y.transpose(0, 1) for y in x.split([Hq, Hkv, Hkv], dim=1))
        s["q"], s["k"], s["v"] = (q, k, v) if c["layout"] == "token" else (q.contiguous(), k.contiguous(), v.contiguous())
        i = torch.arange(c["rot"] // 2, dtype=torch.float64)
        s["inv_freq"] = (c["base"] ** (-2.0 * i / c["rot"])).to(torch.float32).cuda()
    if not _packed(c):          # [H, B * n, d] -> [B, H, n, d]
        for key in ("q", "k", "v"):
            if key in s:
                s[key] = s[key].unflatten(1, (B, new[0])).transpose(0, 1)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    c, new = case, _new(case)
    shape = lambda H: (H, s["T"], c["d"]) if _packed(c) else (len(new), H, new[0], c["d"])
    empty = lambda H: torch.empty(shape(H), device="cuda", dtype=_dtype(c))
    if c["kind"] == "append":
        s["q_out"], s["k_out"] = empty(c["Hq"]), empty(c["Hkv"])
    if c["kind"] == "read" or c["kind"] == "append" and c["fmt"] == "fp4":
        s["k_read"], s["v_read"] = empty(c["Hkv"]), empty(c["Hkv"])
    if c["kind"] == "attn":
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(c["Hq"] * s["T"], device="cuda", dtype=torch.float32)
    if own:                     # the call's description and workspace, which a serving loop keeps
        from paper_2505_23520_amd import api
        cache = dict(k=s["kc"], v=s["vc"], k_scale=s["ks"], v_scale=s["vs"])
        kw = dict(cu_seqlens=s["cu"] if _packed(c) else None, max_new=max(new), max_len=max(_lens(c)))
        if c["kind"] == "attn":
            s["p"] = api.make_kv_params(cache, s["table"], s["kv_len"], q=s["q"], out=s["out"], **kw)
            s["ws"] = torch.empty(api.kv_attn_workspace_bytes(s["p"]), device="cuda", dtype=torch.uint8)
        if c["kind"] == "append":
            s["p"] = api.make_kv_params(cache, s["table"], s["kv_len"], q=s["q"], k=s["k"], v=s["v"], out=s["q_out"],
                                        k_out=s["k_out"], rot_dim=c["rot"], rot_interleaved=c["pairs"] == "even", **kw)
        if "k_read" in s:
            s["p_read"] = api.make_kv_params(cache, s["table"], s["kv_len"], k=s["k_read"], v=s["v_read"], **kw)
    return s


# ------------------------------------------------------------------ one pass
def run(state):
    s = state
    c = s["case"]
    if own:
        return _run_own(s, c)
    return {"append": _plain_append, "read": _plain_read, "attn": _plain_attn}[c["kind"]](s, c)


def _run_own(s, c):
    from paper_2505_23520_amd import api
    if c["kind"] == "attn":
        api.kv_attn(s["p"], s["q"], s["out"], s["lse"], s["ws"])
        return dict(out=s["out"], lse=s["lse"])
    if c["kind"] == "append":
        api.kv_append(s["p"], s["q"], s["k"], s["v"], s["inv_freq"], None, s["q_out"], s["k_out"])
        if c["fmt"] == "plain":
            return dict(q=s["q_out"], k=s["k_out"], k_cache=s["kc"], v_cache=s["vc"])
    api.kv_read(s["p_read"], s["k_read"], s["v_read"])
    if c["kind"] == "read":
        return dict(k_cache=s["k_read"], v_cache=s["v_read"])
    return dict(q=s["q_out"], k=s["k_out"], k_cache=s["k_read"], v_cache=s["v_read"])


def _places(s, c):
    """For every new token, in packed order: its sequence, its place in the cache, and that place's page."""
    cu, n = s["cu"].long(), (s["cu"][1:] - s["cu"][:-1]).long()
    b = torch.repeat_interleave(torch.arange(n.numel(), device="cuda"), n, output_size=s["T"])
    i = torch.arange(s["T"], device="cuda") - cu[b]
    at = s["kv_len"].long()[b] - n[b] + i
    return b, i, at, s["table"].long()[b, at // c["page"]]


def _tokens(c, x):
    """[T, H, d] of a batch [B, H, n, d] or a packed [H, T, d]."""
    return x.transpose(0, 1) if _packed(c) else x.transpose(1, 2).flatten(0, 1)


def _as_laid(c, x):
    """The other way round: [T, H, d] as the case's tensors have it."""
    return x.transpose(0, 1) if _packed(c) else x.unflatten(0, (len(_lens(c)), -1)).transpose(1, 2)


def _rotate(c, x, cos, sin):
    """x [T, H, d]; cos, sin [T, 1, rot / 2] of the same type."""
    r = c["rot"]
    if c["pairs"] == "even":
        x1, x2 = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([x1 * cos - x2 * sin, x2 * cos + x1 * sin], dim=-1).flatten(-2)
    else:
        x1, x2 = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat([x1 * cos - x2 * sin, x2 * cos + x1 * sin], dim=-1)
    return torch.cat([y, x[..., r:]], dim=-1)


_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _to_fp4(x):
    """Groups of 32 channels of x [..., d] (64 bits: values next to a border) -> codes [..., d], scale bytes [..., d / 32].
    Scale: the least 2^e, -120 <= e <= 125, with max |x| <= 7 * 2^e; code: nearest, ties to the even code."""
    g = x.unflatten(-1, (-1, 32))
    top = g.abs().amax(dim=-1)
    f, e = torch.frexp(top)                 # top = f * 2^e, f in [0.5, 1): 7 * 2^(e - 3) is 0.875 * 2^e
    e = torch.where(f > 0.875, e - 2, e - 3)
    e = torch.where(top > 0, e, -120).clamp(-120, 125)
    a = g.abs() * torch.exp2(-e.double())[..., None]
    code = ((a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int() + (a > 2.5).int()
            + (a >= 3.5).int() + (a > 5.0).int())
    code = code + 8 * (g < 0).int()
    return code.flatten(-2).to(torch.uint8), (e + 127).to(torch.uint8)


def _from_fp4(codes, scales):
    """codes [..., page, d / 2], scales [..., d / 32, page] -> float32 [..., page, d]"""
    table = torch.tensor(_E2M1 + [-x for x in _E2M1], device="cuda")
    x = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2)
    scale = torch.exp2(scales.float() - 127.0).transpose(-1, -2)
    return (table[x.int()].unflatten(-1, (-1, 32)) * scale[..., None]).flatten(-2)


def _plain_append(s, c):
    b, _, at, page = _places(s, c)
    q, k, v = (_tokens(c, s[key]) for key in ("q", "k", "v"))
    angle = at.double()[:, None, None] * s["inv_freq"].double()          # positions are far: 64 bits
    cos, sin = angle.cos(), angle.sin()
    q_rot = _rotate(c, q.float(), cos.float(), sin.float()).to(_dtype(c))
    k_rot = _rotate(c, k.float(), cos.float(), sin.float()).to(_dtype(c))
    s["q_out"].copy_(_as_laid(c, q_rot))
    s["k_out"].copy_(_as_laid(c, k_rot))
    row = at % c["page"]
    if c["fmt"] == "plain":
        s["kc"][page, :, row] = k_rot
        s["vc"][page, :, row] = v
        return dict(q=s["q_out"], k=s["k_out"], k_cache=s["kc"], v_cache=s["vc"])
    for x, codes, scales, read in ((_rotate(c, k.double(), cos, sin), s["kc"], s["ks"], s["k_read"]),
                                   (v.double(), s["vc"], s["vs"], s["v_read"])):
        code, e = _to_fp4(x)
        codes[page, :, row] = code[..., 0::2] | code[..., 1::2] << 4
        scales[page, :, :, row] = e
        read.copy_(_as_laid(c, _from_fp4(codes[page, :, row][..., None, :], scales[page, :, :, row][..., None])[..., 0, :]))
    return dict(q=s["q_out"], k=s["k_out"], k_cache=s["k_read"], v_cache=s["v_read"])


def _plain_read(s, c):
    _, _, at, page = _places(s, c)
    row = at % c["page"]
    for codes, scales, read in ((s["kc"], s["ks"], s["k_read"]), (s["vc"], s["vs"], s["v_read"])):
        if c["fmt"] == "plain":
            x = codes[page, :, row]
        else:
            x = _from_fp4(codes[page, :, row][..., None, :], scales[page, :, :, row][..., None])[..., 0, :]
        read.copy_(_as_laid(c, x))
    return dict(k_cache=s["k_read"], v_cache=s["v_read"])


def _rows(s, c, codes, scales):
    """The whole cache of every sequence, padded: float32 [B, Hkv, length, d]"""
    t = s["table"].long()
    x = codes[t].float() if c["fmt"] == "plain" else _from_fp4(codes[t], scales[t])     # [B, pages, Hkv, page, d]
    return x.transpose(1, 2).flatten(2, 3)


def _plain_attn(s, c):
    b, i, _, _ = _places(s, c)
    n = (s["cu"][1:] - s["cu"][:-1]).long()
    B, most, grp, d = n.numel(), max(_new(c)), c["Hq"] // c["Hkv"], c["d"]
    K, V = _rows(s, c, s["kc"], s["ks"]), _rows(s, c, s["vc"], s["vs"])
    V = V.masked_fill((torch.arange(V.shape[2], device="cuda") >= s["kv_len"][:, None])[:, None, :, None], 0.0)
    tok = (s["cu"][:-1].long()[:, None] + torch.arange(most, device="cuda")).clamp(max=s["T"] - 1)     # [B, most]
    q = _tokens(c, s["q"])[tok].float()                                               # [B, most, Hq, d]
    q = q.unflatten(2, (c["Hkv"], grp)).permute(0, 2, 3, 1, 4).flatten(2, 3)          # [B, Hkv, grp * most, d]
    score = (q @ K.transpose(2, 3)).mul_(1.0 / math.sqrt(d))
    seen = s["kv_len"].long()[:, None] - n[:, None] + torch.arange(most, device="cuda") + 1               # [B, most]
    hide = torch.arange(K.shape[2], device="cuda") >= seen[:, :, None]                # [B, most, length]
    score.unflatten(2, (grp, most)).masked_fill_(hide[:, None, None], -math.inf)
    m = score.amax(dim=-1, keepdim=True)
    p = score.sub_(m).exp_()
    l = p.sum(dim=-1, keepdim=True)
    o = ((p @ V) / l).unflatten(2, (grp, most)).permute(0, 3, 1, 2, 4).flatten(2, 3)  # [B, most, Hq, d]
    lse = (m + l.log())[..., 0].unflatten(2, (grp, most)).permute(0, 3, 1, 2).flatten(2)
    s["out"].copy_(_as_laid(c, o[b, i].to(_dtype(c))))
    lse = lse[b, i]                                                                   # [T, Hq]
    s["lse"].copy_((lse.t() if _packed(c) else lse.unflatten(0, (B, most)).transpose(1, 2)).reshape(-1))
    return dict(out=s["out"], lse=s["lse"])


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    lens, new, d = _lens(c), _new(c), c["d"]
    T, item = sum(new), 2 if c["dtype"] == "bf16" else 4
    row = d * item if c["fmt"] == "plain" else d // 2 + d // 32          # one key or value row in the cache
    if c["kind"] == "append":
        elems = T * (c["Hq"] + 2 * c["Hkv"]) * d + T * (c["Hq"] + c["Hkv"]) * d       # q, k, v in; q, k out
        values = 2 * T * c["Hkv"] * d if c["fmt"] == "fp4" else 0                     # the rows as values
        return dict(bytes=(elems + values) * item + 2 * T * c["Hkv"] * row, flops=3 * T * (c["Hq"] + c["Hkv"]) * c["rot"])
    if c["kind"] == "read":
        return dict(bytes=2 * T * c["Hkv"] * (row + d * item), flops=T * c["Hkv"] * d)
    pairs = sum(n * m - n * (n - 1) // 2 for n, m in zip(new, lens))
    return dict(bytes=sum(lens) * c["Hkv"] * 2 * row + T * c["Hq"] * (2 * d * item + 4), flops=4 * d * c["Hq"] * pairs)


# ------------------------------------------------------------------ the same in 64 bits
def _exact_row(c, codes, scales, table, b, length):
    """[Hkv, length, d] of sequence b, float64, page by page"""
    out = torch.empty(c["Hkv"], length, c["d"], device="cuda", dtype=torch.float64)
    at = torch.arange(length, device="cuda")
    page, row = table[b].long()[at // c["page"]], at % c["page"]
    for h in range(c["Hkv"]):
        x = codes[page, h, row]
        if c["fmt"] == "plain":
            out[h] = x.double()
            continue
        for half, nibble in ((0, x & 15), (1, x >> 4)):
            e, m = (nibble >> 1) & 3, (nibble & 1).double()
            a = torch.where(e == 0, 0.5 * m, (1.0 + 0.5 * m) * torch.exp2(e.double() - 1.0))
            out[h, :, half::2] = torch.where(nibble >= 8, -a, a)
        for g in range(c["d"] // 32):
            out[h, :, 32 * g:32 * g + 32] *= torch.exp2(scales[page, h, g, row].double() - 127.0)[:, None]
    return out


def _exact_quantised(x):
    """The values that 4 bits keep of x [..., 32] in 64 bits: each against all that the group's scale offers."""
    top = x.abs().amax(dim=-1, keepdim=True)
    e = torch.ceil(torch.log2(top / 7.0)).clamp(-120, 125)
    e = torch.where(top > 7.0 * torch.exp2(e), e + 1, e)                 # log2 next to a whole number
    e = torch.where((e > -120) & (top <= 7.0 * torch.exp2(e - 1)), e - 1, e)
    scale = torch.exp2(torch.where(top > 0, e, torch.full_like(e, -120.0)))
    best, far = torch.zeros_like(x), torch.full_like(x, math.inf)
    for value in (0.0, 1.0, 2.0, 4.0, 0.5, 1.5, 3.0, 6.0):               # even codes first: they win ties
        d = (x.abs() / scale - value).abs()
        best, far = torch.where(d < far, value, best), torch.minimum(d, far)
    return torch.where(x < 0, -best, best) * scale


def exact(case, seed):
    c = case
    s = _inputs(c, seed)
    lens, new, d = _lens(c), _new(c), c["d"]
    grp = c["Hq"] // c["Hkv"]
    start, outs = 0, {}

    def part(x, b):              # [H, n, d] of sequence b
        return (x[:, start:start + new[b]] if _packed(c) else x[b]).double()

    def keep(key, x):
        outs.setdefault(key, []).append(x)

    pools = {}
    if c["kind"] == "append" and c["fmt"] == "plain":
        pools = dict(k_cache=s["kc"].double(), v_cache=s["vc"].double())
    for b, (n, m) in enumerate(zip(lens, new)):
        if c["kind"] == "attn":
            K, V = (_exact_row(c, x, y, s["table"], b, n) for x, y in ((s["kc"], s["ks"]), (s["vc"], s["vs"])))
            q = part(s["q"], b)
            o, lse = torch.empty_like(q), torch.empty(c["Hq"], m, device="cuda", dtype=torch.float64)
            hide = torch.arange(n, device="cuda") > torch.arange(n - m, n, device="cuda")[:, None]
            for h in range(c["Hq"]):
                sc = (q[h] @ K[h // grp].T / math.sqrt(d)).masked_fill(hide, -math.inf)
                lse[h] = torch.logsumexp(sc, dim=1)
                o[h] = torch.exp(sc - lse[h][:, None]) @ V[h // grp]
            keep("out", o)
            keep("lse", lse)
        elif c["kind"] == "read":
            keep("k_cache", _exact_row(c, s["kc"], s["ks"], s["table"], b, n)[:, n - m:])
            keep("v_cache", _exact_row(c, s["vc"], s["vs"], s["table"], b, n)[:, n - m:])
        else:
            r, half = c["rot"], c["rot"] // 2
            at = torch.arange(n - m, n, device="cuda")
            turn = torch.polar(torch.ones(m, half, device="cuda", dtype=torch.float64),
                               at.double()[:, None] * s["inv_freq"].double()[None])
            first = torch.arange(half, device="cuda") * (2 if c["pairs"] == "even" else 1)
            second = first + (1 if c["pairs"] == "even" else half)
            made = {}
            for key in ("q", "k"):
                x = part(s[key], b).clone()
                z = torch.complex(x[..., first], x[..., second]) * turn
                x[..., first], x[..., second] = z.real, z.imag
                keep(key, x)
                made[key] = x
            for key, x in (("k_cache", made["k"]), ("v_cache", part(s["v"], b))):
                if c["fmt"] == "fp4":
                    keep(key, _exact_quantised(x.unflatten(-1, (-1, 32))).flatten(-2))
                else:
                    pools[key][s["table"][b].long()[at // c["page"]], :, at % c["page"]] = x.transpose(0, 1)
        start += m
    join = lambda xs: torch.cat(xs, dim=1) if _packed(c) else torch.stack(xs)
    got = {key: join(xs) for key, xs in outs.items()}
    if "lse" in got:
        got["lse"] = got["lse"].reshape(-1)
    return {**got, **pools}
