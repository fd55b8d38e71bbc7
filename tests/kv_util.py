"""The paged cache's operators written out plainly in 64 bits, and caches with known contents (shared by the cache's tests)."""
import math

import torch

E2M1 = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
NAN_BYTE = 255


def fp4_pack(x):
    """x [..., d] (64 bits) -> codes uint8 [..., d / 2], scale bytes uint8 [..., d / 32], by trying every exponent and every code."""
    g = x.double().cpu().unflatten(-1, (-1, 32))
    bad = ~torch.isfinite(g).all(dim=-1)
    top = torch.where(bad, 0.0, g.abs().amax(dim=-1))
    e = torch.arange(-120, 126, dtype=torch.float64)
    fits = top[..., None] <= 7.0 * torch.exp2(e)
    e = torch.where(fits.any(dim=-1), e[fits.int().argmax(dim=-1)], 125.0)
    a = torch.where(bad[..., None], 0.0, g.abs() * torch.exp2(-e)[..., None])
    dist = (a[..., None] - E2M1).abs()
    even = dist[..., 0::2].min(dim=-1)
    odd = dist[..., 1::2].min(dim=-1)
    code = torch.where(odd.values < even.values, 2 * odd.indices + 1, 2 * even.indices)
    code = (code + 8 * (g < 0)).masked_fill(bad[..., None], 0).flatten(-2)
    byte = torch.where(bad, float(NAN_BYTE), e + 127)
    return (code[..., 0::2] | code[..., 1::2] << 4).to(torch.uint8), byte.to(torch.uint8)


def fp4_values(codes, scales):
    """codes [..., d / 2], scales [..., d / 32] -> float64 [..., d]"""
    c = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2).long()
    x = torch.cat([E2M1, -E2M1]).to(codes.device)[c].unflatten(-1, (-1, 32))
    s = torch.where(scales == NAN_BYTE, math.nan, torch.exp2(scales.double() - 127))
    return (x * s[..., None]).flatten(-2)


def rotate(x, pos, inv_freq, interleaved):
    """x [..., n, d] at positions pos [n], in 64 bits"""
    half = inv_freq.numel()
    x = x.double().clone()
    t = pos.double()[:, None] * inv_freq.double()
    first = torch.arange(half, device=x.device) * (2 if interleaved else 1)
    second = first + (1 if interleaved else half)
    x1, x2 = x[..., first].clone(), x[..., second].clone()
    x[..., first] = x1 * t.cos() - x2 * t.sin()
    x[..., second] = x2 * t.cos() + x1 * t.sin()
    return x


class Cache:
    """A paged cache on `device`, every byte of its storage poisoned (NaN rows, NaN scale bytes), with pages dealt out in a
    shuffled order.  put / rows move dense values [Hkv, n, d] of a sequence in and out by the documented layout."""

    def __init__(self, api, lens, Hkv, d, dtype=torch.bfloat16, fp4=False, page=16, seed=0, device="cuda", spare=2, room=None, views=False):
        self.api, self.lens, self.Hkv, self.d, self.page, self.fp4 = api, list(lens), Hkv, d, page, fp4
        gen = torch.Generator().manual_seed(seed)
        per = [-(-n // page) for n in lens]
        self.max_pages = max(max(per), 1) if room is None else room
        n_pages = sum(per) + spare
        order = torch.randperm(n_pages, generator=gen).int()
        table = torch.full((len(lens), self.max_pages), -1, dtype=torch.int32)
        at = 0
        for b, n in enumerate(per):
            table[b, :n] = order[at:at + n]
            at += n
        self.table = table.to(device)
        self.kv_len = torch.tensor(lens, dtype=torch.int32, device=device)
        fmt = api.AA_KV_FP4 if fp4 else api.AA_KV_PLAIN
        c = api.alloc_kv_cache(n_pages, Hkv, page, d, dtype, fmt, device)
        if views:                       # token-major pages, K and V side by side: every stride another
            if fp4:
                both = torch.zeros(n_pages, page, Hkv, d, dtype=torch.uint8, device=device)
                c["k"], c["v"] = both[..., :d // 2].transpose(1, 2), both[..., d // 2:].transpose(1, 2)
                s = torch.zeros(n_pages, 2, Hkv, d // 32, page, dtype=torch.uint8, device=device)
                c["k_scale"], c["v_scale"] = s[:, 0], s[:, 1]
            else:
                both = torch.zeros(n_pages, page, Hkv, 2 * d, dtype=dtype, device=device)
                c["k"], c["v"] = both[..., :d].transpose(1, 2), both[..., d:].transpose(1, 2)
        for key in ("k", "v"):
            if fp4:
                c[key].fill_(0x77)
                c[key + "_scale"].fill_(NAN_BYTE)
            else:
                c[key].fill_(math.nan)
        self.c = c

    def _at(self, b, first, n):
        j = torch.arange(first, first + n)
        return self.table[b].cpu()[j // self.page].long().to(self.table.device), (j % self.page).to(self.table.device)

    def put(self, key, b, first, x):
        page, row = self._at(b, first, x.shape[1])
        x = x.to(self.table.device).transpose(0, 1)
        if not self.fp4:
            self.c[key][page, :, row] = x.to(self.c[key].dtype)
            return
        codes, scales = fp4_pack(x)
        self.c[key][page, :, row] = codes.to(page.device)
        self.c[key + "_scale"][page, :, :, row] = scales.to(page.device)

    def rows(self, key, b, first, n):
        """float64 [Hkv, n, d]"""
        page, row = self._at(b, first, n)
        x = self.c[key][page, :, row]
        x = x.double() if not self.fp4 else fp4_values(x, self.c[key + "_scale"][page, :, :, row])
        return x.transpose(0, 1)

    def fill(self, seed=1, scale=1.0):
        gen = torch.Generator().manual_seed(seed)
        for b, n in enumerate(self.lens):
            if n:
                for key in ("k", "v"):
                    self.put(key, b, 0, scale * torch.randn(self.Hkv, n, self.d, generator=gen, dtype=torch.float64))
        return self


def attend(q, K, V, first_pos, scale, causal=True, there=None):
    """q [Hq, n, d] (row i at position first_pos + i), K, V [Hkv, len, d], all float64.  Returns out, lse, sum_j p_j |v_j|, and the
    largest sum of |q_c k_c| of a row; rows without a key: zeros and -inf."""
    Hq, n, d = q.shape
    grp, length = Hq // K.shape[0], K.shape[1]
    K, V = K.repeat_interleave(grp, dim=0), V.repeat_interleave(grp, dim=0)
    j = torch.arange(length, device=q.device)
    hide = torch.zeros(n, length, dtype=torch.bool, device=q.device)
    if causal:
        hide = j > (first_pos + torch.arange(n, device=q.device))[:, None]
    if there is not None:
        hide = hide | ~there
        K, V = K.masked_fill(~there[None, :, None], 0.0), V.masked_fill(~there[None, :, None], 0.0)
    s = (torch.matmul(q, K.transpose(1, 2).contiguous()) * scale).masked_fill(hide, -math.inf)
    size = (torch.matmul(q.abs(), K.abs().transpose(1, 2).contiguous()) * scale).masked_fill(hide, 0.0)
    empty = hide.all(dim=1)[None].expand(Hq, n)
    if length == 0:
        z = torch.zeros_like(q)
        return z, torch.full((Hq, n), -math.inf, dtype=q.dtype, device=q.device), z, torch.zeros(Hq, n, dtype=q.dtype, device=q.device)
    lse = torch.logsumexp(s, dim=2)
    p = torch.exp(s - torch.where(empty, 0.0, lse)[..., None])
    p = torch.where(empty[..., None], 0.0, p)
    return torch.matmul(p, V), torch.where(empty, -math.inf, lse), torch.matmul(p, V.abs()), size.amax(dim=2)


def tolerances(out, A, size, lse, keys, d, dtype):
    """How far an attention in `dtype` with 32-bit sums may be off, element by element.
    u = 2^-24, half a step of 32 bits.  A score: d products summed, scaled, base changed: (d + 4) u size =: e (and as much again for
    the exponential's argument).  A weight: relative 2 e + 4 u.  The sums over `keys` weights: keys * u.  bf16: a weight and the result
    are rounded by 2^-8 of their value at most."""
    u = 2.0 ** -24
    e = (d + 4) * u * size + 4 * u * (1 + size)
    rel = (4 * e + 8 * u + 2 * keys * u)[..., None]
    o = rel * A
    if dtype == torch.bfloat16:
        o = o + 2.0 ** -8 * (out.abs() + 2 * A)        # 2 A: the weights' rounding, in the numerator alone, of both signs
    else:
        o = o + u * out.abs()
    return o + 1e-30, 2 * e + 8 * u + keys * u + 2 * u * lse.abs().clamp(max=1e30)
