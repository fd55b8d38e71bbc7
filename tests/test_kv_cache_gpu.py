"""kv_append, kv_attn and kv_read against the operators written out in 64 bits, at the sizes, masks and layouts where they can go wrong."""
import math

import pytest
import torch

from kv_util import Cache, attend, fp4_pack, fp4_values, rotate, tolerances

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def api():
    from paper_2505_23520_amd import api as _api
    assert torch.cuda.is_available()
    return _api


def _randn(*shape, seed=0, dtype=BF):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64).to(dtype).cuda()


def _attn(api, cache, q, cu=None, max_new=None, ws=None, stream=None, out=None, **kw):
    """kv_attn on poisoned outputs and workspace: out like q, lse as documented."""
    out = torch.full_like(q, 7.0) if out is None else out
    p = api.make_kv_params(cache.c, cache.table, cache.kv_len, q=q, out=out, cu_seqlens=cu, max_new=max_new, **kw)
    lse = torch.full((q.shape[:-1].numel(),), 7.0, device="cuda")
    if ws is None:
        ws = torch.full((api.kv_attn_workspace_bytes(p),), 0xff, dtype=torch.uint8, device="cuda")
    api.kv_attn(p, q, out, lse, ws, stream=stream)
    return out, lse.view(q.shape[:-1])


def _check_attn(api, cache, q, new, packed=False, causal=True, there=None, **kw):
    """Every row of the call against attend(); the rows of nobody stay as they were."""
    ends = [0]
    for n in new:
        ends.append(ends[-1] + n)
    cu = torch.tensor(ends, dtype=torch.int32, device="cuda") if packed else None
    out, lse = _attn(api, cache, q, cu, max(max(new), 1) if packed else None, causal=causal, **kw)
    torch.cuda.synchronize()
    d = q.shape[-1]
    for b, n in enumerate(new):
        if n == 0:
            continue
        sl = (slice(None), slice(ends[b], ends[b + 1])) if packed else (b,)
        ln = max(cache.lens[b], 0)
        K, V = (cache.rows(x, b, 0, ln) for x in ("k", "v"))
        want, wl, A, size = attend(q[sl].double(), K, V, ln - n, kw.get("softmax_scale") or 1 / math.sqrt(d), causal,
                                   None if there is None else there[b])
        to, tl = tolerances(want, A, size, wl, max(ln, 1), d, q.dtype)
        err, el = (out[sl].double() - want).abs(), (lse[sl].double() - wl).abs()
        el = torch.where(torch.isinf(wl) & (lse[sl].double() == wl), 0.0, el)
        assert torch.isfinite(out[sl]).all()
        assert bool((err <= to).all()), (b, float((err / to).max()))
        assert bool((el <= tl).all()), (b, float((el / tl).max()))
    if packed and ends[-1] < q.shape[1]:
        assert torch.all(out[:, ends[-1]:] == 7.0) and torch.all(lse[:, ends[-1]:] == 7.0)
    return out, lse


FORMATS = [(BF, False, 128), (BF, True, 128), (BF, False, 64), (BF, True, 64), (F32, False, 128), (F32, False, 64), (F32, False, 32)]
LENS = [0, 1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 255, 257, 511, 700, 1025, 2049]


@pytest.mark.parametrize("dtype,fp4,d", FORMATS)
@pytest.mark.parametrize("Hq,Hkv,page", [(8, 2, 16), (4, 4, 64), (5, 1, 128), (40, 2, 32)])
def test_attn_one_token(api, dtype, fp4, d, Hq, Hkv, page):
    cache = Cache(api, LENS, Hkv, d, dtype, fp4, page, seed=d + Hq).fill()
    _check_attn(api, cache, _randn(len(LENS), Hq, 1, d, seed=3, dtype=dtype), [1] * len(LENS))


@pytest.mark.parametrize("dtype,fp4,d", FORMATS)
@pytest.mark.parametrize("n", [2, 3, 5, 8, 17, 64, 130])
def test_attn_some_tokens(api, dtype, fp4, d, n):
    """More new tokens than some sequences have: rows that see no key."""
    lens = [0, 1, n - 1, n, n + 1, 47, 130, 333, 1100]
    cache = Cache(api, lens, 2, d, dtype, fp4, 32, seed=n).fill()
    _check_attn(api, cache, _randn(len(lens), 8, n, d, seed=n, dtype=dtype), [n] * len(lens))


@pytest.mark.parametrize("dtype,fp4,d", FORMATS)
@pytest.mark.parametrize("causal", [True, False])
def test_attn_packed(api, dtype, fp4, d, causal):
    """Packed new tokens with empty sequences, and rows behind the last one."""
    new, lens = [0, 3, 1, 0, 70, 129, 0], [5, 2, 400, 0, 70, 700, 33]
    cache = Cache(api, lens, 2, d, dtype, fp4, 16, seed=9).fill()
    q = _randn(sum(new) + 5, 6, d, seed=4, dtype=dtype).transpose(0, 1)          # token-major
    _check_attn(api, cache, q, new, packed=True, causal=causal)


@pytest.mark.parametrize("dtype,fp4,d", [(BF, False, 128), (BF, True, 128), (BF, False, 64), (F32, False, 64)])
@pytest.mark.parametrize("new", [1, 3, 20])
def test_attn_many_sequences(api, dtype, fp4, d, new):
    """More sequences than a wave has lanes, of very different lengths, empty ones among them: packed, some without new tokens."""
    lens = [(i * i * 977) % 1500 if i % 7 else (0, 1, 128, 129)[i // 7 % 4] for i in range(150)] + [5000]
    news = [new if i % 5 else (i // 5) % (new + 1) for i in range(150)] + [new]
    cache = Cache(api, lens, 1, d, dtype, fp4, 16, seed=11).fill()
    q = _randn(sum(news) + 3, 4, d, seed=5, dtype=dtype).transpose(0, 1)
    _check_attn(api, cache, q, news, packed=True)


@pytest.mark.parametrize("dtype,fp4", [(BF, False), (BF, True), (F32, False)])
@pytest.mark.parametrize("n,Hq", [(1, 8), (7, 8), (90, 8), (1, 64)])
def test_attn_long_keys(api, dtype, fp4, n, Hq):
    """Long sequences of unequal length: tiles that many work-groups share, that one finishes, that begin and end inside of stretches."""
    lens = [9001, 130, 20011]
    cache = Cache(api, lens, 2, 128, dtype, fp4, 64, seed=12).fill()
    _check_attn(api, cache, _randn(3, Hq, n, 128, seed=6, dtype=dtype), [n] * 3)
    one = Cache(api, [20011], 2, 128, dtype, fp4, 128, seed=13).fill()
    _check_attn(api, one, _randn(1, Hq, n, 128, seed=7, dtype=dtype), [n])


@pytest.mark.parametrize("dtype,fp4,d", [(BF, False, 64), (BF, True, 64), (F32, False, 128), (F32, False, 64), (BF, True, 128), (BF, False, 128)])
@pytest.mark.parametrize("n,length", [(9, 4000), (24, 4000), (150, 3000), (700, 700)])
def test_attn_one_sequence_many_rows(api, dtype, fp4, d, n, length):
    """One sequence whose rows take several row tiles, the keys of each in shares."""
    cache = Cache(api, [length], 2, d, dtype, fp4, 64, seed=n).fill()
    _check_attn(api, cache, _randn(1, 8, n, d, seed=n, dtype=dtype), [n])


@pytest.mark.parametrize("dtype,fp4", [(BF, False), (BF, True), (F32, False)])
@pytest.mark.parametrize("n", [1, 40])
def test_attn_shared_pages(api, dtype, fp4, n):
    """Two sequences on the pages of one prefix, and a sequence that has a page twice."""
    lens = [700, 650, 300]
    cache = Cache(api, lens, 2, 128, dtype, fp4, 32, seed=2).fill()
    cache.table[1, :15] = cache.table[0, :15]
    cache.table[2, 5] = cache.table[2, 1]
    _check_attn(api, cache, _randn(3, 8, n, 128, seed=n, dtype=dtype), [n] * 3)


@pytest.mark.parametrize("n", [1, 33])
def test_attn_fp4_nan_group(api, n):
    """A group that held a NaN: every row that sees the key is NaN, rows of other sequences and KV heads are not."""
    cache = Cache(api, [300, 300], 2, 128, BF, True, 16, seed=3).fill()
    x = torch.zeros(2, 1, 128, dtype=torch.float64)
    x[0, 0, 40] = math.nan
    cache.put("k", 0, 77, x)
    out, lse = _attn(api, cache, _randn(2, 4, n, 128, seed=1))
    assert torch.isnan(out[0, :2]).all() and torch.isnan(lse[0, :2]).all()
    assert torch.isfinite(out[0, 2:]).all() and torch.isfinite(out[1]).all()


@pytest.mark.parametrize("dtype,fp4,d", FORMATS)
@pytest.mark.parametrize("n", [1, 33])
def test_attn_holes(api, dtype, fp4, d, n):
    """Pages that are not there (-1, or outside the pool) are not attended: in the middle, the first, the last, all."""
    lens, page = [500, 500, 500, 500, 90], 16
    cache = Cache(api, lens, 2, d, dtype, fp4, page, seed=2).fill()
    there = [torch.ones(x, dtype=torch.bool, device="cuda") for x in lens]
    bad = cache.table.clone()
    for b, pages in ((0, [3, 4, 9]), (1, [0]), (2, [31]), (3, list(range(32)))):
        for x in pages:
            bad[b, x] = (-1, cache.c["k"].shape[0], 2**31 - 1, -2**31)[x % 4]
            there[b][x * page:(x + 1) * page] = False
    good, cache.table = cache.table, bad
    q = _randn(len(lens), 4, n, d, seed=5, dtype=dtype)
    rows = cache.rows
    cache.table = good
    K = {(x, b): rows(x, b, 0, lens[b]) for x in ("k", "v") for b in range(len(lens))}
    cache.rows = lambda x, b, first, m: K[x, b]
    cache.table = bad
    _check_attn(api, cache, q, [n] * len(lens), there=there)


@pytest.mark.parametrize("dtype,fp4", [(BF, False), (BF, True), (F32, False)])
def test_attn_strides_and_orders(api, dtype, fp4):
    """Pools as views of a token-major buffer, q and out with strides of their own, batch of one and single heads."""
    for lens, Hq, Hkv in (([300, 41], 8, 2), ([129], 4, 1)):
        cache = Cache(api, lens, Hkv, 128, dtype, fp4, 32, seed=1, views=True).fill()
        big = _randn(len(lens), 3, Hq + 2, 160, seed=6, dtype=dtype)
        q = big[:, :, 1:Hq + 1, 16:144].transpose(1, 2)
        out = torch.full((len(lens), Hq, 3, 192), 7.0, dtype=dtype, device="cuda")
        _check_attn(api, cache, q, [3] * len(lens), out=out[..., 32:160])
        assert torch.all(out[..., :32] == 7.0) and torch.all(out[..., 160:] == 7.0)


@pytest.mark.parametrize("dtype,fp4", [(BF, False), (BF, True), (F32, False)])
@pytest.mark.parametrize("max_len", [0, 1, 100, 2000, 2**31 - 1])
def test_attn_length_hint(api, dtype, fp4, max_len):
    """max_len deals the keys out; it never changes which are attended."""
    lens = [2000, 3, 1999, 640]
    cache = Cache(api, lens, 1, 128, dtype, fp4, 64, seed=8, room=300).fill()
    _check_attn(api, cache, _randn(4, 4, 2, 128, seed=8, dtype=dtype), [2] * 4, max_len=max_len)


@pytest.mark.parametrize("dtype,fp4", [(BF, False), (BF, True), (F32, False)])
def test_attn_length_beyond_the_table(api, dtype, fp4):
    """A kv_len beyond the table's pages: what has storage is attended."""
    cache = Cache(api, [64], 1, 64 if fp4 else 128, dtype, fp4, 16, seed=8).fill()
    q = _randn(1, 2, 1, cache.d, seed=8, dtype=dtype)
    want, wl = _attn(api, cache, q)
    for much in (65, 1000, 2**31 - 1):
        cache.kv_len.fill_(much)
        got, gl = _attn(api, cache, q)
        assert torch.equal(got, want) and torch.equal(gl, wl)


@pytest.mark.parametrize("dtype,fp4,scale", [(BF, False, 30.0), (BF, True, 30.0), (F32, False, 30.0), (F32, False, 1e-3)])
def test_attn_magnitudes(api, dtype, fp4, scale):
    """Scores of hundreds (one key holds a row), or all alike; and softmax_scale given."""
    lens = [1, 77, 1500]
    cache = Cache(api, lens, 2, 128, dtype, fp4, 32, seed=3).fill(scale=scale)
    _check_attn(api, cache, _randn(3, 4, 2, 128, seed=2, dtype=dtype), [2] * 3)
    _check_attn(api, cache, _randn(3, 4, 2, 128, seed=2, dtype=dtype), [2] * 3, softmax_scale=0.5)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n", [1, 40])
def test_attn_nonfinite(api, dtype, n):
    """Infinite scores as the formula has them: +inf makes a row NaN, -inf takes a key out, all -inf leaves the row empty."""
    cache = Cache(api, [200, 200, 200, 200], 1, 128, dtype, False, 16, seed=3).fill()
    q = torch.ones(4, 2, n, 128, dtype=dtype, device="cuda")
    page, row = cache._at(0, 50, 1)
    cache.c["k"][page, :, row, 0] = math.inf
    page, row = cache._at(1, 50, 1)
    cache.c["k"][page, :, row, 0] = -math.inf
    for j in range(200):
        page, row = cache._at(2, j, 1)
        cache.c["k"][page, :, row, 0] = -math.inf
    page, row = cache._at(3, 50, 1)
    cache.c["k"][page, :, row, 0] = math.nan
    out, lse = _attn(api, cache, q)
    assert torch.isnan(out[0]).all() and torch.isnan(out[3]).all() and torch.isnan(lse[3]).all()
    assert torch.all(out[2] == 0) and torch.all(lse[2] == -math.inf)
    there = torch.ones(200, dtype=torch.bool, device="cuda")
    there[50] = False
    want, wl, A, size = attend(q[1].double(), cache.rows("k", 1, 0, 200), cache.rows("v", 1, 0, 200), 200 - n, 1 / math.sqrt(128), True, there)
    to, tl = tolerances(want, A, size, wl, 200, 128, dtype)
    assert bool(((out[1].double() - want).abs() <= to).all()) and bool(((lse[1].double() - wl).abs() <= tl).all())


@pytest.mark.parametrize("dtype,fp4,d", FORMATS)
@pytest.mark.parametrize("n", [2, 5, 9, 14, 40, 130])
def test_attn_values_not_finite(api, dtype, fp4, d, n):
    """Infinities and NaN among the new tokens' values: rows that do not see them are as if 0 stood there (or have no key at all), rows that
    do have them in their channels and are right in the others."""
    lens = [200, max(n - 3, 1), n, 777]
    cache = Cache(api, lens, 2, d, dtype, fp4, 16, seed=n).fill()
    q = _randn(4, 8, n, d, seed=n, dtype=dtype)
    bad = {}                                           # (sequence, token) -> {channel: value} of KV head 1
    for b, ln in enumerate(lens):
        first = max(ln - n, 0)
        for j, put in ((ln - 1, {3: math.inf}), (first + (ln - first) // 2, {d - 1: math.nan}), (max(ln - 2, first), {3: -math.inf, 17: -math.inf})):
            bad.setdefault((b, j), {}).update(put)
    K = [cache.rows("k", b, 0, ln) for b, ln in enumerate(lens)]
    V = [cache.rows("v", b, 0, ln).clone() for b, ln in enumerate(lens)]
    marks = [torch.zeros(2, ln, d, dtype=torch.float64, device="cuda") for ln in lens]
    for (b, j), put in bad.items():
        page, row = cache._at(b, j, 1)
        for c, x in put.items():
            if fp4:
                cache.c["v_scale"][page, 1, c // 32, row] = 255
                V[b][1, j, c // 32 * 32:c // 32 * 32 + 32] = 0
                marks[b][1, j, c // 32 * 32:c // 32 * 32 + 32] = math.nan
            else:
                cache.c["v"][page, 1, row, c] = x
                V[b][1, j, c] = 0
                marks[b][1, j, c] = x
    out, lse = _attn(api, cache, q)
    for b, ln in enumerate(lens):
        want, wl, A, size = attend(q[b].double(), K[b], V[b], ln - n, 1 / math.sqrt(d))
        to, _ = tolerances(want, A, size, wl, ln, d, dtype)
        for i in range(n):
            seen = max(ln - n + i + 1, 0)
            extra = marks[b][:, :seen].sum(dim=1).repeat_interleave(4, dim=0)             # 0, an infinity, or NaN
            fine = extra == 0
            err = (out[b, :, i].double() - want[:, i]).abs()
            assert bool((err[fine] <= to[:, i][fine]).all()), (b, i)
            got = out[b, :, i][~fine].double()
            assert torch.equal(got.nan_to_num(nan=5.0), extra[~fine].nan_to_num(nan=5.0)), (b, i)


@pytest.mark.parametrize("dtype,fp4,d", FORMATS)
@pytest.mark.parametrize("Hq,length", [(8, 2500), (8, 400), (64, 9000)])
def test_attn_nan_in_one_share(api, dtype, fp4, d, Hq, length):
    """A NaN key, and a NaN value, far from the end of keys that several work-groups take: rows that see it are NaN (values: in their
    channels), with a NaN lse for the key; the rows before it and the other KV head's are right."""
    n, at = 150, length - 100                              # new tokens 50 .. see it
    q = _randn(1, Hq, n, d, seed=3, dtype=dtype)
    for key in ("k", "v"):
        cache = Cache(api, [length], 2, d, dtype, fp4, 64, seed=3).fill()
        K, V = cache.rows("k", 0, 0, length), cache.rows("v", 0, 0, length)
        page, row = cache._at(0, at, 1)
        if fp4:
            cache.c[key + "_scale"][page, 0, 1, row] = 255
        else:
            cache.c[key][page, 0, row, 40 % d] = math.nan
        out, lse = _attn(api, cache, q)
        want, wl, A, size = attend(q[0].double(), K, V, length - n, 1 / math.sqrt(d))
        to, tl = tolerances(want, A, size, wl, length, d, dtype)
        bad = torch.zeros(Hq, n, d, dtype=torch.bool, device="cuda")
        bad[:Hq // 2, 50:, slice(None) if key == "k" else slice(32, 64) if fp4 else 40 % d] = True
        assert torch.equal(torch.isnan(out[0]), bad)
        assert torch.equal(torch.isnan(lse[0]), bad.all(dim=2))
        fine = ~bad
        assert bool(((out[0].double() - want).abs()[fine] <= to[fine]).all())
        assert bool(((lse[0].double() - wl).abs() <= tl)[~bad.all(dim=2)].all())


@pytest.mark.parametrize("fp4", [False, True])
def test_offsets_beyond_32_bits(api, fp4):
    """A pool whose last pages lie beyond 2^32 bytes: appended to, read and attended there."""
    d, Hkv, page = 128, 8, 64
    per_page = Hkv * page * (d // 2 if fp4 else 2 * d)
    n_pages = (5 << 30) // per_page
    c = {x: torch.empty(n_pages, Hkv, page, d // 2 if fp4 else d, dtype=torch.uint8 if fp4 else BF, device="cuda") for x in ("k", "v")}
    for x in ("k", "v"):
        c[x + "_scale"] = torch.empty(n_pages, Hkv, d // 32, page, dtype=torch.uint8, device="cuda") if fp4 else None
    small = Cache(api, [200], Hkv, d, BF, fp4, page, seed=1)
    big = Cache(api, [200], Hkv, d, BF, fp4, page, seed=1)
    big.c, big.table = c, torch.arange(n_pages - 4, n_pages, dtype=torch.int32, device="cuda")[None]
    got = []
    for cache in (small, big):
        q, k, v = (_randn(1, H, 200, d, seed=s) for H, s in ((16, 1), (Hkv, 2), (Hkv, 3)))
        qo, f = torch.empty_like(q), torch.rand(d // 2, generator=torch.Generator().manual_seed(1)).cuda()
        p = api.make_kv_params(cache.c, cache.table, cache.kv_len, q=q, k=k, v=v, out=qo, rot_dim=d)
        api.kv_append(p, q, k, v, f, None, qo)
        out, lse = _attn(api, cache, qo)
        ko, vo = torch.empty_like(k), torch.empty_like(v)
        api.kv_read(api.make_kv_params(cache.c, cache.table, cache.kv_len, k=ko, v=vo), ko, vo)
        got.append((out, lse, ko, vo))
    assert all(torch.equal(a, b) for a, b in zip(*got))


# ------------------------------------------------------------------ append and read
def _append(api, cache, q, k, v, rot, interleaved=False, positions=None, cu=None, max_new=None, inv_freq=None, k_out=True):
    f = torch.pow(10000.0, -torch.arange(max(rot // 2, 1), dtype=torch.float64) * 2 / max(rot, 1)).float().cuda() if inv_freq is None else inv_freq
    qo = None if q is None else torch.full_like(q, 7.0)
    ko = torch.full_like(k, 7.0) if k_out and k is not None else None
    p = api.make_kv_params(cache.c, cache.table, cache.kv_len, q=q, k=k, v=v, out=qo, k_out=ko, cu_seqlens=cu, max_new=max_new,
                           rot_dim=rot, rot_interleaved=interleaved)
    api.kv_append(p, q, k, v, f[:rot // 2] if rot else None, positions, qo, ko)
    return qo, ko, f[:rot // 2]


def _near(got, want, dtype, size=None):
    """Rounded once from sums of two products in 32 bits: half a step, and the sums' own 4 u of the magnitudes in them."""
    half = 2.0 ** -8 if dtype == BF else 2.0 ** -24
    size = want.abs() if size is None else size
    assert bool(((got.double() - want).abs() <= half * want.abs() + 6 * 2.0 ** -24 * size + 1e-40).all())


def _storage(cache):
    return [t.clone() for t in cache.c.values() if t is not None]


@pytest.mark.parametrize("dtype,fp4,d", FORMATS)
@pytest.mark.parametrize("rot,interleaved", [(0, False), (16, False), (16, True), (32, False), (0.5, True), (1, False), (1, True)])
def test_append(api, dtype, fp4, d, rot, interleaved):
    """Batches with tokens before the sequence's start, whole prompts, and one token; q, k, v as one fused projection."""
    rot = int(rot * d) if rot in (0.5, 1) else rot
    n, lens, Hq, Hkv = 35, [35, 36, 20, 99, 0, 4000], 4, 2
    cache = Cache(api, lens, Hkv, d, dtype, fp4, 16, seed=d)
    x = _randn(len(lens), n, Hq + 2 * Hkv, d, seed=rot, dtype=dtype)
    q, k, v = (y.transpose(1, 2) for y in x.split([Hq, Hkv, Hkv], dim=2))
    before = _storage(cache)
    qo, ko, f = _append(api, cache, q, k, v, rot, interleaved)
    written = [torch.zeros(t.shape, dtype=torch.bool, device="cuda") for t in before]
    keys = [key for key, t in cache.c.items() if t is not None]
    for b, ln in enumerate(lens):
        pos = torch.arange(ln - n, ln, device="cuda")
        for got, src in ((qo[b], q[b]), (ko[b], k[b])):
            want = rotate(src, pos, f, interleaved)
            _near(got, want, dtype, src.double().abs().amax(dim=-1, keepdim=True) * 2)
        first = max(ln - n, 0)
        skip = first - (ln - n)
        if ln == 0:
            continue
        K, V = rotate(k[b], pos, f, interleaved)[:, skip:], v[b].double()[:, skip:]
        if fp4:
            assert torch.equal(cache.rows("k", b, first, ln - first), fp4_values(*fp4_pack(K)).cuda())
            assert torch.equal(cache.rows("v", b, first, ln - first), fp4_values(*fp4_pack(V)).cuda())
        else:
            assert torch.equal(cache.rows("k", b, first, ln - first), ko[b].double()[:, skip:])
            assert torch.equal(cache.rows("v", b, first, ln - first), V)
        page, row = cache._at(b, first, ln - first)
        for key, w in zip(keys, written):
            if "scale" in key:
                w[page, :, :, row] = True
            else:
                w[page, :, row] = True
    for t, key, w in zip(before, keys, written):                      # nothing else of the storage was touched
        same = (t == cache.c[key]) | (torch.isnan(t.float()) & torch.isnan(cache.c[key].float()))
        assert bool((same | w).all())


@pytest.mark.parametrize("dtype,fp4,d", FORMATS)
@pytest.mark.parametrize("Hq,Hkv,interleaved", [(4, 2, False), (4, 1, True), (32, 8, False), (40, 4, True)])
def test_append_many_tokens(api, dtype, fp4, d, Hq, Hkv, interleaved):
    """Enough tokens for the work-groups that take four of them: few rows a token and many, a last work-group that is not full,
    packed sequences of all lengths beside it."""
    new = [700, 0, 1, 333, 2, 66, 1]
    lens = [x + (i * 37) % 100 for i, x in enumerate(new)]
    T, rot = sum(new), d
    cache = Cache(api, lens, Hkv, d, dtype, fp4, 32, seed=d)
    q, k, v = (_randn(T + 1, H, d, seed=s, dtype=dtype).transpose(0, 1) for H, s in ((Hq, 1), (Hkv, 2), (Hkv, 3)))
    cu = torch.tensor([0] + new).cumsum(0).int().cuda()
    qo, ko, f = _append(api, cache, q, k, v, rot, interleaved, cu=cu, max_new=max(new))
    pos = torch.cat([torch.arange(ln - n, ln) for n, ln in zip(new, lens)]).cuda()
    _near(qo[:, :T], rotate(q[:, :T], pos, f, interleaved), dtype, q[:, :T].double().abs().amax(dim=-1, keepdim=True) * 2)
    want = rotate(k[:, :T], pos, f, interleaved)
    _near(ko[:, :T], want, dtype, k[:, :T].double().abs().amax(dim=-1, keepdim=True) * 2)
    at = 0
    for b, n in enumerate(new):
        if n:
            sl = slice(at, at + n)
            K, V = cache.rows("k", b, lens[b] - n, n), cache.rows("v", b, lens[b] - n, n)
            assert torch.equal(K, fp4_values(*fp4_pack(want[:, sl])).cuda() if fp4 else ko[:, sl].double())
            assert torch.equal(V, fp4_values(*fp4_pack(v[:, sl].double())).cuda() if fp4 else v[:, sl].double())
        at += n
    back_k, back_v = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    api.kv_read(api.make_kv_params(cache.c, cache.table, cache.kv_len, k=back_k, v=back_v, cu_seqlens=cu, max_new=max(new)), back_k, back_v)
    rows = lambda x: torch.cat([cache.rows(x, b, lens[b] - n, n) for b, n in enumerate(new) if n], dim=1)
    assert torch.equal(back_k[:, :T].double(), rows("k")) and torch.equal(back_v[:, :T].double(), rows("v"))
    assert torch.all(back_k[:, T:] == 7.0) and torch.all(qo[:, T:] == 7.0) and torch.all(ko[:, T:] == 7.0)


@pytest.mark.parametrize("dtype,fp4", [(BF, False), (BF, True), (F32, False)])
def test_append_packed_with_positions(api, dtype, fp4):
    """Packed tokens, empty sequences, rows of nobody, positions of their own (far, negative), more sequences than a wave has lanes."""
    new = [0, 3, 1, 0, 40] + [i % 3 for i in range(140)] + [0]
    lens = [x + i % 7 for i, x in enumerate(new)]
    T, d, Hq, Hkv = sum(new) + 4, 128, 4, 2
    cache = Cache(api, lens, Hkv, d, dtype, fp4, 16, seed=3)
    q, k, v = (_randn(H, T, d, seed=s, dtype=dtype) for H, s in ((Hq, 1), (Hkv, 2), (Hkv, 3)))
    pos = torch.randint(-5, 2_000_000, (T,), generator=torch.Generator().manual_seed(5)).int().cuda()
    ends = torch.tensor([0] + new).cumsum(0).int().cuda()
    qo, ko, f = _append(api, cache, q, k, v, d, positions=pos, cu=ends, max_new=max(new))
    n = sum(new)
    _near(qo[:, :n], rotate(q[:, :n], pos[:n], f, False), dtype, q[:, :n].double().abs().amax(dim=-1, keepdim=True) * 2)
    want = rotate(k[:, :n], pos[:n], f, False)
    _near(ko[:, :n], want, dtype, k[:, :n].double().abs().amax(dim=-1, keepdim=True) * 2)
    assert torch.all(qo[:, n:] == 7.0) and torch.all(ko[:, n:] == 7.0)
    at = 0
    for b, m in enumerate(new):
        if m:
            K = cache.rows("k", b, lens[b] - m, m)
            W = fp4_values(*fp4_pack(want[:, at:at + m])).cuda() if fp4 else ko[:, at:at + m].double()
            assert torch.equal(K, W)
        at += m


@pytest.mark.parametrize("B", [65, 200, 4097, 5000])
def test_append_packed_many_sequences(api, B):
    """Which sequence a packed row belongs to, many of them without rows: each row stored at its sequence's end, and read back."""
    gen = torch.Generator().manual_seed(B)
    new = torch.randint(0, 4, (B,), generator=gen)
    new[torch.rand(B, generator=gen) < 0.3] = 0
    lens = (new + torch.randint(0, 9, (B,), generator=gen)).tolist()
    T, d = int(new.sum()), 64
    cache = Cache(api, lens, 1, d, BF, False, 16, seed=1)
    k, v = (_randn(1, T + 2, d, seed=s) for s in (1, 2))
    cu = torch.cat([torch.zeros(1, dtype=torch.int64), new.cumsum(0)]).int().cuda()
    _append(api, cache, None, k, v, 0, cu=cu, max_new=3)
    b = torch.repeat_interleave(torch.arange(B), new)
    j = torch.tensor(lens)[b] - new[b] + torch.arange(T) - cu[:-1].cpu()[b]
    page = cache.table.cpu()[b, 0].long().cuda()
    assert torch.equal(cache.c["k"][page, 0, j.cuda()], k[0, :T]) and torch.equal(cache.c["v"][page, 0, j.cuda()], v[0, :T])
    assert int((~torch.isnan(cache.c["k"][..., 0])).sum()) == T
    ko, vo = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    api.kv_read(api.make_kv_params(cache.c, cache.table, cache.kv_len, k=ko, v=vo, cu_seqlens=cu, max_new=3), ko, vo)
    assert torch.equal(ko[:, :T], k[:, :T]) and torch.equal(vo[:, :T], v[:, :T]) and torch.all(ko[:, T:] == 7.0)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_append_in_place_and_parts(api, dtype):
    """q_out == q and k_out == k; queries alone; keys and values alone; no k_out."""
    n, d = 21, 128
    for interleaved in (False, True):
        cache = Cache(api, [n, 300], 2, d, dtype, False, 16, seed=3)
        q, k, v = (_randn(2, H, n, d, seed=s, dtype=dtype) for H, s in ((4, 1), (2, 2), (2, 3)))
        qo, ko, f = _append(api, cache, q, k, v, d, interleaved)
        pool = _storage(cache)
        q2, k2 = q.clone(), k.clone()
        p = api.make_kv_params(cache.c, cache.table, cache.kv_len, q=q2, k=k2, v=v, out=q2, k_out=k2, rot_dim=d, rot_interleaved=interleaved)
        api.kv_append(p, q2, k2, v, f, None, q2, k2)
        assert torch.equal(q2, qo) and torch.equal(k2, ko)
        empty = Cache(api, [n, 300], 2, d, dtype, False, 16, seed=3)
        q3, _, _ = _append(api, empty, q, None, None, d, interleaved)
        assert torch.equal(q3, qo) and torch.isnan(empty.c["k"]).all()
        _append(api, empty, None, k, v, d, interleaved, k_out=False)
        assert all(torch.equal(a.nan_to_num(), b.nan_to_num()) for a, b in zip(_storage(empty), pool))


@pytest.mark.parametrize("d", [64, 128])
def test_append_fp4_codes(api, d):
    """Every group shape of the 4-bit format: ties, the borders of the scale, zeros, tiny and huge values, infinities and NaN."""
    vals = [0.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, 7.03125, 6.0, -0.25, -5.0, 1e-38, 3e38, 2.0 ** -120, 2.0 ** -119 * 7, 9e-41]
    rows = []
    for top in (7.0, 6.0, 7.03125, 4.0, 8.0, 3.5, 2.0 ** -118, 2.0 ** -125, 2.0 ** 127 * 1.9, 0.0, math.inf, -math.inf, math.nan):
        for scale in (1.0, 2.0 ** -10, 2.0 ** 20):
            x = torch.tensor(vals[:13] + [0.0] * 19, dtype=torch.float64)
            x = x * (abs(top) / 7.03125 if math.isfinite(top) else 1.0) * scale
            x[-1] = top * scale if abs(top * scale) < 3.3e38 or not math.isfinite(top) else top
            rows.append(x)
    x = torch.stack(rows + [torch.tensor(vals + [0.0] * 14, dtype=torch.float64)]).repeat(1, d // 32)
    x = torch.cat([x, -x, torch.roll(x, 5, dims=1)]).to(BF)                   # [tokens, d]
    n = x.shape[0]
    v = x.cuda()[None, None].contiguous()
    cache = Cache(api, [n], 1, d, BF, True, 16, seed=1)
    _append(api, cache, None, v, v, 0)
    want = fp4_values(*fp4_pack(x.double()))
    for key in ("k", "v"):
        got = cache.rows(key, 0, 0, n)[0].cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(), want.nan_to_num())
    ko, vo = torch.empty_like(v), torch.empty_like(v)
    api.kv_read(api.make_kv_params(cache.c, cache.table, cache.kv_len, k=ko, v=vo), ko, vo)
    assert torch.equal(ko[0, 0].double().cpu().nan_to_num(), want.nan_to_num()) and torch.equal(torch.isnan(vo[0, 0]).cpu(), torch.isnan(want))


@pytest.mark.parametrize("dtype,fp4,d", FORMATS)
def test_read(api, dtype, fp4, d):
    """Rows back, with tokens before the start, pages that are not there and rows of nobody; K or V alone."""
    lens, new, page = [70, 3, 0, 200], [70, 5, 2, 31], 16
    cache = Cache(api, lens, 2, d, dtype, fp4, page, seed=1, views=True).fill()
    K = [cache.rows("k", b, 0, x) if x else None for b, x in enumerate(lens)]
    V = [cache.rows("v", b, 0, x) if x else None for b, x in enumerate(lens)]
    cache.table[0, 1] = -1
    cu = torch.tensor([0] + new).cumsum(0).int().cuda()
    T = sum(new) + 3
    for both in (True, False):
        ko = torch.full((T, 2, d + 16), 7.0, dtype=dtype, device="cuda")[..., :d].transpose(0, 1)
        vo = torch.full((2, T, d), 7.0, dtype=dtype, device="cuda")
        p = api.make_kv_params(cache.c, cache.table, cache.kv_len, k=ko, v=vo, cu_seqlens=cu, max_new=70)
        api.kv_read(p, ko if both else None, vo)
        at = 0
        for b, (ln, n) in enumerate(zip(lens, new)):
            for got, src in ((ko, K), (vo, V)):
                if got is ko and not both:
                    continue
                want = torch.zeros(2, n, d, dtype=torch.float64, device="cuda")
                m = min(n, ln)
                if m:
                    want[:, n - m:] = src[b][:, ln - m:]
                if b == 0:
                    want[:, 16:32] = 0
                assert torch.equal(got[:, at:at + n].double(), want)
            at += n
        assert torch.all(vo[:, at:] == 7.0) and torch.all(ko[:, at:] == 7.0)
        assert both or torch.all(ko == 7.0)


# ------------------------------------------------------------------ together, streams, graphs
@pytest.mark.parametrize("fp4", [False, True])
def test_prompt_then_tokens(api, fp4):
    """A prompt is appended, prefilled and answered token by token: every output against attention in 64 bits over the rotated
    keys of the whole sequence (from 4 bits: over the cached values)."""
    Hq, Hkv, d, n, more = 8, 2, 128, 400, 5
    total = n + more
    q, k, v = (_randn(1, H, total, d, seed=s) for H, s in ((Hq, 1), (Hkv, 2), (Hkv, 3)))
    f = torch.pow(500000.0, -torch.arange(64, dtype=torch.float64) / 64).float().cuda()
    cache = Cache(api, [total], Hkv, d, BF, fp4, 16, seed=1)
    pos = torch.arange(total, device="cuda")
    step = lambda t, a, b: t[:, :, a:b].contiguous()
    outs, lses = [], []
    for a, b in [(0, n)] + [(i, i + 1) for i in range(n, total)]:
        cache.kv_len.fill_(b)
        qs, ks, vs = step(q, a, b), step(k, a, b), step(v, a, b)
        qo, ko, _ = _append(api, cache, qs, ks, vs, d, inv_freq=f)
        if a == 0:
            p = api.make_params(api.Config(theta=math.inf), qo, ko, vs)
            o, lse = torch.empty_like(qo), torch.empty(Hq * n, device="cuda")
            ws = torch.empty(api.anchor_sizes(p).prefill_ws_bytes, dtype=torch.uint8, device="cuda")
            api.anchor_attention_prefill(p, qo, ko, vs, o, lse, None, ws)
            mine, ml = _attn(api, cache, qo)
            if not fp4:                            # the same rows from the cache
                assert float((mine.double() - o.double()).abs().max()) <= 2e-2
                assert float((ml.flatten() - lse).abs().max()) <= 1e-3
        else:
            o, lse = _attn(api, cache, qo)
        outs.append(o)
        lses.append(lse.view(1, Hq, b - a))
    out, lse = torch.cat(outs, dim=2)[0], torch.cat(lses, dim=2)[0]
    Q = rotate(q[0], pos, f, False).to(BF).double()
    K, V = rotate(k[0], pos, f, False).to(BF).double(), v[0].double()
    for lo, hi in ((0, n), (n, total)):
        if fp4 and lo:
            K, V = cache.rows("k", 0, 0, total), cache.rows("v", 0, 0, total)
        want, wl, A, size = attend(Q[:, lo:hi], K[:, :hi], V[:, :hi], lo, 1 / math.sqrt(d))
        to, tl = tolerances(want, A, size, wl, hi, d, BF)
        assert bool(((out[:, lo:hi].double() - want).abs() <= 2 * to + 2.0 ** -8 * A).all())     # q, k: a step of bf16 at a tie
        assert bool(((lse[:, lo:hi].double() - wl).abs() <= tl + 2e-3).all())


@pytest.mark.parametrize("dtype,fp4", [(BF, False), (BF, True), (F32, False)])
def test_captured_step_replays(api, dtype, fp4):
    """A decode step captured into a graph, replayed with eager work in between and with lengths and inputs that changed in place."""
    B, Hq, Hkv, d = 3, 8, 2, 128
    room = [900, 33, 400]
    cache = Cache(api, room, Hkv, d, dtype, fp4, 16, seed=4).fill()
    q, k, v = (_randn(B, H, 1, d, seed=s, dtype=dtype) for H, s in ((Hq, 1), (Hkv, 2), (Hkv, 3)))
    f = torch.rand(d // 2, device="cuda")
    qo, out = torch.empty_like(q), torch.empty_like(q)
    lse = torch.empty(B * Hq, device="cuda")
    pa = api.make_kv_params(cache.c, cache.table, cache.kv_len, q=q, k=k, v=v, out=qo, rot_dim=d)
    pt = api.make_kv_params(cache.c, cache.table, cache.kv_len, q=qo, out=out)
    ws = torch.empty(api.kv_attn_workspace_bytes(pt), dtype=torch.uint8, device="cuda")

    def step():
        api.kv_append(pa, q, k, v, f, None, qo)
        api.kv_attn(pt, qo, out, lse, ws)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for t, lens in enumerate(([900, 33, 400], [17, 1, 399], [0, 32, 64], [555, 20, 1])):
        cache.kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
        q.copy_(_randn(B, Hq, 1, d, seed=20 + t, dtype=dtype))
        k.copy_(_randn(B, Hkv, 1, d, seed=40 + t, dtype=dtype))
        step()
        want = [out.clone(), lse.clone()] + _storage(cache)
        out.fill_(7.0), lse.fill_(7.0), ws.fill_(0xff)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, [out, lse] + _storage(cache)):
            assert torch.equal(a.float().nan_to_num(), b.float().nan_to_num())


@pytest.mark.parametrize("dtype,fp4", [(BF, False), (BF, True), (F32, False)])
def test_captured_chunk_replays(api, dtype, fp4):
    """A packed chunk captured into a graph and replayed with other splits of the same rows, other lengths and other inputs."""
    Hq, Hkv, d, total = 8, 2, 128, 400
    cache = Cache(api, [3000, 500, 400], Hkv, d, dtype, fp4, 16, seed=4).fill()
    q, k, v = (_randn(H, total, d, seed=s, dtype=dtype) for H, s in ((Hq, 1), (Hkv, 2), (Hkv, 3)))
    f = torch.rand(d // 2, device="cuda")
    cu = torch.tensor([0, 100, 150, 390], dtype=torch.int32, device="cuda")
    qo, out, ko, vo = (torch.empty_like(x) for x in (q, q, k, v))
    lse = torch.empty(Hq * total, device="cuda")
    kw = dict(cu_seqlens=cu, max_new=300)
    pa = api.make_kv_params(cache.c, cache.table, cache.kv_len, q=q, k=k, v=v, out=qo, rot_dim=d, **kw)
    pt = api.make_kv_params(cache.c, cache.table, cache.kv_len, q=qo, out=out, **kw)
    pr = api.make_kv_params(cache.c, cache.table, cache.kv_len, k=ko, v=vo, **kw)
    ws = torch.empty(api.kv_attn_workspace_bytes(pt), dtype=torch.uint8, device="cuda")

    def step():
        api.kv_append(pa, q, k, v, f, None, qo)
        api.kv_attn(pt, qo, out, lse, ws)
        api.kv_read(pr, ko, vo)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for t, (ends, lens) in enumerate((([0, 100, 150, 390], [3000, 500, 400]), ([0, 0, 300, 400], [77, 301, 100]), ([0, 1, 2, 3], [2900, 0, 399]),
                                      ([0, 300, 300, 320], [300, 400, 20]))):
        cache.kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
        cu.copy_(torch.tensor(ends, dtype=torch.int32))
        q.copy_(_randn(Hq, total, d, seed=20 + t, dtype=dtype))
        k.copy_(_randn(Hkv, total, d, seed=40 + t, dtype=dtype))
        results = [out, lse, ko, vo]
        for x in results:
            x.fill_(7.0)
        step()
        want = [x.clone() for x in results] + _storage(cache)
        for x in results:
            x.fill_(7.0)
        ws.fill_(0xff)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.all(out[:, ends[-1]:] == 7.0)
        for a, b in zip(want, results + _storage(cache)):
            assert torch.equal(a.float().nan_to_num(), b.float().nan_to_num())


@pytest.mark.parametrize("n", [1, 90])
@pytest.mark.parametrize("dtype,fp4", [(BF, False), (BF, True), (F32, False)])
def test_two_streams_and_repeats(api, dtype, fp4, n):
    """Two calls at once, each with its workspace, on streams other than the tensors' own: the bits of calls one after the other."""
    d = 128
    caches = [Cache(api, lens, 2, d, dtype, fp4, 32, seed=s).fill(seed=s) for s, lens in ((1, [3000, 5]), (2, [1200, 2500]))]
    qs = [_randn(2, 8, n, d, seed=s, dtype=dtype) for s in (1, 2)]
    want = [_attn(api, c, q) for c, q in zip(caches, qs)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        outs = []
        for c, q, st in zip(caches, qs, streams):
            with torch.cuda.stream(st):
                outs.append(_attn(api, c, q, stream=st))
        torch.cuda.synchronize()
        for a, b in zip(want, outs):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ------------------------------------------------------------------ calls of the largest descriptions
@pytest.mark.parametrize("dtype,fp4,d", [(BF, False, 128), (BF, True, 128), (BF, False, 64), (F32, False, 64)])
def test_long_table_many_sequences(api, dtype, fp4, d):
    """A packed step whose description allows far more than is there: 128 sequences of up to 8192 new tokens over a table of 131072."""
    Hq, Hkv, page, N = 32, 8, 16, 8192
    new = [i % 3 for i in range(127)] + [150]
    lens = [n + (i * 37) % 300 for i, n in enumerate(new)]
    T = sum(new)
    cache = Cache(api, lens, Hkv, d, dtype, fp4, page, seed=5, room=131072 // page).fill()
    x = _randn(N + 100, Hq + 2 * Hkv, d, seed=5, dtype=dtype).transpose(0, 1)
    q, k, v = x.split([Hq, Hkv, Hkv])
    ends = torch.tensor([0] + new).cumsum(0)
    cu = ends.int().cuda()
    qo, ko, _ = _append(api, cache, q, k, v, 0, cu=cu, max_new=N)
    assert torch.equal(qo[:, :T], q[:, :T]) and torch.all(qo[:, T:] == 7.0)
    back_k, back_v = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    api.kv_read(api.make_kv_params(cache.c, cache.table, cache.kv_len, k=back_k, v=back_v, cu_seqlens=cu, max_new=N), back_k, back_v)
    out, lse = _attn(api, cache, q, cu, N)
    for b, n in enumerate(new):
        sl = slice(int(ends[b]), int(ends[b + 1]))
        if n == 0:
            continue
        for got, src, key in ((back_k, k, "k"), (back_v, v, "v")):
            want = fp4_values(*fp4_pack(src[:, sl])).cuda() if fp4 else src[:, sl].double()
            assert torch.equal(got[:, sl].double(), want) and torch.equal(cache.rows(key, b, lens[b] - n, n), want)
        want, wl, A, size = attend(q[:, sl].double(), cache.rows("k", b, 0, lens[b]), cache.rows("v", b, 0, lens[b]), lens[b] - n, 1 / math.sqrt(d))
        to, tl = tolerances(want, A, size, wl, lens[b], d, dtype)
        assert bool(((out[:, sl].double() - want).abs() <= to).all()) and bool(((lse[:, sl].double() - wl).abs() <= tl).all()), b
    assert torch.all(back_k[:, T:] == 7.0) and torch.all(out[:, T:] == 7.0) and torch.all(lse[:, T:] == 7.0)


@pytest.mark.parametrize("dtype,d", [(F32, 32), (BF, 64)])
def test_units_beyond_32_bits(api, dtype, d):
    """A table of 2^30 tokens and 256 tiles of rows: keys in units of 128 would be 2^31, so every tile is taken whole."""
    n, length = 4096, 5000
    cache = Cache(api, [length], 1, d, dtype, False, 1 << 20, seed=1, room=1024, spare=0).fill()
    q = _randn(1, 4, n, d, seed=1, dtype=dtype)
    p = api.make_kv_params(cache.c, cache.table, cache.kv_len, q=q, out=q)
    assert api.kv_attn_workspace_bytes(p) == 0
    _check_attn(api, cache, q, [n])


@pytest.mark.parametrize("dtype,fp4,d", FORMATS)
def test_rows_beyond_the_most(api, dtype, fp4, d):
    """Of a packed sequence with more rows than max_new the first max_new take part, as its last tokens; the others stay as they were."""
    new, lens, most = [5, 70, 3], [50, 300, 3], 40
    cache = Cache(api, lens, 2, d, dtype, fp4, 16, seed=1).fill()
    q = _randn(8, 78, d, seed=1, dtype=dtype)
    cu = torch.tensor([0, 5, 75, 78], dtype=torch.int32, device="cuda")
    out, lse = _attn(api, cache, q, cu, most)
    at = 0
    for b, n in enumerate(new):
        m = min(n, most)
        sl = slice(at, at + m)
        want, wl, A, size = attend(q[:, sl].double(), cache.rows("k", b, 0, lens[b]), cache.rows("v", b, 0, lens[b]), lens[b] - m, 1 / math.sqrt(d))
        to, tl = tolerances(want, A, size, wl, lens[b], d, dtype)
        assert bool(((out[:, sl].double() - want).abs() <= to).all()) and bool(((lse[:, sl].double() - wl).abs() <= tl).all()), b
        assert torch.all(out[:, at + m:at + n] == 7.0) and torch.all(lse[:, at + m:at + n] == 7.0)
        at += n
