"""Host-only checks of the paged cache: argument checks of the C entry points and of the binding, struct layout, the 4-bit format's
code compiled for the host against the definition."""
import ctypes
import os
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def api():
    from paper_2505_23520_amd import api as _api
    return _api


def _three(a, b, c):
    return (ctypes.c_int64 * 3)(a, b, c)


def _params(api, **kw):
    p = api.aa_kv_params()
    p.B, p.Hq, p.Hkv, p.N, p.d, p.dtype, p.format = 2, 8, 2, 1, 128, api.AA_BF16, api.AA_KV_PLAIN
    p.page_size, p.n_pages, p.max_pages, p.table_stride, p.causal, p.rot_dim = 16, 10, 4, 4, 1, 128
    for f in ("q_stride", "o_stride"):
        setattr(p, f, _three(8 * 128, 128, 128))
    for f in ("k_stride", "v_stride", "ko_stride"):
        setattr(p, f, _three(2 * 128, 128, 128))
    for f in ("kc_stride", "vc_stride"):
        setattr(p, f, _three(2 * 16 * 128, 16 * 128, 128))
    for f in ("ks_stride", "vs_stride"):
        setattr(p, f, _three(2 * 4 * 16, 4 * 16, 16))
    p.kc = p.vc = p.ks = p.vs = p.page_table = p.kv_len = 4096        # never dereferenced on the host
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def test_struct_layout(api, tmp_path):
    """aa_kv_params of the binding is the header's, field by field; the header stays plain C99."""
    src, exe = tmp_path / "h.c", str(tmp_path / "h")
    names = [f[0] for f in api.aa_kv_params._fields_]
    src.write_text('#include "anchor_attention.h"\n#include <stdio.h>\nint main(void) {\nprintf("%zu\\n", sizeof(aa_kv_params));\n'
                   + "".join('printf("%%zu\\n", offsetof(aa_kv_params, %s));\n' % n for n in names) + "return 0; }\n")
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Wextra", "-pedantic", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe])
    got = [int(x) for x in subprocess.check_output([exe], text=True).split()]
    assert got == [ctypes.sizeof(api.aa_kv_params)] + [getattr(api.aa_kv_params, n).offset for n in names]


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), -1), (dict(Hq=7), -1), (dict(Hkv=0), -1), (dict(N=0), -1), (dict(d=0), -1), (dict(dtype=2), -1), (dict(format=2), -1),
    (dict(page_size=0), -1), (dict(page_size=24), -1), (dict(page_size=-16), -1), (dict(n_pages=0), -1), (dict(max_pages=0), -1),
    (dict(max_len=-1), -1), (dict(causal=2), -1), (dict(rot_dim=-16), -1), (dict(rot_dim=256), -1), (dict(rot_dim=7), -1),
    (dict(rot_interleaved=2), -1), (dict(softmax_scale=float("nan")), -1), (dict(softmax_scale=-1.0), -1), (dict(table_stride=3), -1),
    (dict(page_table=None), -1), (dict(kv_len=None), -1), (dict(cu_seqlens=4096, total_tokens=0), -1),
    (dict(cu_seqlens=4096, total_tokens=3, N=4), -1), (dict(kc=None), -1), (dict(vc=4100), -1), (dict(format=1, ks=None), -1),
    (dict(format=1, vs=4104), -1), (dict(kc_stride=_three(4096, 2048, 100)), -1), (dict(vc_stride=_three(4096, 2048, 132)), -1),
    (dict(kc_stride=_three(-4096, 2048, 128)), -1), (dict(kc_stride=_three(0, 2048, 128)), -1), (dict(vc_stride=_three(1 << 59, 2048, 128)), -1),
    (dict(format=1, ks_stride=_three(128, 64, 8)), -1), (dict(format=1, ks_stride=_three(128, 72, 16)), -1),
    (dict(d=96, rot_dim=0), -2), (dict(d=256), -2), (dict(d=32, rot_dim=0), -2), (dict(page_size=8), -2), (dict(page_size=1 << 21), -2), (dict(rot_dim=24), -2),
    (dict(format=1, dtype=0), -2), (dict(B=65536), -2), (dict(Hq=65536, Hkv=1), -2), (dict(B=65535, N=65535), -2), (dict(B=256, N=65536), -2), (dict(B=1, N=100, cu_seqlens=4096, total_tokens=1 << 24), -2), (dict(N=2**30, B=1), -2),
    (dict(max_pages=2**26 + 1, table_stride=2**26 + 1), -2), (dict(kc_stride=_three(1 << 33, 1 << 32, 1 << 25)), -2),
    (dict(kc_stride=_three(1 << 33, 1 << 32, 1 << 15), page_size=1 << 15), -2),
    (dict(format=1, vs_stride=_three(1 << 33, 1 << 32, 1 << 28)), -2),
])
def test_rejects_bad_params(api, kw, code):
    """Before anything is enqueued: no GPU here, and none is asked for."""
    n = ctypes.c_size_t()
    p = _params(api, **kw)
    assert api._lib.kv_attn_workspace_bytes(ctypes.byref(p), ctypes.byref(n)) == code
    assert api._lib.kv_append(ctypes.byref(p), 4096, 4096, 4096, 4096, None, 4096, None, None) == code
    assert api._lib.kv_attn(ctypes.byref(p), 4096, 4096, None, 4096, 1 << 40, None) == code
    assert api._lib.kv_read(ctypes.byref(p), 4096, 4096, None) == code


def test_rejects_bad_calls(api):
    lib, ref = api._lib, ctypes.byref
    p = _params(api)
    ok = 4096
    E = api.AA_EINVAL
    assert lib.kv_append(None, ok, ok, ok, ok, None, ok, None, None) == E
    for args in ((None, None, None, ok, None, None, None),       # nothing to do
                 (ok, ok, ok, ok, None, None, None),             # queries without q_out
                 (None, ok, ok, ok, None, ok, None),             # q_out without queries
                 (ok, ok, None, ok, None, ok, None), (ok, None, ok, ok, None, ok, None), (ok, None, None, ok, None, ok, ok),
                 (ok, ok, ok, None, None, ok, None),             # rotation without frequencies
                 (ok + 2, ok, ok, ok, None, ok, None), (ok, ok + 8, ok, ok, None, ok, None), (ok, ok, ok, ok, None, ok + 4, None)):
        assert lib.kv_append(ref(p), *args, None) == E, args
    for field, st in (("q_stride", (1024, 128, 4)), ("k_stride", (256, -128, 128)), ("v_stride", (1 << 40, 128, 128)), ("o_stride", (0, 128, 128)),
                      ("o_stride", (1024, 64, 128)), ("ko_stride", (256, 0, 128))):
        q = _params(api, **{field: _three(*st)})
        assert lib.kv_append(ref(q), ok, ok, ok, ok, None, ok, ok, None) == E, field
    q = _params(api, N=3, o_stride=_three(8 * 128, 128, 64))
    assert lib.kv_attn(ref(q), ok, ok, None, ok, 1 << 40, None) == E                       # rows of out that overlap
    assert lib.kv_attn(ref(p), None, ok, None, ok, 1 << 40, None) == E
    assert lib.kv_attn(ref(p), ok, ok + 2, None, ok, 1 << 40, None) == E
    assert lib.kv_read(ref(p), None, None, None) == E
    assert lib.kv_attn_workspace_bytes(ref(p), None) == E


def test_binding_rejects(api):
    c = api.alloc_kv_cache(6, 2, 16, 128, device="cpu")
    c4 = api.alloc_kv_cache(6, 2, 16, 128, format=api.AA_KV_FP4, device="cpu")
    table, lens = torch.zeros(3, 2, dtype=torch.int32), torch.ones(3, dtype=torch.int32)
    q, k = torch.zeros(3, 8, 1, 128, dtype=torch.bfloat16), torch.zeros(3, 2, 1, 128, dtype=torch.bfloat16)
    p = api.make_kv_params(c, table, lens, q=q, k=k, v=k, out=q)
    assert (p.B, p.Hq, p.Hkv, p.N, p.d, p.page_size, p.max_pages, p.format) == (3, 8, 2, 1, 128, 16, 2, api.AA_KV_PLAIN)
    assert api.make_kv_params(c4, table, lens, q=q, out=q).format == api.AA_KV_FP4
    bad = [dict(), dict(q=q[:2]), dict(q=q, out=q.float()), dict(q=q, k=k[:, :1]), dict(q=q.half()), dict(q=q[0]),
           dict(q=q.transpose(2, 3).contiguous().transpose(2, 3)[..., ::2]), dict(q=q, max_new=2), dict(q=q[..., :64], k=k[..., :64])]
    for kw in bad:
        with pytest.raises(ValueError):
            api.make_kv_params(c, table, lens, **kw)
    for cache, t, n in ((c, table.long(), lens), (c, table, lens[:2]), (c, table, lens.float()), (dict(c, v=c["v"][:5]), table, lens),
                        (dict(c, k=c["k"].float()), table, lens), (dict(c4, v_scale=c4["v_scale"][:, :, :2]), table, lens)):
        with pytest.raises(ValueError):
            api.make_kv_params(cache, t, n, q=q, out=q)
    f = torch.ones(64)
    p = api.make_kv_params(c, table, lens, q=q, k=k, v=k, out=q, rot_dim=128)
    for args in ((q, k, k, f[:32], None, q), (q, k, k, f.double(), None, q), (q, k, k, None, None, q), (q, k, k, f, torch.zeros(3), q),
                 (q, k, k, f, torch.zeros(2, dtype=torch.int32), q), (q.expand(3, 8, 1, 128)[:, ::2], k, k, f, None, q)):
        with pytest.raises(ValueError):
            api.kv_append(p, *args)


def test_params_let_their_tensors_go(api):
    """A description keeps its tensors as long as it lives, and no longer: a server makes one for every packed step."""
    import weakref
    c = api.alloc_kv_cache(6, 2, 16, 128, device="cpu")
    q, lens = torch.zeros(1, 8, 1, 128, dtype=torch.bfloat16), torch.ones(1, dtype=torch.int32)
    p = api.make_kv_params(c, torch.zeros(1, 2, dtype=torch.int32), lens, q=q, out=q)
    with pytest.raises(ValueError):
        api.kv_attn(p, q, q)                             # (no GPU tensors)
    seen = [weakref.ref(x) for x in (q, lens, p)]
    del q, lens
    assert all(r() is not None for r in seen)
    del p
    assert all(r() is None for r in seen)


def test_binding_takes_one_entry_of_any_stride(api):
    """A batch of one whose length, row ends or only page are a column of another array: the stride of one entry is never used."""
    c = api.alloc_kv_cache(6, 2, 16, 128, device="cpu")
    q = torch.zeros(1, 8, 1, 128, dtype=torch.bfloat16)
    many = torch.arange(12, dtype=torch.int32).view(4, 3)
    lens, table = many.t()[:1, 2], many.t()[1:2, :1]
    lens = torch.as_strided(lens, (1,), (3,), lens.storage_offset())
    assert table.stride(-1) != 1 and lens.stride(0) != 1
    p = api.make_kv_params(c, table, lens, q=q, out=q)
    assert (p.B, p.max_pages, p.table_stride, p.kv_len) == (1, 1, 1, lens.data_ptr()) and p.page_table == table.data_ptr()
    for t, n in ((many.t()[:1, :3], lens), (table, many[:2, 0])):
        with pytest.raises(ValueError):
            api.make_kv_params(c, t, n, q=q, out=q)


def test_fp4_scale_on_the_host(tmp_path):
    """fp4_scale_byte against every exponent tried out."""
    from kv_util import fp4_pack
    src, exe = tmp_path / "f.cpp", str(tmp_path / "f")
    src.write_text('''#include "%s/paper_2505_23520_amd/csrc/aa_kv_fp4.h"
#include <stdio.h>
int main() {
    unsigned u;
    while (fread(&u, 4, 1, stdin) == 1) printf("%%d\\n", aa::fp4_scale_byte(u));
}''' % ROOT)
    subprocess.check_call(["g++", "-O2", "-std=c++17", str(src), "-o", exe])
    gen = torch.Generator().manual_seed(1)
    x = torch.randn(400, generator=gen).abs()
    x = torch.cat([x, x * 2.0 ** -125, x * 2.0 ** 126, 7 * torch.exp2(torch.arange(-125.0, 126.0)), torch.tensor([0.0, float("inf"), float("nan"), 1e-45])])
    x = torch.cat([x, torch.nextafter(x, torch.tensor(float("inf"))), torch.nextafter(x, torch.tensor(0.0))])
    got = subprocess.run([exe], input=x.numpy().tobytes(), capture_output=True, check=True).stdout.split()
    scales = fp4_pack(torch.stack([x.double()] + [torch.zeros(x.numel(), dtype=torch.float64)] * 31, dim=1))[1]
    assert [int(t) for t in got] == scales[:, 0].tolist()


def test_series_on_the_host(tmp_path):
    """The sine and cosine series evaluated in 64 bits of mantissa: what they leave out stays within their bounds (and 2^-60 for the evaluation's
    own roundings) up to pi / 4."""
    src, exe = tmp_path / "s.cpp", str(tmp_path / "s")
    src.write_text('''#include "%s/paper_2505_23520_amd/csrc/aa_kv_turn.h"
#include <cmath>
#include <stdio.h>
int main() {
    static_assert(__LDBL_MANT_DIG__ >= 64, "");
    long double worst[2] = {0, 0};
    for (int i = -20000; i <= 20000; ++i) {
        const long double x = i / 20000.0L * 0.78539816339744830962L;
        long double c, s;
        for (int k = 0; k < 2; ++k) {
            if (k) aa::series64(x, &c, &s); else aa::series32(x, &c, &s);
            const long double ec = fabsl(c - cosl(x)) / cosl(x), es = i ? fabsl(s - sinl(x)) / fabsl(sinl(x)) : fabsl(s);
            if (ec > worst[k]) worst[k] = ec;
            if (es > worst[k]) worst[k] = es;
        }
    }
    printf("%%La %%La\\n", worst[0], worst[1]);
    return worst[0] > 0x1p-24L + 0x1p-60L ? 1 : worst[1] > 0x1p-54L + 0x1p-60L ? 2 : 0;
}''' % ROOT)
    subprocess.check_call(["g++", "-O1", "-std=c++17", str(src), "-o", exe])
    assert subprocess.run([exe]).returncode == 0


def test_deal_on_the_host(tmp_path):
    """Every unit belongs to exactly one work-group, the work-groups' numbers of units differ by one at most, and the places of the
    shares of a tile are all different, whatever the lengths."""
    src, exe = tmp_path / "d.cpp", str(tmp_path / "d")
    src.write_text('''#include "%s/paper_2505_23520_amd/csrc/aa_kv_deal.h"
#include <stdio.h>
int main() {
    unsigned total, groups;
    while (scanf("%%u %%u", &total, &groups) == 2) {
        aa::Deal d;
        d.each = total / groups;
        d.more = total - d.each * groups;
        if (aa::deal_start(d, 0) != 0 || aa::deal_start(d, groups) != total) return 1;
        for (unsigned g = 0; g < groups; ++g) {
            const unsigned a = aa::deal_start(d, g), b = aa::deal_start(d, g + 1);
            if (b - a != d.each && b - a != d.each + 1) return 2;
            if (a < b && (aa::deal_group(d, a) != g || aa::deal_group(d, b - 1) != g)) return 3;
        }
        // tiles of many lengths along the line: each work-group leaves at most one share in each of its two places
        static int used[4096];
        for (unsigned i = 0; i < 2 * groups; ++i) used[i] = 0;
        unsigned first = 0, units = 1;
        while (first < total) {
            if (first + units > total) units = total - first;
            const unsigned g0 = aa::deal_group(d, first), g1 = aa::deal_group(d, first + units - 1);
            for (unsigned g = g0; g0 < g1 && g <= g1; ++g) {
                const unsigned t = g == g0 ? 0 : aa::deal_start(d, g) - first;
                const int place = aa::deal_place((int)g, (int)t);
                if (place < 0 || place >= (int)(2 * groups) || used[place]++) return 4;
                if (place != aa::deal_place((int)(g0 + (g - g0)), (int)(g - g0))) return 5;          // how the joining kernel counts them
            }
            first += units;
            units = units * 7 %% 23 + 1;
        }
    }
    if (aa::deal_units(0, 0) != 0 || aa::deal_units(5000, 0) != 0 || aa::deal_units(0, 3) != 1 || aa::deal_units(128, 1) != 1 ||
        aa::deal_units(129, 1) != 2 || aa::deal_units(1 << 30, 1) != 1 << 23) return 6;
    return 0;
}''' % ROOT)
    subprocess.check_call(["g++", "-O2", "-std=c++17", str(src), "-o", exe])
    pairs = [(t, g) for t in list(range(1, 200)) + [511, 512, 513, 767, 1000, 4097, 100003] for g in (1, 2, 7, 8, 256, 512, 768, 1024)]
    run = subprocess.run([exe], input="".join("%d %d\n" % p for p in pairs), text=True)
    assert run.returncode == 0


def test_cache_kernels_honour_nans():
    """A NaN among a row's keys or values has to reach its result and lse: no source of the cache is compiled as if there were none."""
    from paper_2505_23520_amd import build
    relaxed = {"-fno-honor-nans", "-fno-honor-infinities", "-ffinite-math-only", "-ffast-math", "-Ofast"}
    for source in build.CACHE_SOURCES:
        assert not relaxed & set(build.FLAGS + build.EXTRA.get(source, [])), source


@pytest.fixture(scope="module")
def compiled(tmp_path_factory):
    """The cache's kernel sources compiled as the build does: source -> (the compiler's report on registers, assembly)."""
    from paper_2505_23520_amd import build
    out = {}
    for source in sorted(set(build.CACHE_SOURCES) - {"aa_kv_api.hip"}):
        asm = tmp_path_factory.mktemp("s") / "x.s"
        cmd = ["hipcc", *build.FLAGS, *build.EXTRA.get(source, []), "--cuda-device-only", "-S", "-Rpass-analysis=kernel-resource-usage",
               os.path.join(build.CSRC, source), "-o", str(asm)]
        out[source] = (subprocess.run(cmd, capture_output=True, text=True, check=True).stderr, asm.read_text())
    return out


def test_cache_kernels_do_not_spill(compiled):
    """A spilled register's reload is a vector-memory load, and the wait for it waits for the tiles in flight.  As many waves per SIMD
    as the dealing of the keys counts on."""
    import re
    want = {"aa_kv_append.hip": lambda name: 3, "aa_kv_chunk.hip": lambda name: 3,
            "aa_kv_attn.hip": lambda name: 1 if "join" in name else {"1": {"128": 3 if "ILi2E" in name else 2, "64": 3, "32": 4},
                                                                     "2": {"128": 2 if "ILi2E" in name else 1, "64": 2, "32": 2}, "4": {"64": 1, "32": 1}}
            [re.search(r"ILi\dELi(\d+)ELi(\d)E", name).group(2)][re.search(r"ILi\dELi(\d+)ELi(\d)E", name).group(1)]}
    assert sorted(want) == sorted(compiled)
    for source, waves in want.items():
        report = compiled[source][0]
        names = re.findall(r"Function Name: (\S+)", report)
        spills = [int(x) for x in re.findall(r"VGPRs Spill: (\d+)", report)]
        occupancy = [int(x) for x in re.findall(r"Occupancy \[waves/SIMD\]: (\d+)", report)]
        assert len(names) >= 2 and len(spills) == len(occupancy) == len(names)
        assert not any(spills) or "append" in source, dict(zip(names, spills))      # (kv_append has nothing in flight across a reload)
        for name, o in zip(names, occupancy):
            assert o >= waves(name), (name, o)


def test_append_and_read_kernels_do_not_spill(compiled):
    """One kernel of kv_append keeps up to 6 registers in scratch memory, by measurement: 4 bits, d = 128, halves, four tokens, three rows in flight."""
    import re
    report = compiled["aa_kv_append.hip"][0]
    names, spills = re.findall(r"Function Name: (\S+)", report), [int(x) for x in re.findall(r"VGPRs Spill: (\d+)", report)]
    assert len(names) == len(spills) and sum("kv_read_kernel" in n for n in names) == 7 and sum("kv_append_kernel" in n for n in names) == 63
    for name, n in zip(names, spills):
        assert n <= (6 if "kv_append_kernelIDF16bLb1ELi128ELi1ELi4ELi3E" in name else 0), (name, n)


# Wait states between a matrix instruction and another instruction that reads or overwrites its result: two (products of floats) or three more
# than its passes.
WAIT_STATES = {"v_mfma_f32_16x16x4_f32": 10, "v_mfma_f32_16x16x32_bf16": 7, "v_mfma_f32_32x32x16_bf16": 11}


def _registers(text):
    import re
    out = set()
    for kind, lo, hi, one in re.findall(r"\b([va])(?:\[(\d+):(\d+)\]|(\d+)\b)", text):
        out |= {(kind, i) for i in (range(int(lo), int(hi) + 1) if lo else [int(one)])}
    return out


def _blocks(asm):
    """(kernel, [(label, [instruction])]) of every kernel."""
    name, blocks = None, None
    for line in asm.splitlines():
        t = line.split(";")[0].strip()
        if t.startswith("_Z") and t.endswith(":"):
            name, blocks = t[:-1], [("", [])]
        elif name and t.startswith(".Lfunc_end"):
            yield name, blocks
            name = None
        elif name and t.startswith(".LBB"):
            blocks.append((t[:-1], []))
        elif name and t and not t.startswith(".") and not t.endswith(":"):
            blocks[-1][1].append(t)


def _too_early(blocks):
    """Instructions that touch a matrix instruction's result before its wait states are over, on any path."""
    at = {label: i for i, (label, _) in enumerate(blocks)}
    state, work, bad = [{} for _ in blocks], list(range(len(blocks))), set()
    while work:
        b = work.pop(0)
        left, ends = dict(state[b]), [b + 1]
        for t in blocks[b][1]:
            op, _, rest = t.partition(" ")
            operands = rest.split(", ")
            touched = set()
            if op.startswith("v_mfma"):
                touched = _registers(", ".join(operands[1:3]))           # (its addend and its result follow without waiting)
            elif op.startswith(("v_", "ds_", "buffer_", "global_", "scratch_", "flat_")):
                touched = _registers(rest)
            if any(r in left for r in touched):
                bad.add(t)
            n = int(rest) + 1 if op == "s_nop" else 1
            left = {r: x - n for r, x in left.items() if x > n}
            if op.startswith("v_mfma"):
                left.update((r, WAIT_STATES[op]) for r in _registers(operands[0]))
            if op.startswith(("s_cbranch", "s_branch")):
                ends.append(at[rest.strip()])
                for r, x in left.items():
                    if state[ends[-1]].get(r, 0) < x:
                        state[ends[-1]][r] = x
                        work.append(ends[-1])
            if op in ("s_branch", "s_endpgm"):
                ends[0] = None
        if ends[0] is not None and ends[0] < len(blocks):
            for r, x in left.items():
                if state[ends[0]].get(r, 0) < x:
                    state[ends[0]][r] = x
                    work.append(ends[0])
    return sorted(bad)


def test_matrix_results_are_waited_for(compiled):
    """The compiler has left the wait out for reads behind a branch (float scores, whose maximum was then taken of older values)."""
    one = [("", ["v_mfma_f32_16x16x4_f32 v[4:7], v0, v1, 0", "s_cbranch_vccz .L1", "s_nop 7"]), (".L1", ["v_add_f32_e32 v8, v9, v7"])]
    assert _too_early(one) == ["v_add_f32_e32 v8, v9, v7"]
    one[1][1].insert(0, "s_nop 8")
    assert _too_early(one) == []
    kernels = 0
    for source in ("aa_kv_attn.hip", "aa_kv_chunk.hip"):
        for name, blocks in _blocks(compiled[source][1]):
            kernels += any(t.startswith("v_mfma") for _, b in blocks for t in b)
            assert not _too_early(blocks), name
    assert kernels == 20


def _accepted(api, p):
    """What the workspace query, kv_append, kv_read and kv_attn say to the description alone: each call has a fault that is looked for after it."""
    n, ref = ctypes.c_size_t(), ctypes.byref(p)
    return (api._lib.kv_attn_workspace_bytes(ref, ctypes.byref(n)), api._lib.kv_append(ref, 4096, None, None, 4096, None, None, None, None),
            api._lib.kv_read(ref, None, None, None), api._lib.kv_attn(ref, None, 4096, None, 4096, 1 << 40, None))


@pytest.mark.parametrize("form", [dict(), dict(format=1), dict(d=64, rot_dim=64), dict(d=64, rot_dim=64, format=1), dict(dtype=0), dict(dtype=0, d=32, rot_dim=32)])
@pytest.mark.parametrize("B,N,rows,room", [(1, 131072, 131072, 1 << 20), (1, 131072, 131072, 1 << 30), (16, 131072, 131200, 131072), (64, 16384, 20000, 131072),
                                           (128, 8192, 9000, 131072), (256, 4096, 5000, 131072), (64, 1 << 20, 1 << 20, 131072), (4000, 1, 4000, 1 << 30),
                                           (64, 100000, (1 << 24) - 1, 1 << 20)])
def test_large_batches_are_taken(api, form, B, N, rows, room):
    """Packed batches with a long table and one long prompt among the sequences, 32 / 8 heads: no entry point has a reason to refuse them."""
    p = _params(api, B=B, N=N, Hq=32, Hkv=8, cu_seqlens=4096, total_tokens=rows, page_size=1024, max_pages=room >> 10, table_stride=room >> 10, **form)
    for f in ("kc_stride", "vc_stride"):
        setattr(p, f, _three(8 * 1024 * 128, 1024 * 128, 128))
    for f in ("ks_stride", "vs_stride"):
        setattr(p, f, _three(8 * 4 * 1024, 4 * 1024, 1024))
    assert _accepted(api, p) == (api.AA_OK, api.AA_EINVAL, api.AA_EINVAL, api.AA_EINVAL)
    p.cu_seqlens, p.N = None, max(1, ((1 << 24) - 1) // B)            # as many rows in a batch as a call may have
    assert _accepted(api, p) == (api.AA_OK, api.AA_EINVAL, api.AA_EINVAL, api.AA_EINVAL)


@pytest.mark.parametrize("kw", [dict(B=65535, Hq=65535, Hkv=65535), dict(Hq=65535, Hkv=1, N=(1 << 24) - 1), dict(Hq=65535, Hkv=65535, N=(1 << 24) - 1),
                                dict(Hq=65535, Hkv=65535, N=(1 << 24) - 1, d=64, rot_dim=0)])
def test_attention_that_cannot_be_counted(api, kw):
    """Tiles of rows beyond 32 bits: refused by the workspace query and by kv_attn, alike; kv_append and kv_read have no tiles."""
    p = _params(api, **dict(dict(B=1), **kw))
    n, ref = ctypes.c_size_t(), ctypes.byref(p)
    assert _accepted(api, p)[:3] == (api.AA_EUNSUPPORTED, api.AA_EINVAL, api.AA_EINVAL)
    for f in ("q_stride", "o_stride"):
        setattr(p, f, _three(1 << 39, 128, 1 << 23))
    assert api._lib.kv_attn(ref, 4096, 4096, None, 4096, 1 << 40, None) == api.AA_EUNSUPPORTED
