"""The decode-step operators' C ABI without a GPU: exports, struct layouts, and every refusal (a rejected call launches
nothing, so the pointers here are host addresses that nothing reads)."""
import ctypes as C
import math
import os
import re
import subprocess

import pytest

from conftest import ROOT

HEADER = os.path.join(ROOT, "include", "ctr_decode.h")


@pytest.fixture(scope="module")
def ctr():
    from paper_2609_16206_gb300 import build
    build.build()
    from paper_2609_16206_gb300 import ctr
    ctr.lib()
    return ctr


def _functions():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    return sorted(set(re.findall(r"^(?:int|size_t)\s+(ctr_\w+)\s*\(", text, flags=re.M)))


def test_both_libraries_export_every_declared_function():
    from paper_2609_16206_gb300 import build
    names = _functions()
    assert names == ["ctr_attention_workspace_bytes", "ctr_kv_append", "ctr_sample", "ctr_tree_attention"]
    for checked in (False, True):
        lib = C.CDLL(build.build(checked=checked))
        for name in names:
            assert hasattr(lib, name), (name, checked)


def test_package_names():
    import paper_2609_16206_gb300 as pkg
    for name in ("ctr_kv_append", "ctr_tree_attention", "ctr_sample", "KvCache", "Rope", "attention_workspace"):
        assert callable(getattr(pkg, name))


def test_struct_layout_matches_header(ctr, tmp_path):
    structs = {"ctr_kv_cache": ctr.CtrKvCache, "ctr_rows": ctr.CtrRows, "ctr_rope": ctr.CtrRope}
    lines = ['#include <stdio.h>', '#include <stddef.h>', f'#include "{HEADER}"', "int main(void){"]
    for cname, py in structs.items():
        lines.append(f'printf("{cname} sizeof %zu\\n", sizeof({cname}));')
        lines += [f'printf("{cname} {f[0]} %zu\\n", offsetof({cname}, {f[0]}));' for f in py._fields_]
    lines += ['printf("c CTR_MAX_NODES %d\\nc CTR_MAX_SEQS %d\\nc CTR_MAX_VOCAB %d\\n", CTR_MAX_NODES, CTR_MAX_SEQS, CTR_MAX_VOCAB);',
              'printf("c CTR_BF16 %d\\nc CTR_F16 %d\\nc CTR_F32 %d\\n", CTR_BF16, CTR_F16, CTR_F32);', "return 0;}"]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines))
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c11", "-o", str(exe), str(src)], check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split("\n")
    got = {tuple(x.split()[:2]): int(x.split()[2]) for x in out if x.strip()}
    for cname, py in structs.items():
        assert got.pop((cname, "sizeof")) == C.sizeof(py)
        for field, _ in py._fields_:
            assert got.pop((cname, field)) == getattr(py, field).offset
    for (_, name), value in got.items():
        assert getattr(ctr, name) == value, name


BUF = C.create_string_buffer(1 << 14)
PTR = (C.addressof(BUF) + 511) // 512 * 512


def _cache(ctr, **kw):
    base = dict(k=PTR, v=PTR, dtype=0, n_kv_heads=2, head_dim=64, page_tokens=16, n_pages=4, page_stride=2048, head_stride=1024,
                token_stride=64)
    base.update(kw)
    return ctr.CtrKvCache(**base)


BAD_CACHES = [dict(k=None), dict(v=None), dict(dtype=2), dict(dtype=-1), dict(n_kv_heads=0), dict(n_kv_heads=1025), dict(head_dim=0),
              dict(head_dim=68), dict(head_dim=264), dict(page_tokens=8), dict(page_tokens=48), dict(page_tokens=2048),
              dict(n_pages=0), dict(n_pages=1 << 31), dict(page_stride=-64), dict(head_stride=-1), dict(token_stride=-8),
              dict(token_stride=1 << 62), dict(page_stride=1 << 40, n_pages=(1 << 31) - 1)]


def _append(ctr, cache=None, rope=None, rows=None, n=3, heads=4, positions=PTR, slots=PTR):
    rope = rope or ctr.CtrRope(PTR, 64, 0, 1.0, 0)
    r = dict(q=ctr.CtrRows(PTR, 256, 64), k=ctr.CtrRows(PTR, 128, 64), v=ctr.CtrRows(PTR, 128, 64), o=ctr.CtrRows(PTR, 256, 64))
    r.update(rows or {})
    return ctr.lib().ctr_kv_append(C.byref(cache or _cache(ctr)), C.byref(rope), r["q"], r["k"], r["v"], r["o"], n, heads, positions,
                                   slots, None)


def test_append_refusals(ctr):
    for kw in BAD_CACHES:
        assert _append(ctr, cache=_cache(ctr, **kw)) == ctr.CTR_EINVAL, kw
    assert ctr.lib().ctr_kv_append(None, None, *[ctr.CtrRows()] * 4, 0, 0, None, None, None) == ctr.CTR_EINVAL
    for rope in ((PTR, 63, 0, 1.0, 0), (PTR, 66, 0, 1.0, 0), (PTR, -2, 0, 1.0, 0), (PTR, 64, 2, 1.0, 0), (PTR, 64, 0, math.nan, 0),
                 (PTR, 64, 0, math.inf, 0), (PTR, 64, 0, 1.0, 1), (None, 64, 0, 1.0, 0)):
        assert _append(ctr, rope=ctr.CtrRope(*rope)) == ctr.CTR_EINVAL, rope
    for n, heads in ((-1, 4), (1 << 31, 4), (3, -1), (3, 4097)):
        assert _append(ctr, n=n, heads=heads) == ctr.CTR_EINVAL
    for name in "qkvo":
        for rows in ((None, 256, 64), (PTR + 1, 256, 64), (PTR, -1, 64), (PTR, 256, -1), (PTR, 1 << 60, 64)):
            assert _append(ctr, rows={name: ctr.CtrRows(*rows)}) == ctr.CTR_EINVAL, (name, rows)
    assert _append(ctr, positions=None) == ctr.CTR_EINVAL and _append(ctr, slots=None) == ctr.CTR_EINVAL
    assert _append(ctr, n=0) == ctr.CTR_OK


def _attention(ctr, cache=None, q=None, out=None, rows=5, heads=4, seqs=2, nodes=4, start=PTR, lens=PTR, table=PTR, stride=3,
               scale=1.0, ws=PTR, ws_bytes=1 << 40):
    r = ctr.CtrRows(PTR, 256, 64)
    return ctr.lib().ctr_tree_attention(C.byref(cache or _cache(ctr)), q or r, out or r, rows, heads, seqs, nodes, start, lens, table,
                                        stride, None, scale, None, None, ws, ws_bytes, None)


def test_attention_refusals(ctr):
    for kw in BAD_CACHES + [dict(head_dim=80), dict(head_dim=256), dict(k=PTR + 8), dict(v=PTR + 2), dict(token_stride=68),
                            dict(head_stride=1028), dict(page_stride=2052)]:
        assert _attention(ctr, cache=_cache(ctr, **kw)) == ctr.CTR_EINVAL, kw
    for kw in (dict(rows=-1), dict(rows=1 << 31), dict(heads=0), dict(heads=3), dict(heads=130), dict(seqs=-1),
               dict(seqs=ctr.CTR_MAX_SEQS + 1), dict(nodes=0), dict(nodes=65), dict(start=None), dict(lens=None), dict(table=None),
               dict(stride=0), dict(stride=1 << 30), dict(scale=math.nan), dict(scale=math.inf), dict(ws=None), dict(ws=PTR + 16),
               dict(ws_bytes=0)):
        assert _attention(ctr, **kw) == ctr.CTR_EINVAL, kw
    for rows in ((None, 256, 64), (PTR + 8, 256, 64), (PTR, 252, 64), (PTR, 256, 60), (PTR, -256, 64)):
        assert _attention(ctr, q=ctr.CtrRows(*rows)) == ctr.CTR_EINVAL, rows
        assert _attention(ctr, out=ctr.CtrRows(*rows)) == ctr.CTR_EINVAL, rows
    assert _attention(ctr, rows=0) == ctr.CTR_OK and _attention(ctr, seqs=0) == ctr.CTR_OK
    size = ctr.lib().ctr_attention_workspace_bytes
    assert size(C.byref(_cache(ctr, head_dim=80)), 4, 2, 4) == 0 and size(C.byref(_cache(ctr)), 5, 2, 4) == 0


def _sample(ctr, x=PTR, dtype=2, stride=100, n=2, vocab=100, t=PTR, u=PTR, token=PTR):
    return ctr.lib().ctr_sample(x, dtype, stride, n, vocab, t, None, None, None, u, token, None, None, None)


def test_sample_refusals(ctr):
    for kw in (dict(x=None), dict(x=PTR + 2), dict(dtype=3), dict(dtype=-1), dict(stride=99), dict(stride=1 << 62), dict(n=-1),
               dict(n=1 << 31), dict(vocab=0), dict(vocab=ctr.CTR_MAX_VOCAB + 1, stride=1 << 20), dict(t=None), dict(u=None),
               dict(token=None), dict(x=PTR + 1, dtype=0)):
        assert _sample(ctr, **kw) == ctr.CTR_EINVAL, kw
    assert _sample(ctr, n=0) == ctr.CTR_OK


def test_the_binding_refuses_what_it_can_see():
    torch = pytest.importorskip("torch")
    from paper_2609_16206_gb300 import ctr
    k = torch.zeros(2, 2, 16, 64, dtype=torch.bfloat16)
    for a, b in ((k, k), (k.float(), k.float()), (k, k.half()), (k, k[:1]), (k[0], k[0]), (k[..., ::2], k[..., ::2])):
        with pytest.raises(ValueError):
            ctr.KvCache(a, b)
    for turns in (torch.zeros(32), torch.zeros(2, 16, dtype=torch.int64), torch.zeros(32, dtype=torch.int64)):
        with pytest.raises(ValueError):
            ctr.Rope(turns)
    with pytest.raises(ValueError):
        ctr.ctr_sample(torch.zeros(3, 10), None, None, None)
