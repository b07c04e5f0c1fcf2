"""What the binding of the decode operators refuses before a call: tensors on the host, of another type, shape or stride."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ctr():
    from paper_2609_16206_gb300 import build
    build.build()
    from paper_2609_16206_gb300 import ctr
    return ctr


def test_host_tensors_and_other_objects_are_refused(ctr):
    m = ctr.marshal()
    cache = ctr.CtrKvCache(4096, 4096, ctr.CTR_BF16, 2, 64, 16, 4, 2048, 1024, 64)
    rope = ctr.CtrRope(4096, 64, 0, 1.0, 0)
    at, turns = C.addressof(cache), C.addressof(rope)
    x = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    i64, i32, f32 = (torch.zeros(3, dtype=t) for t in (torch.int64, torch.int32, torch.float32))
    table, logits = torch.zeros(3, 5, dtype=torch.int32), torch.zeros(3, 10)
    for bad in (x, None, 7, [x]):
        with pytest.raises(ValueError):
            m.kv_append(at, turns, bad, x, x, i64, i64, x, 0)
        with pytest.raises(ValueError):
            m.tree_attention(at, bad, i32, i32, table, x, i64, 4, None, None, 1.0, None, 0)
        with pytest.raises(ValueError):
            m.sample(bad, f32, f32, i32, None, None, None, None, None, 0)
    with pytest.raises(ValueError):
        m.sample(logits, f32, f32, i32, None, None, None, None, None, 0)
    for call, n in ((m.kv_append, 9), (m.tree_attention, 13), (m.sample, 10), (m.bind, 3)):
        with pytest.raises(TypeError):
            call(*[None] * (n - 1))


def test_a_missing_module_fails_loudly(ctr, monkeypatch, tmp_path):
    monkeypatch.setattr(ctr, "_marshal", None)
    monkeypatch.setattr(ctr, "MARSHAL_PATH", str(tmp_path / "_marshal.so"))
    with pytest.raises(ctr.CtrError) as e:
        ctr.ctr_sample(torch.zeros(3, 10), None, None, None)
    assert "_marshal.so" in str(e.value)


def _append_args(ctr, dev):
    k = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16, device=dev)
    row = lambda heads: torch.zeros(3, heads, 64, dtype=torch.bfloat16, device=dev)  # noqa: E731
    vec = lambda: torch.zeros(3, dtype=torch.int64, device=dev)  # noqa: E731
    rope = ctr.Rope(torch.zeros(32, dtype=torch.int64, device=dev))
    return dict(cache=ctr.KvCache(k, torch.zeros_like(k)), rope=rope, q=row(4), k=row(2), v=row(2), positions=vec(), slots=vec(), q_out=row(4))


@pytest.mark.gpu
@pytest.mark.parametrize("change", ["host", "dtype", "dim", "heads", "tokens", "stride"])
@pytest.mark.parametrize("name", ["q", "k", "v", "q_out"])
def test_append_rows_that_do_not_fit(ctr, name, change):
    a = _append_args(ctr, "cuda")
    t = a[name]
    a[name] = {"host": lambda: t.cpu(), "dtype": lambda: t.half(), "dim": lambda: t[..., :32], "heads": lambda: t[:, :1], "tokens": lambda: t[:2],
               "stride": lambda: torch.zeros(3, t.shape[1], 128, dtype=t.dtype, device="cuda")[..., ::2]}[change]()
    with pytest.raises(ValueError):
        ctr.ctr_kv_append(**a)


@pytest.mark.gpu
def test_vectors_that_do_not_fit(ctr):
    for name in ("positions", "slots"):
        good = _append_args(ctr, "cuda")[name]
        for bad in (good.cpu(), good.int(), good[:2], torch.zeros(6, dtype=torch.int64, device="cuda")[::2]):
            with pytest.raises(ValueError):
                ctr.ctr_kv_append(**{**_append_args(ctr, "cuda"), name: bad})
        with pytest.raises(ctr.CtrError):  # the entry point itself: it may not be missing
            ctr.ctr_kv_append(**{**_append_args(ctr, "cuda"), name: None})


def _attention_args(ctr):
    cache = _append_args(ctr, "cuda")["cache"]
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16, device="cuda")
    return dict(cache=cache, q=q, q_start=i32([0, 1, 3]), kv_len=i32([1, 5]), page_table=i32([[0], [1]]), out=torch.zeros_like(q),
                workspace=ctr.attention_workspace(cache, 4, 2, 2), max_nodes=2, tree_mask=torch.ones(3, dtype=torch.int64, device="cuda"),
                lse=torch.zeros(3, 4, device="cuda"))


@pytest.mark.gpu
def test_attention_arguments_that_do_not_fit(ctr):
    a = _attention_args(ctr)
    ctr.ctr_tree_attention(**a)
    bad = [("q", a["q"][:2]), ("q", a["q"].cpu()), ("out", a["out"].half()), ("out", a["out"][:, :2]), ("q_start", a["q_start"][:2]),
           ("q_start", a["q_start"].long()), ("kv_len", a["kv_len"].cpu()), ("kv_len", a["kv_len"][:1]), ("page_table", a["page_table"][:1]),
           ("page_table", a["page_table"].long()), ("page_table", a["page_table"].flatten()), ("tree_mask", a["tree_mask"].int()),
           ("tree_mask", a["tree_mask"][:2]), ("lse", a["lse"].half()), ("lse", a["lse"][:2]), ("workspace", a["workspace"].cpu()),
           ("status", torch.zeros(2, dtype=torch.int32, device="cuda")), ("workspace", None), ("kv_len", None)]
    for name, value in bad:
        with pytest.raises(ValueError):
            ctr.ctr_tree_attention(**{**a, name: value})
    for name, value in (("max_nodes", 0), ("max_nodes", 65), ("workspace", a["workspace"][:256]), ("scale", float("nan")), ("q_start", None)):
        with pytest.raises(ctr.CtrError):
            ctr.ctr_tree_attention(**{**a, name: value})


@pytest.mark.gpu
def test_sample_arguments_that_do_not_fit(ctr):
    f32 = lambda n=3: torch.ones(n, device="cuda")  # noqa: E731
    i32 = lambda n=3: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
    a = dict(logits=torch.zeros(3, 40, device="cuda"), temperature=f32(), u=torch.zeros(3, device="cuda"), token=i32(), top_k=i32(), top_p=f32(),
             min_p=torch.zeros(3, device="cuda"), logprob=f32(), n_kept=i32())
    ctr.ctr_sample(**a)
    for name, value in (("logits", a["logits"].cpu()), ("logits", a["logits"].double()), ("logits", a["logits"][:, ::2]), ("logits", a["logits"][0]),
                        ("temperature", f32(2)), ("temperature", f32().half()), ("u", f32(4)), ("token", i32().long()), ("top_k", i32(2)),
                        ("top_p", f32().cpu()), ("min_p", f32(6)[::2]), ("logprob", f32(2)), ("n_kept", f32())):
        with pytest.raises(ValueError):
            ctr.ctr_sample(**{**a, name: value})
    for name in ("temperature", "u", "token"):
        with pytest.raises(ctr.CtrError):
            ctr.ctr_sample(**{**a, name: None})


@pytest.mark.gpu
def test_the_calls_follow_the_library_in_use(ctr):
    from paper_2609_16206_gb300 import build
    build.build(checked=True)
    before = ctr.use_library(ctr.LIB_CHECKED_PATH)
    try:
        first = ctr.marshal()
        a = _append_args(ctr, "cuda")
        a["v"].fill_(3.0)
        a["slots"].copy_(torch.tensor([5, -1, 17], device="cuda"))
        ctr.ctr_kv_append(**a)
        got = a["cache"].v
        assert float(got[0, :, 5].min()) == 3.0 and float(got[1, :, 1].min()) == 3.0 and int((got != 0).sum()) == 2 * 2 * 64
    finally:
        ctr.use_library(before)
    assert first is not None and ctr.marshal() is not None
