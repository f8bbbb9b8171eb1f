"""The hybrid operators' native marshalling against the Python path: the same
results, the same refusals."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture()
def swr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2512_13921_amd as lib
    lib.load()
    return lib


class _Nothing:
    """A native module that handles no call."""
    def __getattr__(self, name):
        return lambda *args: None


def _inputs(dtype):
    g = torch.Generator(device="cuda").manual_seed(3)

    def t(*shape):
        return torch.randn(shape, generator=g, device="cuda").to(dtype)

    lengths = torch.tensor([40, 0, 77], dtype=torch.int32, device="cuda")
    return {"x": t(3, 5, 96), "r": t(3, 9, 96)[:, 2:7], "w": t(96), "wf": t(96).float(), "m": t(7, 96),
            "weights": t(50, 96), "q": t(3, 4, 64), "kv": t(3, 4, 64), "caches": t(2, 12, 16, 2, 64),
            "lengths": lengths, "table": torch.arange(15, dtype=torch.int32, device="cuda").reshape(3, 5) % 12,
            "stack": torch.arange(9, dtype=torch.int32, device="cuda"),
            "count": torch.tensor([9], dtype=torch.int32, device="cuda")}


def _calls(swr, i):
    x, r, w = i["x"], i["r"], i["w"]
    yield swr.swr_rms_norm(x, w)
    yield swr.swr_rms_norm(x, i["wf"], residual=r, eps=1e-3)
    yield swr.swr_rms_norm(x, w, fp8=True)
    q, s, h = swr.swr_rms_norm(x, w, residual=r, fp8=True)
    yield q, s, h
    yield swr.swr_rms_norm(x[0, 0], w, residual=r[0, 0])
    yield swr.swr_rms_norm_backward(h, w, x, dh=r)
    yield swr.swr_rms_norm_backward(h, i["wf"], x)
    codes, powers = swr.swr_fp4_pack(i["weights"])
    yield codes, powers
    yield swr.swr_fp4_linear(i["m"], codes, powers)
    yield swr.swr_fp4_linear(q.reshape(-1, 96), codes, powers, scale=s.reshape(-1))
    yield swr.swr_fp4_linear(q, codes, powers, scale=s)
    yield swr.swr_fp4_linear(i["m"], codes, powers, scale=s.reshape(-1)[:7], out_dtype=F32)
    table = i["table"].clone()
    slots, *rest = swr.swr_block_tables(i["lengths"], i["lengths"] * 0 + 9, table, i["stack"], i["count"], 16, 27)
    yield (slots, table, *rest)
    kc, vc = i["caches"].clone()
    swr.swr_cache_append(i["kv"][:, :2], i["kv"][:, 2:], kc, vc, slots[:3])
    yield kc, vc
    yield swr.swr_paged_attention(i["q"], kc, vc, i["table"], i["lengths"])
    yield swr.swr_paged_attention(i["q"], kc, vc, i["table"], i["lengths"], scale=0.3, window=20, want_lse=True)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_native_and_python_paths_agree(swr, monkeypatch, dtype):
    inputs = _inputs(dtype)
    native = list(_calls(swr, inputs))
    monkeypatch.setattr(swr, "_native", (swr._lib, _Nothing()))
    python = list(_calls(swr, inputs))
    torch.cuda.synchronize()
    assert len(native) == len(python)
    for n, (u, w) in enumerate(zip(native, python)):
        u, w = (r if isinstance(r, tuple) else (r,) for r in (u, w))
        assert len(u) == len(w), n
        for p, q in zip(u, w):
            assert p.dtype == q.dtype and p.shape == q.shape and p.stride() == q.stride(), n
            as_bytes = (t.contiguous().view(torch.uint8) for t in (p, q))
            assert torch.equal(*as_bytes), n


@pytest.mark.parametrize("native", [True, False])
def test_refusals(swr, monkeypatch, native):
    if not native:
        monkeypatch.setattr(swr, "_native", (swr._lib, _Nothing()))
    i = _inputs(BF16)
    x, w, m = i["x"], i["w"], i["m"]
    codes, powers = swr.swr_fp4_pack(i["weights"])
    kc, vc = i["caches"]
    q, kv, n, t = i["q"], i["kv"], i["lengths"], i["table"]
    slots = torch.zeros(3, dtype=torch.int64, device="cuda")
    for error, call in (
            (TypeError, lambda: swr.swr_rms_norm(x.half(), w)),
            (ValueError, lambda: swr.swr_rms_norm(x, w[:95])),
            (ValueError, lambda: swr.swr_rms_norm(x, w.cpu())),
            (ValueError, lambda: swr.swr_rms_norm(x, w, residual=x[:2])),
            (ValueError, lambda: swr.swr_rms_norm(x, w, residual=x.float())),
            (ValueError, lambda: swr.swr_rms_norm(x.transpose(1, 2), x[0, :, 0])),
            (swr.SwrError, lambda: swr.swr_rms_norm(x, w, eps=-1.0)),
            (swr.SwrError, lambda: swr.swr_rms_norm(x.float(), w)),
            (ValueError, lambda: swr.swr_rms_norm_backward(x, w, x[:, :4])),
            (TypeError, lambda: swr.swr_fp4_linear(m.half(), codes, powers)),
            (ValueError, lambda: swr.swr_fp4_linear(m[:, :60], codes, powers)),
            (ValueError, lambda: swr.swr_fp4_linear(m, codes, powers[:, :2])),
            (ValueError, lambda: swr.swr_fp4_linear(m, codes.int(), powers)),
            (ValueError, lambda: swr.swr_fp4_linear(m, codes, powers, scale=w)),
            (swr.SwrError, lambda: swr.swr_fp4_linear(m, codes.flatten()[8:8 + 49 * 48].reshape(49, 48), powers[:49])),
            (ValueError, lambda: swr.swr_block_tables(n.long(), n, t, i["stack"], i["count"], 16, 3)),
            (ValueError, lambda: swr.swr_block_tables(n, n[:2], t, i["stack"], i["count"], 16, 3)),
            (ValueError, lambda: swr.swr_block_tables(n, n, t, i["stack"], i["count"], 16, -3)),
            (swr.SwrError, lambda: swr.swr_block_tables(n, n, t, i["stack"], i["count"], 0, 3)),
            (swr.SwrError, lambda: swr.swr_block_tables(n, n, t, t.flatten(), i["count"], 16, 3)),
            (ValueError, lambda: swr.swr_cache_append(kv, kv, kc, vc, slots)),
            (ValueError, lambda: swr.swr_cache_append(kv[:, :2], kv[:, 2:], kc, vc, slots.int())),
            (swr.SwrError, lambda: swr.swr_cache_append(kv[:, :2], kv[:, 2:], kc, kc, slots)),
            (ValueError, lambda: swr.swr_paged_attention(q[:, :3], kc, vc, t, n)),
            (ValueError, lambda: swr.swr_paged_attention(q[..., :48], kc, vc, t, n)),
            (ValueError, lambda: swr.swr_paged_attention(q, kc, vc[:5], t, n)),
            (ValueError, lambda: swr.swr_paged_attention(q, kc, vc, t[:2], n)),
            (ValueError, lambda: swr.swr_paged_attention(q, kc, vc, t, n.long())),
            (swr.SwrError, lambda: swr.swr_paged_attention(q, kc, vc, t, n, window=-1))):
        with pytest.raises(error):
            call()
    torch.cuda.synchronize()


def test_the_current_and_a_given_stream(swr):
    """Both paths launch on torch's current stream, or on the one that is given."""
    i = _inputs(BF16)
    x = torch.zeros_like(i["x"])
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for given in (False, True):
        with torch.cuda.stream(s):
            for _ in range(50):   # work that the call has to come after
                big = torch.randn(1 << 20, device="cuda")
            x.copy_(i["x"])
            if not given:
                y = swr.swr_rms_norm(x, i["w"])
        if given:
            y = swr.swr_rms_norm(x, i["w"], stream=s)
        s.synchronize()
        assert torch.equal(y, swr.swr_rms_norm(i["x"], i["w"]))
        x.zero_()
        torch.cuda.synchronize()
        del big
