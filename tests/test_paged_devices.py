"""Where a call's tensors lie: a workspace on the host, or a tensor on another device than the one that the
call launches on, is refused before the library is called. Stand-ins for tensors, without a GPU."""
import pytest

torch = pytest.importorskip("torch")
cg = pytest.importorskip("paper_2607_20538_gb300")
paged = cg.paged


class OnDevice:
    """A tensor as if on a GPU: what the binding asks of one, and no memory."""

    def __init__(self, shape, dtype, index=0):
        self._t, self._index = torch.empty(shape, dtype=dtype, device="meta"), index
        self.is_cuda, self.device = index >= 0, torch.device("cuda", index) if index >= 0 else torch.device("cpu")

    def get_device(self):
        return self._index

    def data_ptr(self):
        return 1 << 20

    def __getattr__(self, name):
        return getattr(self._t, name)


@pytest.fixture(autouse=True)
def calls(monkeypatch):
    """The library's calls are recorded instead; the current device is 0."""
    made = []
    monkeypatch.setattr(paged, "_fn", lambda name: lambda *a: made.append(name) or 0)
    monkeypatch.setattr(paged, "_device", lambda: 0)
    monkeypatch.setattr(paged, "_stream", lambda stream: 0)
    return made


I32, I64, BF16, U8 = torch.int32, torch.int64, torch.bfloat16, torch.uint8


def _tensors(call):
    """Shapes and types of each call's tensors."""
    if call == "plan":
        return dict(ctx_lens=([2], I32), new_lens=([2], I32), free_pages=([8], I32), free_count=([1], I32), block_table=([2, 4], I32),
                    seq_lens=([2], I32), cu_new=([3], I32), positions=([5], I32), slots=([5], I64), free_left=([1], I32))
    if call == "release":
        return dict(lens=([2], I32), done=([2], I32), block_table=([2, 4], I32), free_pages=([8], I32), free_count=([1], I32),
                    lens_left=([2], I32), free_left=([1], I32))
    if call == "rotary":
        return dict(x=([5, 8, 128], BF16), positions=([5], I32), table=([64], I64), out=([5, 8, 128], BF16))
    if call == "append":
        return dict(q=([5, 8, 128], BF16), k=([5, 2, 128], BF16), v=([5, 2, 128], BF16), positions=([5], I32), slots=([5], I64),
                    table=([64], I64), q_out=([5, 8, 128], BF16), pool=([2, 8, 2, 16, 128], BF16))
    return dict(q=([5, 8, 128], BF16), pool=([2, 8, 2, 16, 128], BF16), block_table=([2, 4], I32), seq_lens=([2], I32), cu_new=([3], I32),
                out=([5, 8, 128], BF16), lse=([5, 8], torch.float32), workspace=([1 << 20], U8))


def _make(call, t, **kw):
    pages = cg.Pages(n_pages=8, page=16, H=2, d=128, n_req=2, max_pages=4)
    {"plan": lambda: cg.page_plan(pages, **t, **kw), "release": lambda: cg.page_release(pages, **t, **kw),
     "rotary": lambda: cg.rotary(cg.Rotary(128), **t, **kw), "append": lambda: cg.rotary_append(pages, cg.Rotary(128), **t, **kw),
     "attention": lambda: cg.paged_attention(pages, cg.PagedAttention(4, 4, 0.1), **t, **kw)}[call]()


def test_a_workspace_on_the_host_is_refused(calls):
    t = {k: OnDevice(*v) for k, v in _tensors("attention").items()}
    _make("attention", t)
    assert len(calls) == 1
    for bad in (torch.empty(1 << 20, dtype=U8), OnDevice([1 << 10, 1 << 10], U8, 0).t()):
        with pytest.raises(cg.CodecGaugeError) as e:
            _make("attention", dict(t, workspace=bad))
        assert e.value.code == -1 and "workspace" in str(e.value)
    assert len(calls) == 1


@pytest.mark.parametrize("call", ["plan", "release", "rotary", "append", "attention"])
def test_every_tensor_is_on_the_calls_device(call, calls):
    shapes = _tensors(call)
    make = lambda **index: {k: OnDevice(*v, index.get(k, 0)) for k, v in shapes.items()}  # noqa: E731
    _make(call, make())
    assert len(calls) == 1
    for name in shapes:
        for index in (1, -1):
            with pytest.raises(cg.CodecGaugeError) as e:
                _make(call, make(**{name: index}))
            assert e.value.code == -1 and str(e.value).startswith(f"CG_EINVAL: {name}:"), name
    assert len(calls) == 1


@pytest.mark.parametrize("call", ["plan", "release", "rotary", "append", "attention"])
def test_a_stream_of_another_device_is_refused(call, calls, monkeypatch):
    monkeypatch.undo()
    monkeypatch.setattr(paged, "_fn", lambda name: lambda *a: calls.append(name) or 0)
    monkeypatch.setattr(paged, "_device", lambda: 0)

    class Stream:
        cuda_stream = 5

        def __init__(self, index):
            self.device_index = index

    t = {k: OnDevice(*v) for k, v in _tensors(call).items()}
    _make(call, t, stream=Stream(0))
    with pytest.raises(cg.CodecGaugeError) as e:
        _make(call, t, stream=Stream(1))
    assert e.value.code == -1 and "stream" in str(e.value) and len(calls) == 1


@pytest.mark.skipif(torch.cuda.is_available(), reason="a machine without a GPU is meant")
def test_without_a_gpu_the_refusal_is_the_same(calls, monkeypatch):
    monkeypatch.undo()
    t = {k: torch.empty(shape, dtype=dt) for k, (shape, dt) in _tensors("attention").items()}
    with pytest.raises(cg.CodecGaugeError) as e:
        _make("attention", t)
    assert e.value.code == -1
