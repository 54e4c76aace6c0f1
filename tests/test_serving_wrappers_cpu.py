"""The Python entry points for sequences of different lengths hand the library no address that is not memory of the
current device: checked here with stand-ins for CUDA tensors and for the library, so that no GPU is needed."""
import pytest

torch = pytest.importorskip("torch")
from paper_2609_37924_gb300 import tadm  # noqa: E402


class Cuda:
    """A CPU tensor that says it is on CUDA device `index`."""

    def __init__(self, t, index=0):
        self.t, self.index = t, index

    def __getattr__(self, name):
        return getattr(self.t, name)

    is_cuda = True

    @property
    def device(self):
        return torch.device("cuda", self.index)

    def get_device(self):
        return self.index


class Library:
    """Takes every call and keeps its name."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *a: self.calls.append(name) or 0


@pytest.fixture
def lib(monkeypatch):
    so = Library()
    monkeypatch.setattr(tadm, "load_library", lambda *a: so)
    monkeypatch.setattr(tadm, "_stream", lambda stream=None: None)
    monkeypatch.setattr(tadm, "_device", lambda: 0, raising=False)
    return so


def ints(*shape, device=0):
    return Cuda(torch.zeros(shape, dtype=torch.int32), device)


def rows(n, heads=2, device=0):
    return Cuda(torch.zeros((n, heads, 64), dtype=torch.bfloat16), device)


def pool(device=0):
    z = lambda shape, dt: Cuda(torch.zeros(shape, dtype=dt), device)  # noqa: E731
    return tadm.PagePool(z((1, 4, 2, 64, 64), torch.uint8), z((1, 4, 2, 64, 64), torch.uint8), z((1, 4, 2), torch.float32),
                         z((1, 4, 2), torch.float32))


def scratch(device=0):
    return Cuda(torch.zeros(4096, dtype=torch.uint8), device)


def calls():
    return {
        "tadm_attention_packed": dict(q=rows(5), k=rows(5), v=rows(5), o=rows(5), cu_rows=ints(2), max_rows=5),
        "tadm_page_write": dict(pool=pool(), layer=0, k=rows(5), v=rows(5), cu_rows=ints(2), start=ints(1), table=ints(1, 2), max_rows=5),
        "tadm_page_read": dict(pool=pool(), layer=0, k=rows(5), v=rows(5), cu_rows=ints(2), start=ints(1), table=ints(1, 2), max_rows=5),
        "tadm_page_attention": dict(q=rows(5), pool=pool(), layer=0, o=rows(5), cu_rows=ints(2), lens=ints(1), table=ints(1, 2),
                                    max_rows=5, max_len=100, scratch=scratch()),
        "tadm_pages_reserve": dict(tables=ints(2, 2), refs=ints(4), seqs=ints(1), new_len=ints(1), tables_out=ints(2, 2),
                                   refs_out=ints(4), status=ints(1), scratch=scratch()),
        "tadm_pages_fork": dict(pool=pool(), tables=ints(2, 2), lens=ints(2), refs=ints(4), src=ints(1), dst=ints(1),
                                tables_out=ints(2, 2), lens_out=ints(2), refs_out=ints(4), status=ints(1), scratch=scratch()),
        "tadm_pages_free": dict(tables=ints(2, 2), lens=ints(2), refs=ints(4), seqs=ints(1), tables_out=ints(2, 2), lens_out=ints(2),
                                refs_out=ints(4), status=ints(1), scratch=scratch()),
        "tadm_pages_compact": dict(pool=pool(), tables=ints(2, 2), refs=ints(4), tables_out=ints(2, 2), refs_out=ints(4),
                                   n_live=ints(1), scratch=scratch()),
        "tadm_pages_copy": dict(pool=pool(), src=ints(1), dst=ints(1)),
    }


@pytest.mark.parametrize("name", list(calls()))
def test_well_formed_calls_reach_the_library(lib, name):
    getattr(tadm, name)(**calls()[name])
    assert lib.calls == [name]


def on_device_1(name, value):
    if name == "pool":
        return pool(1)
    return Cuda(value.t, 1)


OPERANDS = [(name, arg) for name, args in calls().items() for arg, v in args.items() if not isinstance(v, int)]


@pytest.mark.parametrize("name,arg", OPERANDS)
def test_operands_of_another_device_are_refused(lib, name, arg):
    args = calls()[name]
    args[arg] = on_device_1(arg, args[arg])
    with pytest.raises(tadm.TadmError):
        getattr(tadm, name)(**args)
    assert lib.calls == []


@pytest.mark.parametrize("name", [n for n, a in calls().items() if "scratch" in a])
@pytest.mark.parametrize("bad", [torch.zeros(4096, dtype=torch.uint8), Cuda(torch.zeros(8192, dtype=torch.uint8)[::2])])
def test_scratch_is_contiguous_memory_of_the_device(lib, name, bad):
    with pytest.raises(tadm.TadmError):
        getattr(tadm, name)(**{**calls()[name], "scratch": bad})
    assert lib.calls == []


@pytest.mark.parametrize("name", [n for n, a in calls().items() if "status" in a or "n_live" in a])
def test_the_outcome_has_a_place(lib, name):
    args = calls()[name]
    args["n_live" if "n_live" in args else "status"] = ints(0)
    with pytest.raises(tadm.TadmError):
        getattr(tadm, name)(**args)
    assert lib.calls == []


def test_fp32_attention_needs_no_scratch(lib):
    f = lambda: Cuda(torch.zeros((5, 2, 64)))  # noqa: E731
    tadm.tadm_page_attention(**{**calls()["tadm_page_attention"], "q": f(), "o": f(), "scratch": None})
    assert lib.calls == ["tadm_page_attention"]


def test_strides_of_single_rows_and_heads_do_not_matter(lib):
    """A tensor of one row has no distance between rows, one of one head none between heads, whatever their strides say."""
    leading = []
    lib.tadm_attention_packed = lambda *a: leading.append(a[11:15]) or 0
    one_row = lambda h: Cuda(torch.zeros((h, 1, 64), dtype=torch.bfloat16).transpose(0, 1))  # noqa: E731
    tadm.tadm_attention_packed(one_row(8), one_row(2), one_row(2), one_row(8), ints(2), 1)
    assert leading.pop() == (512, 128, 128, 512)
    one_head = lambda: Cuda(torch.zeros((1, 5, 64), dtype=torch.bfloat16).transpose(0, 1))  # noqa: E731
    tadm.tadm_attention_packed(one_head(), one_head(), one_head(), one_head(), ints(2), 5)
    assert leading.pop() == (64, 64, 64, 64)
    with pytest.raises(tadm.TadmError):
        tadm.tadm_attention_packed(*[Cuda(torch.zeros((2, 5, 64), dtype=torch.bfloat16).transpose(0, 1)) for _ in range(4)], ints(2), 5)


def test_stream_and_device_without_torchs_private_functions(monkeypatch):
    """The quick lookups of the current stream and device are not part of torch's interface: where a version lacks them, its
    public ones serve."""
    for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"):
        monkeypatch.delattr(torch._C, name, raising=False)
    monkeypatch.setattr(torch.cuda, "init", lambda: None)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: type("S", (), {"cuda_stream": 77})())
    monkeypatch.setattr(tadm, "_raw_stream", None)
    monkeypatch.setattr(tadm, "_current_device", None)
    assert tadm._stream() == 77 and tadm._device() == 3
    assert tadm._stream(type("S", (), {"cuda_stream": 5})()) == 5
