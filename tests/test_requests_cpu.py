"""What the operators for requests with settings of their own refuse, all on the host before anything is enqueued, and what
their Python entry points hand to the library: no GPU is needed."""
import ctypes

import pytest

from test_serving_wrappers_cpu import Cuda, Library, ints, scratch

INVALID, UNSUPPORTED = 1, 2
P = 1 << 20          # stands for an aligned device pointer; no refused call follows it


@pytest.fixture(scope="module")
def T():
    import __graft_entry__ as g
    g.build()
    from paper_2609_37924_gb300 import tadm
    return tadm


SAMPLE = dict(logits=P, ld=1000, rows=4, vocab=1000, mask_id=-1, temperature=P, top_k=P, top_p=P, min_p=P, u=P, tok=P, prob=P,
              dtype=0, scratch=None, scratch_bytes=0, stream=None)


@pytest.mark.parametrize("over", [
    dict(logits=None), dict(u=None), dict(tok=None), dict(rows=-1), dict(vocab=0), dict(vocab=1001), dict(ld=999),
    dict(mask_id=-2), dict(mask_id=1000), dict(dtype=2), dict(dtype=-1), dict(logits=P + 2), dict(logits=P + 1, dtype=1),
    dict(u=P + 2), dict(tok=P + 1), dict(prob=P + 2), dict(top_k=P + 2), dict(top_p=P + 1), dict(min_p=P + 3),
    dict(temperature=P + 2)])
def test_sample_refuses(T, over):
    assert T.load_library().tadm_sample(*{**SAMPLE, **over}.values()) == INVALID


def test_sample_sizes(T):
    f = T.load_library().tadm_sample
    assert f(*{**SAMPLE, "rows": 0, "logits": None, "u": None, "tok": None}.values()) == 0
    big = (1 << 19) + 1
    assert f(*{**SAMPLE, "vocab": big, "ld": big}.values()) == UNSUPPORTED
    assert f(*{**SAMPLE, "rows": (1 << 24) + 1}.values()) == UNSUPPORTED


def test_sample_scratch(T):
    size = T.tadm_sample_scratch_size
    assert size(4, 4096) == 0 and size(0, 100000) == 0
    need = size(4, 100000)
    assert 0 < need <= size(5, 100000) and need <= size(4, 200000)
    call = {**SAMPLE, "vocab": 100000, "ld": 100000, "scratch": P, "scratch_bytes": need}
    for over in (dict(scratch=None), dict(scratch=P + 128), dict(scratch_bytes=need - 1)):
        assert T.load_library().tadm_sample(*{**call, **over}.values()) == INVALID
    n = ctypes.c_size_t()
    for bad in ((-1, 100), (4, 0)):
        assert T.load_library().tadm_sample_scratch_size(*bad, ctypes.byref(n)) == INVALID
    assert T.load_library().tadm_sample_scratch_size(4, 100, None) == INVALID


LORA = dict(x=P, w=P, y=P, cu=P, adapter=P, batch=3, total=10, n_in=64, n_out=40, ldx=64, ldw=64, ldy=40, a=P, b=P, scale=P,
            n=2, rank=16, dtype=1, y_dtype=1, scratch=P, scratch_bytes=1 << 40, stream=None)


@pytest.mark.parametrize("over", [
    dict(x=None), dict(w=None), dict(y=None), dict(cu=None), dict(adapter=None), dict(a=None), dict(b=None), dict(scale=None),
    dict(batch=-1), dict(total=-1), dict(n_in=0), dict(n_out=0), dict(n_in=60, ldx=64, ldw=64), dict(ldx=56), dict(ldx=68),
    dict(ldw=60), dict(ldw=68), dict(ldy=39), dict(n=-1), dict(rank=0), dict(rank=4), dict(rank=12), dict(rank=264),
    dict(dtype=2), dict(y_dtype=2), dict(dtype=0, y_dtype=1), dict(x=P + 8), dict(w=P + 8), dict(y=P + 1), dict(a=P + 8),
    dict(b=P + 4), dict(scale=P + 2), dict(cu=P + 2), dict(adapter=P + 1), dict(scratch=None), dict(scratch=P + 8),
    dict(scratch_bytes=0)])
def test_lora_refuses(T, over):
    assert T.load_library().tadm_lora_project(*{**LORA, **over}.values()) == INVALID


def test_lora_scratch(T):
    f, n = T.load_library().tadm_lora_scratch_size, ctypes.c_size_t()
    for bad in ((-1, 10, 64, 40, 2, 16, 1), (3, -1, 64, 40, 2, 16, 1), (3, 10, 0, 40, 2, 16, 1), (3, 10, 64, 0, 2, 16, 1),
                (3, 10, 64, 40, -1, 16, 1), (3, 10, 64, 40, 2, 20, 1), (3, 10, 64, 40, 2, 16, 2)):
        assert f(*bad, ctypes.byref(n)) == INVALID
    assert f(3, 10, 64, 40, 2, 16, 1, None) == INVALID
    for dtype in (0, 1):
        need = T.tadm_lora_scratch_size(3, 10, 64, 40, 2, 16, dtype)
        call = {**LORA, "dtype": dtype, "y_dtype": 0}
        assert T.load_library().tadm_lora_project(*{**call, "scratch_bytes": need - 1}.values()) == INVALID
    for over in (dict(total=(1 << 20) + 1), dict(batch=(1 << 30) + 1), dict(n_out=(1 << 20) + 1, ldy=1 << 21)):
        assert T.load_library().tadm_lora_project(*{**LORA, **over}.values()) == UNSUPPORTED
    for over in (dict(batch=0), dict(total=0)):
        assert T.load_library().tadm_lora_project(*{**LORA, **over}.values()) == 0


def test_lora_more_factors_than_are_counted(T):
    """Every row an adapter of its own, at the highest rank: refused, none of them is left out."""
    call = {**LORA, "batch": 1 << 20, "total": 1 << 20, "rank": 256, "scratch_bytes": 1 << 60}
    assert T.tadm_lora_scratch_size(1 << 20, 1 << 20, 64, 40, 300, 256, 1) > 1 << 38
    assert T.load_library().tadm_lora_project(*{**call, "n": 300}.values()) == UNSUPPORTED
    assert T.tadm_lora_scratch_size(1 << 20, 1 << 20, 64, 40, 2, 256, 1) <= 1 << 38


NORM = dict(x=P, y=P, x_out=P, n_out=P, cu=P, batch=3, total=10, d=64, ldx=64, ldy=64, ldxo=64, ldn=64, post=P, gate=P, ldg=64,
            pre=P, residual_scale=1.0, eps=1e-6, x_dtype=0, y_dtype=0, dtype=1, stream=None)


@pytest.mark.parametrize("over", [
    dict(x=None), dict(y=None), dict(x_out=None), dict(cu=None), dict(cu=None, batch=0), dict(batch=-1), dict(total=-1),
    dict(d=0), dict(ldx=63), dict(ldy=63), dict(ldxo=63), dict(ldn=63), dict(ldg=63), dict(eps=-1e-6), dict(eps=float("nan")),
    dict(eps=float("inf")), dict(residual_scale=float("nan")), dict(x_dtype=2), dict(y_dtype=-1), dict(dtype=2), dict(x=P + 2),
    dict(y=P + 1), dict(x_out=P + 2), dict(n_out=P + 1), dict(post=P + 1), dict(gate=P + 1), dict(pre=P + 1), dict(cu=P + 2)])
def test_residual_norm_refuses(T, over):
    assert T.load_library().tadm_residual_norm(*{**NORM, **over}.values()) == INVALID


def test_residual_norm_sizes(T):
    f = T.load_library().tadm_residual_norm
    for over in (dict(batch=0), dict(total=0), dict(cu=None, batch=1, total=0)):
        assert f(*{**NORM, **over}.values()) == 0
    wide = dict(d=49153, ldx=49153, ldy=49153, ldxo=49153, ldn=49153, ldg=49153)
    assert f(*{**NORM, **wide}.values()) == UNSUPPORTED
    for over in (dict(total=(1 << 30) + 1), dict(total=2 ** 31 - 1, d=8), dict(batch=(1 << 30) + 1)):
        assert f(*{**NORM, **over}.values()) == UNSUPPORTED


def test_every_bounded_wait_of_the_adapters_names_the_status_word():
    import os
    import re
    src = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_37924_gb300", "csrc", "adapters.cu")).read()
    waits = re.findall(r"(?:mbar|warp)_wait_bounded\((.*)\)", src)
    assert len(waits) > 8
    for w in waits:
        assert "a.status" in w and "nullptr" not in w, w


def test_local_arrays_read_as_vectors_are_aligned_for_them():
    """`T v[N]` read back through a pointer to 16 bytes: the array says so, whatever the compiler keeps it in."""
    import os
    import re
    at = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_37924_gb300", "csrc")
    found = 0
    for name in ("sample_rows.cu", "adapters.cu", "adapters_rows.cu", "residual_norm.cu"):
        src = open(os.path.join(at, name)).read()
        for m in re.finditer(r"reinterpret_cast<(?:const )?(?:uint4|float4|uint2)\*>\(([a-z]+)\)(?!\[)", src):
            decl = [d for d in re.finditer(r"^ *(?:alignas\([^;]*\) )?[\w:]+ " + m.group(1) + r"\[[^\]]+\];", src[:m.start()], re.M)]
            if decl:
                found += 1
                assert "alignas" in decl[-1].group(0), (name, decl[-1].group(0))
    assert found >= 2


# ------------------------------------------------------------------ the Python entry points
torch = pytest.importorskip("torch")
from paper_2609_37924_gb300 import tadm  # noqa: E402


@pytest.fixture
def lib(monkeypatch):
    so = Library()
    monkeypatch.setattr(tadm, "load_library", lambda *a: so)
    monkeypatch.setattr(tadm, "_stream", lambda stream=None: None)
    monkeypatch.setattr(tadm, "_device", lambda: 0)
    return so


def f32(*shape, device=0):
    return Cuda(torch.zeros(shape), device)


def b16(*shape, device=0):
    return Cuda(torch.zeros(shape, dtype=torch.bfloat16), device)


def sample_args(**over):
    return {**dict(logits=f32(4, 100), u=f32(4), tok=ints(4), temperature=f32(4), top_k=ints(4), top_p=f32(4), min_p=f32(4),
                   prob=f32(4), scratch=scratch()), **over}


def lora_args(**over):
    return {**dict(x=b16(10, 64), w=b16(40, 64), y=b16(10, 40), cu_rows=ints(4), adapter=ints(3), lora_a=b16(2, 16, 64),
                   lora_b=b16(2, 40, 16), lora_scale=f32(2), scratch=scratch()), **over}


def norm_args(**over):
    return {**dict(x=f32(10, 64), y=b16(10, 64), x_out=f32(10, 64), n_out=b16(10, 64), cu_rows=ints(4), post_gain=b16(64),
                   gate=b16(3, 64), pre_gain=b16(64)), **over}


@pytest.mark.parametrize("name,args", [("tadm_sample", sample_args), ("tadm_lora_project", lora_args),
                                       ("tadm_residual_norm", norm_args)])
def test_every_operand_is_on_the_current_device(lib, name, args):
    good = args()
    getattr(tadm, name)(**good)
    assert lib.calls == [name]
    for key, t in good.items():
        with pytest.raises(tadm.TadmError):
            getattr(tadm, name)(**{**good, key: Cuda(t.t, 1)})
    assert lib.calls == [name]


@pytest.mark.parametrize("over", [
    dict(u=f32(3)), dict(tok=ints(5)), dict(tok=f32(4)), dict(top_k=f32(4)), dict(top_p=ints(4)), dict(temperature=f32(4, 1)),
    dict(prob=b16(4)), dict(logits=f32(4, 100, 1)), dict(logits=ints(4, 100)), dict(logits=Cuda(torch.zeros(100, 4).T)),
    dict(u=Cuda(torch.zeros(8)[::2]))])
def test_sample_shapes(lib, over):
    with pytest.raises(tadm.TadmError):
        tadm.tadm_sample(**sample_args(**over))
    assert not lib.calls


@pytest.mark.parametrize("over", [
    dict(x=b16(10, 72)), dict(w=b16(40, 72)), dict(w=f32(40, 64)), dict(y=b16(9, 40)), dict(y=b16(10, 41)),
    dict(lora_a=b16(2, 16, 72)), dict(lora_b=b16(3, 40, 16)), dict(lora_b=b16(2, 41, 16)), dict(lora_b=b16(2, 40, 8)),
    dict(lora_a=f32(2, 16, 64)), dict(lora_scale=f32(3)), dict(adapter=ints(4)), dict(x=Cuda(torch.zeros(64, 10).bfloat16().T)),
    dict(lora_b=Cuda(torch.zeros(2, 16, 40).bfloat16().transpose(1, 2)))])
def test_lora_shapes(lib, over):
    with pytest.raises(tadm.TadmError):
        tadm.tadm_lora_project(**lora_args(**over))
    assert not lib.calls


@pytest.mark.parametrize("over", [
    dict(y=b16(10, 72)), dict(x_out=b16(10, 64)), dict(x_out=f32(9, 64)), dict(n_out=b16(10, 63)), dict(gate=b16(2, 64)),
    dict(gate=f32(3, 64)), dict(post_gain=f32(64)), dict(pre_gain=b16(63)), dict(pre_gain=b16(1, 64)),
    dict(x=Cuda(torch.zeros(64, 10).T)), dict(n_out=None, gate=None, post_gain=ints(64), pre_gain=ints(64))])
def test_residual_norm_shapes(lib, over):
    with pytest.raises(tadm.TadmError):
        tadm.tadm_residual_norm(**norm_args(**over))
    assert not lib.calls


def test_optional_operands(lib):
    tadm.tadm_sample(f32(4, 100), f32(4), ints(4))
    tadm.tadm_residual_norm(f32(10, 64), f32(10, 64), f32(10, 64))
    tadm.tadm_residual_norm(f32(10, 64), f32(10, 64), f32(10, 64), gate=f32(1, 64))
    assert [c for c in lib.calls if "scratch" not in c] == ["tadm_sample", "tadm_residual_norm", "tadm_residual_norm"]
