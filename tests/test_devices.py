"""Which GPU a call of the sequence operators runs on, with tensors that only claim to lie on one (no GPU)."""
import contextlib

import pytest
import torch

import paper_2407_13726_b200 as dastac
from paper_2407_13726_b200 import binding


class _Claimed:
    """Stands for a contiguous tensor on GPU ``dev``."""

    def __init__(self, dev, shape, dtype):
        self._t, self._dev = torch.empty(shape, dtype=dtype), dev
        self.shape, self.dtype, self.device = self._t.shape, dtype, torch.device("cuda", dev)
        self.is_cuda = True

    def get_device(self):
        return self._dev

    def __getattr__(self, name):
        return getattr(self._t, name)


class _Library:
    """Records which GPU is current, and the stream, in each call."""

    def __init__(self, state):
        self.calls = []
        for name in ("linrec_forward", "linrec_backward", "linear_forward", "linear_backward"):
            setattr(self, "dastac_" + name, lambda *a, name=name: self.calls.append((name, state[0], a[-1])) or 0)

        def workspace(shape, nbytes):
            nbytes._obj.value = 1000 + state[0]
            self.calls.append(("linrec_workspace", state[0], None))
            return 0

        self.dastac_linrec_workspace = workspace


@pytest.fixture
def library(monkeypatch):
    state = [0]

    @contextlib.contextmanager
    def device(dev):
        before, state[0] = state[0], dev
        yield
        state[0] = before

    lib = _Library(state)
    monkeypatch.setattr(binding, "_packed", lib)
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: state[0])
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 70 + dev)
    binding._linrec_bytes.cache_clear()
    yield lib
    assert state[0] == 0
    binding._linrec_bytes.cache_clear()


def _recurrence(dev):
    s = lambda: _Claimed(dev, (2, 5, 8), torch.float32)  # noqa: E731
    return dict(g=s(), x=s(), out=s(), h0=_Claimed(dev, (2, 8), torch.float32), h_last=_Claimed(dev, (2, 8), torch.float32),
                carries=_Claimed(dev, (2, 1, 8), torch.float32), workspace=_Claimed(dev, (64,), torch.uint8),
                err_word=_Claimed(dev, (1,), torch.int32))


def _recurrence_back(dev):
    s = lambda: _Claimed(dev, (2, 5, 8), torch.float32)  # noqa: E731
    v = lambda: _Claimed(dev, (2, 8), torch.float32)  # noqa: E731
    return dict(g=s(), x=s(), dy=s(), dg=s(), dx=s(), carries=_Claimed(dev, (2, 1, 8), torch.float32), h0=v(), dh_last=v(), dh0=v(),
                workspace=_Claimed(dev, (64,), torch.uint8), err_word=_Claimed(dev, (1,), torch.int32))


def _product(dev):
    m = lambda *s: _Claimed(dev, s, torch.bfloat16)  # noqa: E731
    return dict(x=m(4, 8), w=m(6, 8), y=m(4, 6), bias=_Claimed(dev, (6,), torch.float32), residual=m(4, 6), z=m(4, 6),
                workspace=_Claimed(dev, (64,), torch.uint8), err_word=_Claimed(dev, (1,), torch.int32))


def _product_back(dev):
    m = lambda *s: _Claimed(dev, s, torch.bfloat16)  # noqa: E731
    return dict(dy=m(4, 6), x=m(4, 8), w=m(6, 8), z=m(4, 6), dx=m(4, 8), dw=m(6, 8), db=_Claimed(dev, (6,), torch.float32),
                workspace=_Claimed(dev, (64,), torch.uint8), err_word=_Claimed(dev, (1,), torch.int32))


CALLS = [(lambda **k: dastac.linrec_forward(gate=dastac.GATE_LOG, **k), _recurrence),
         (lambda **k: dastac.linrec_backward(gate=dastac.GATE_LOG, **k), _recurrence_back),
         (lambda **k: dastac.linear_forward(act=dastac.ACT_SILU, **k), _product),
         (lambda **k: dastac.linear_backward(act=dastac.ACT_SILU, **k), _product_back)]


@pytest.mark.parametrize("dev", [0, 1])
@pytest.mark.parametrize("call,tensors", CALLS)
def test_calls_run_on_the_gpu_of_their_tensors(library, call, tensors, dev):
    call(**tensors(dev))
    assert [c[1:] for c in library.calls] == [(dev, 70 + dev)]


@pytest.mark.parametrize("call,tensors", CALLS)
def test_tensors_of_another_gpu_or_of_the_host_are_refused(library, call, tensors):
    names = list(tensors(1))
    for name in names:
        for other in (0, -1):
            k = tensors(1)
            k[name] = _Claimed(other, tuple(k[name].shape), k[name].dtype) if other == 0 else k[name]._t
            with pytest.raises(AssertionError):
                call(**k)
    k = tensors(1)
    k["workspace"]._t = torch.empty(128, dtype=torch.uint8)[::2]   # its bytes do not lie behind one another
    with pytest.raises(AssertionError):
        call(**k)
    assert not library.calls


def test_workspace_of_the_recurrence_is_asked_for_on_each_gpu(library):
    for dev in (0, 1, 0, 1):
        assert dastac.linrec_workspace(_Claimed(dev, (2, 900, 8), torch.float32)) == 1000 + dev
    assert library.calls == [("linrec_workspace", 0, None), ("linrec_workspace", 1, None)]
