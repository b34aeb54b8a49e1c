"""The dense operators refuse tensors that lie on different devices, before
anything is allocated or launched: a kernel would read the other device's
addresses.  The tensors are stand-ins that only claim a device."""
import pytest
import torch

from paper_2512_00385_amd import ezsp

BF, F32 = torch.bfloat16, torch.float32


class Claims(torch.Tensor):
    """A host tensor that gives itself out as device `index`'s."""
    index = 0
    is_cuda = property(lambda self: True)
    device = property(lambda self: torch.device("cuda", self.index))

    def get_device(self):
        return self.index


class ClaimsOther(Claims):
    index = 1


def on(cls, *shape, dtype=BF):
    return torch.Tensor._make_subclass(cls, torch.zeros(shape, dtype=dtype))


def arguments(fields, other):
    return {name: on(ClaimsOther if name == other else Claims, *shape,
                     dtype=dtype) for name, (shape, dtype) in fields.items()}


N, K, M = 4, 8, 16
ROWS_K, ROWS_M, MAT = ((N, K), BF), ((N, M), BF), ((K, M), BF)
OPERATORS = {
    "layer_norm": dict(x=ROWS_K, weight=((K,), F32), bias=((K,), F32)),
    "layer_norm_backward": dict(x=ROWS_K, dy=ROWS_K, mean=((N,), F32),
                                rstd=((N,), F32), weight=((K,), F32),
                                dres=ROWS_K),
    "linear": dict(x=ROWS_K, w=MAT, bias=((M,), F32), residual=ROWS_M),
    "linear_backward": dict(x=ROWS_K, dy=ROWS_M, w=MAT, z=ROWS_M),
    "gated_ff": dict(x=ROWS_K, w_gate=MAT, w_up=MAT, b_gate=((M,), F32),
                     b_up=((M,), F32)),
    "gated_ff_backward": dict(x=ROWS_K, dh=ROWS_M, w_gate=MAT, w_up=MAT,
                              gate=ROWS_M, up=ROWS_M),
}


@pytest.fixture(autouse=True)
def nothing_is_reached(monkeypatch):
    class Library:
        def __getattr__(self, name):
            raise AssertionError(f"{name} was called")

    def allocate(*args, **kw):
        raise AssertionError("a result was allocated")
    monkeypatch.setattr(ezsp, "load", Library)
    monkeypatch.setattr(torch, "empty", allocate)


@pytest.mark.parametrize("op,other", [(op, name) for op, fields in
                                      OPERATORS.items() for name in fields
                                      if name != "x"])
def test_two_devices_are_refused(op, other):
    args = arguments(OPERATORS[op], other)
    with pytest.raises(ValueError, match=f"{other} must be on device 0"):
        getattr(ezsp, op)(**args)


@pytest.mark.parametrize("op", OPERATORS)
def test_one_device_gets_as_far_as_its_results(op):
    with pytest.raises(AssertionError, match="allocated"):
        getattr(ezsp, op)(**arguments(OPERATORS[op], None))


@pytest.mark.parametrize("current", [0, 1])
@pytest.mark.parametrize("op", OPERATORS)
def test_calls_run_on_their_tensors_device(monkeypatch, op, current):
    # a default stream's handle names the current device's, whichever that is
    state = dict(current=current, called=None)

    class Current:
        def __init__(self, device):
            self.index = device

        def __enter__(self):
            self.before, state["current"] = state["current"], self.index

        def __exit__(self, *error):
            state["current"] = self.before

    class Library:
        def __getattr__(self, name):
            def entry(*args):
                state["called"] = (name, state["current"], args[-1])
                return ezsp.OK
            return entry
    monkeypatch.setattr(ezsp, "load", Library)
    monkeypatch.setattr(ezsp, "_dense_bytes", lambda *sizes: 512)
    monkeypatch.setattr(ezsp, "_raw_stream", lambda index: 100 + index)
    monkeypatch.setattr(ezsp, "_current_device", lambda: state["current"])
    monkeypatch.setattr(torch.cuda, "device", Current)
    monkeypatch.setattr(torch, "empty", lambda size, dtype, device:
                        torch.zeros(size, dtype=dtype))
    args = {name: on(ClaimsOther, *shape, dtype=dtype)
            for name, (shape, dtype) in OPERATORS[op].items()}
    getattr(ezsp, op)(**args)
    assert state == dict(current=current, called=("ezsp_" + op, 1, 101))
