"""What the Python entry points of the chains do before anything is launched (no GPU: tensors and the library are stand-ins)."""
import threading
import types

import pytest
import torch

import paper_2604_03446_b200.binding as b


class Fake:
    """A tensor as the entry points look at it: a CUDA one by what it says."""

    def __init__(self, *shape, dtype=torch.bfloat16, device=0, requires_grad=False):
        self.shape, self.dtype, self.device, self.requires_grad = torch.Size(shape), dtype, torch.device("cuda", device), requires_grad

    def get_device(self):
        return self.device.index

    def stride(self, i=None):
        s = torch.empty(self.shape, device="meta").stride()
        return s if i is None else s[i]

    def new_empty(self, shape, dtype=None):
        return Fake(*([shape] if isinstance(shape, int) else shape), dtype=dtype or self.dtype)

    def data_ptr(self):
        return 4096

    def is_contiguous(self):
        return True


def attention(**kw):
    return Fake(2, 3, 4, 64, **kw), Fake(2, 5, 2, 64, **kw), Fake(2, 5, 2, 64, **kw)


def block(**kw):
    return Fake(4, 32, **kw), Fake(64, 32, **kw), Fake(64, 32, **kw), Fake(16, 64, **kw)


def refused(call, *args, **kw):
    with pytest.raises(b.MmeeError) as e:
        call(*args, **kw)
    assert e.value.code == b.ERR_ARG
    return str(e.value)


def calls(which):
    """Each entry point with sound arguments, its tensors made by `which`."""
    q, k, v = attention(**which)
    o, w = Fake(2, 3, 4, 64, **which), block(**which)
    return [(b.mmee_attention, (q, k, v)), (b.mmee_attention_backward, (o, q, k, v, o, None)), (b.mmee_gated_ffn, w),
            (b.mmee_gated_ffn_backward, (Fake(4, 16, **which), *w, (Fake(4, 64, **which), None)))]


# --- gradients ------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("i", range(4))
def test_tensors_that_want_a_gradient_are_refused_where_it_would_be_lost(i):
    call, args = calls(dict(requires_grad=True))[i]
    assert "gradient" in refused(call, *args)


@pytest.mark.parametrize("i", range(4))
def test_tensors_that_want_a_gradient_pass_where_none_is_recorded(i, monkeypatch):
    """Under no_grad (and in a Function's own forward and backward) the call goes on: to its next question, here."""
    class GoesOn(Exception):
        pass

    def device():
        raise GoesOn
    monkeypatch.setattr(b, "_current_device", device)
    call, args = calls(dict(requires_grad=True))[i]
    with torch.no_grad(), pytest.raises(GoesOn):
        call(*args)


def test_dual_numbers_are_refused(monkeypatch):
    import torch.autograd.forward_ad as fwd
    monkeypatch.setattr(fwd, "unpack_dual", lambda t: types.SimpleNamespace(tangent=t))
    for call, args in calls({}):
        with fwd.dual_level():
            assert "gradient" in refused(call, *args)


# --- two threads ----------------------------------------------------------------------------------------------------

def test_a_first_call_of_two_threads_at_once(monkeypatch):
    """Whoever finds the module's view of torch made finds its table of types filled."""
    seen = []

    class Table(dict):
        def update(self, *args):
            seen.append(b._torch)                      # what a thread that comes in now would go by
            super().update(*args)

    monkeypatch.setattr(b, "_torch", None)
    monkeypatch.setattr(b, "_type_codes", Table())
    codes = []
    threads = [threading.Thread(target=lambda: codes.append(b._chain_code("x", 4, *attention()))) for _ in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert codes == [b.BF16] * 4 and seen and seen[0] is None and all(v is None or b._type_codes for v in seen)


# --- streams --------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("i", range(4))
def test_a_stream_of_another_device_than_the_tensors_is_refused(i, monkeypatch):
    """(It was dropped: the call ran on the current stream of the tensors' device.)"""
    entered = []
    monkeypatch.setattr(torch.cuda, "stream", lambda s: entered.append(s) or pytest.fail("made current"))
    call, args = calls({})[i]
    stream = types.SimpleNamespace(device=torch.device("cuda", 1), device_index=1, cuda_stream=4096)
    assert "stream" in refused(call, *args, stream=stream) and not entered


def test_a_stream_of_the_tensors_device_is_made_current(monkeypatch):
    class Entered(Exception):
        pass

    def enter(s):
        raise Entered
    monkeypatch.setattr(torch.cuda, "stream", enter)
    for call, args in calls({}):
        with pytest.raises(Entered):
            call(*args, stream=types.SimpleNamespace(device=torch.device("cuda", 0), device_index=0, cuda_stream=4096))


# --- arguments that no call struct holds -----------------------------------------------------------------------------

@pytest.fixture
def no_library(monkeypatch):
    """Everything up to the library's call, which a sound call gets to."""
    made = []

    class Calls:
        def __getattr__(self, name):
            return lambda *args: (None if name.endswith("workspace") else made.append(name)) or b.OK
    monkeypatch.setattr(b, "_chain", Calls)
    monkeypatch.setattr(b, "_current_device", lambda: 0)
    monkeypatch.setattr(b, "_current_stream", lambda: 0)
    return made


def test_sound_calls_get_to_the_library(no_library):
    b.mmee_attention(*attention())
    b.mmee_gated_ffn(*block(), save=True)
    b.mmee_gated_ffn_backward(Fake(4, 16), *block(), (Fake(4, 64), KEPT))
    assert no_library == ["attention", "gated_ffn", "gated_ffn_backward"]


KEPT = Fake(2, 4, 64, dtype=torch.float32)


@pytest.mark.parametrize("scale", ["a", 1e39, 1j, [1.0]])
def test_a_scale_that_is_no_32_bit_number_is_refused(scale, no_library):
    refused(b.mmee_attention, *attention(), scale=scale)
    assert not no_library


@pytest.mark.parametrize("activation", [-1, 1 << 32, "silu", 1.5, None])
def test_an_activation_that_is_no_number_of_one_is_refused(activation, no_library):
    refused(b.mmee_gated_ffn, *block(), activation=activation)
    refused(b.mmee_gated_ffn_backward, Fake(4, 16), *block(), (Fake(4, 64), KEPT), activation=activation)
    assert not no_library


def test_sizes_of_more_than_32_bits_are_refused(no_library):
    refused(b.mmee_gated_ffn, Fake((1 << 32) + 4, 32), *block()[1:])
    refused(b.mmee_attention, Fake(2, 1 << 32, 4, 64), *attention()[1:])
    assert not no_library


@pytest.mark.parametrize("saved", [None, (), (Fake(4, 64), None), (None, KEPT), (Fake(4, 64), KEPT, KEPT), [Fake(4, 64), KEPT]])
def test_what_the_forward_call_did_not_return_is_refused(saved, no_library):
    refused(b.mmee_gated_ffn_backward, Fake(4, 16), *block(), saved)
    assert not no_library
