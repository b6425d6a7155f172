"""A few-token decoder reads its weights where they are at the call, as the other planned layers
do (CPU only: the library's call is recorded instead of made)."""
import contextlib

import pytest
import torch

import paper_2604_01622_amd as ec
from paper_2604_01622_amd import binding

D, E, H, HS = 128, 4, 64, 64
ORDER = ("X", "Wg", "W1", "W3", "W2", "Ws1", "Ws3", "Ws2")


class Recorder:
    """The library, with the arguments of its last few-token call kept."""

    def __init__(self, real):
        self.real = real

    def __getattr__(self, name):
        return getattr(self.real, name)

    def ec_tc_decode(self, p, k, scales, *rest):
        self.got = dict(zip(ORDER, rest))
        self.scales = {n: getattr(scales._obj, n) for n, _ in binding._MxScales._fields_}
        return 0


@pytest.fixture
def calls(monkeypatch):
    rec = Recorder(ec.lib())
    monkeypatch.setattr(binding, "lib", lambda: rec)
    monkeypatch.setattr(binding, "_on", lambda dev: contextlib.nullcontext())
    monkeypatch.setattr(binding, "_raw_stream", lambda dev: 0)
    monkeypatch.setattr(binding, "_rows", lambda name, t: (1, t.shape[-1]))
    # the host stands for the GPU
    monkeypatch.setattr(binding, "_operand", _operand)
    return rec


def _operand(name, t, dtype, shape=None, device=None):
    if not (isinstance(t, torch.Tensor) and t.dtype == dtype and (shape is None or t.shape == shape)
            and t.is_contiguous()):
        raise ec.ECError(2, f"{name}")


def weight(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def eight(*shape):
    return ec.Mx(torch.zeros(shape, dtype=torch.uint8).view(torch.float8_e4m3fn),
                 torch.zeros((*shape[:-1], shape[-1] // 32), dtype=torch.uint8).view(
                     torch.float8_e8m0fnu))


def decoder(make):
    return ec.TcDecoder(weight(E, D), make(E, H, D), make(E, H, D), make(E, D, H), 2,
                        shared=[make(HS, D), make(HS, D), make(D, HS)], max_tokens=8)


def check(dec, calls):
    dec.forward(weight(3, D))
    held = dict(zip(ORDER[1:], (dec.Wg, dec.W1, dec.W3, dec.W2, *dec.shared)))
    for n, t in held.items():
        assert calls.got[n] == binding._codes(t).data_ptr(), n
        if n != "Wg":
            assert calls.scales[n] == (t.scales.data_ptr() if isinstance(t, ec.Mx) else None), n


@pytest.mark.parametrize("make", [weight, eight])
def test_other_weights(calls, make):
    dec = decoder(make)
    check(dec, calls)
    shapes = {"W1": (E, H, D), "W3": (E, H, D), "W2": (E, D, H)}
    for n, s in shapes.items():
        setattr(dec, n, make(*s))
        check(dec, calls)
    dec.Wg = weight(E, D)
    check(dec, calls)
    dec.shared = (make(HS, D), make(HS, D), make(D, HS))
    check(dec, calls)


@pytest.mark.parametrize("make", [weight, eight])
def test_other_memory(calls, make):
    """The same tensors, moved (their old memory is someone else's)."""
    dec = decoder(make)
    for t in (dec.Wg, dec.W1, dec.W3, dec.W2, *dec.shared):
        for part in (t if isinstance(t, ec.Mx) else (t,)):
            keep, part.data = part.data, part.data.clone()
            check(dec, calls)
            del keep


@pytest.mark.parametrize("make", [weight, eight])
def test_weights_that_do_not_fit_are_refused(calls, make):
    other = {weight: eight, eight: weight}[make]
    for n, bad in (("Wg", weight(E + 1, D)), ("W1", make(E, H, D // 2)), ("W1", make(E - 1, H, D)),
                   ("W2", make(E, D, 2 * H)), ("W3", other(E, H, D)), ("W2", None),
                   ("Wg", weight(E, D).float()), ("shared", None),
                   ("shared", (make(HS, D), make(HS, D))),
                   ("shared", (make(2 * HS, D), make(2 * HS, D), make(D, 2 * HS)))):
        dec = decoder(make)
        good = getattr(dec, n)
        setattr(dec, n, bad)
        with pytest.raises(ec.ECError):
            dec.forward(weight(3, D))
        setattr(dec, n, good)
        check(dec, calls)
    dec = decoder(make)
    if make is weight:
        dec.W1.data = dec.W1.data[:1]           # the same address
        with pytest.raises(ec.ECError):
            dec.forward(weight(3, D))


def test_the_number_of_choices_is_fixed(calls):
    """The places of the choice and the gates are planned for it: with 64 tokens and one choice of
    256 narrow experts, the workspace would do for 16 tokens and ten choices, whose 160 pairs do
    not fit the 64 places."""
    size = ec.lib().ec_tc_decode_workspace_size

    def problem(n):
        return binding.Problem(n, 64, 256, 64, [0, n], [0], 1.0, torch.bfloat16).ref

    assert size(problem(16), 10) <= size(problem(64), 1)
    dec = decoder(weight)
    with pytest.raises(AttributeError):
        dec.top_k = 3
    assert dec.top_k == 2 and dec.experts.shape == (8, 2)
