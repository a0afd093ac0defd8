"""Arguments of the recurrent block's operators that have to be refused before the library is called, on the CPU: the binding is given CPU tensors and a library that notes
its calls."""
from types import SimpleNamespace

import pytest
import torch

import paper_2604_16834_amd as hx
from test_block_arguments import Library, words

N, LEVEL, CHANNELS, HEADS = 16, 5, 4, 2


@pytest.fixture
def library(monkeypatch):
    lib = Library()
    monkeypatch.setattr(hx.binding, "_expect_device", "cpu")
    monkeypatch.setattr(hx.binding, "_lib", lib)
    return lib


KEY = SimpleNamespace(handle=SimpleNamespace(value=None))
CTX = SimpleNamespace(handle=None, N=N, _check=lambda rc: None, workspace=lambda n: words(n, dtype=torch.uint8))
KEYS = SimpleNamespace(handle=None)


def ct(n=CHANNELS, limbs=LEVEL + 1, **kw):
    return words(n, 2, limbs, N, **kw)


def scan(**kw):
    return hx.he_scan_gated(CTX, LEVEL, **{**dict(x=ct(), gate=ct(HEADS), k=[1, 2], rot_keys=[KEY] * 2, cross_keys=[KEY] * 2), **kw})


def back(**kw):
    a = {**dict(grad=ct(), gate=ct(HEADS), states=ct(limbs=LEVEL - 1), k=[1, 2], rot_keys=[KEY] * 2, cross_keys=[KEY] * 2, back_rot=KEYS, back_cross=KEYS), **kw}
    return hx.he_scan_gated_backward(CTX, LEVEL, **a)


def step(**kw):
    return hx.he_scan_step(CTX, LEVEL, **{**dict(gate=ct(HEADS), state=ct(), cross_key=KEYS, x=ct(), k=3), **kw})


def norm(**kw):
    return hx.he_layer_norm(CTX, LEVEL, **{**dict(x=ct(), k_eps=1, k_slope=1, k_start=1, k_newton=(), rlk=KEYS, gain=ct(limbs=3), bias=ct(limbs=3)), **kw})


def grad(**kw):
    return hx.he_layer_norm_backward(CTX, LEVEL, **{**dict(grad=ct(), norm=ct(), inv=words(2, LEVEL + 1, N), k_grad=1, k_norm=-1, rlk=KEYS, gain=ct(), sum_keys=[[KEY], [KEY] * 3]), **kw})


CALLS = {"he_scan_gated": scan, "he_scan_gated_backward": back, "he_scan_step": step, "he_layer_norm": norm, "he_layer_norm_backward": grad}
OUTS = {"he_scan_gated": dict(out=(CHANNELS, 2, LEVEL - 1, N)), "he_scan_gated_backward": dict(dx=(CHANNELS, 2, LEVEL - 1, N), dgate=(HEADS, 2, LEVEL - 2, N)),
        "he_scan_step": dict(out=(CHANNELS, 2, LEVEL, N)), "he_layer_norm": dict(norm=(CHANNELS, 2, 3, N), inv=(2, 4, N), out=(CHANNELS, 2, 2, N)),
        "he_layer_norm_backward": dict(dx=(CHANNELS, 2, LEVEL - 3, N), dgain=(CHANNELS, 2, LEVEL, N), dbias=(CHANNELS, 2, LEVEL, N))}
OPERANDS = {"he_scan_gated": dict(x=CHANNELS, gate=HEADS), "he_scan_gated_backward": dict(grad=CHANNELS, gate=HEADS, states=CHANNELS), "he_scan_step": dict(gate=HEADS, state=CHANNELS, x=CHANNELS),
            "he_layer_norm": dict(x=CHANNELS, gain=CHANNELS, bias=CHANNELS), "he_layer_norm_backward": dict(grad=CHANNELS, norm=CHANNELS, gain=CHANNELS)}
each = pytest.mark.parametrize("name", list(CALLS))


@each
def test_well_formed_arguments_reach_the_library(library, name):
    outs = CALLS[name]()
    outs = outs if isinstance(outs, tuple) else (outs,)
    assert [tuple(o.shape) for o in outs] == list(OUTS[name].values())
    CALLS[name](**{k: words(*s) for k, s in OUTS[name].items()}, ws=words(512, dtype=torch.uint8))
    CALLS[name](**{k: words(*s, dtype=torch.uint64) for k, s in OUTS[name].items()})
    assert library.calls == [name] * 3


@each
def test_outputs_are_words_of_the_right_number(library, name):
    for out, shape in OUTS[name].items():
        for bad in [words(*shape, dtype=d) for d in (torch.uint8, torch.int32, torch.float64)] + [words(*shape[:-1], shape[-1] - 1), words(*shape, 2)[..., 0]]:
            with pytest.raises(ValueError):
                CALLS[name](**{out: bad})
    assert library.calls == []


@each
def test_operands_are_words_of_enough_limbs_at_equal_distances(library, name):
    for arg, n in OPERANDS[name].items():
        least = {"states": LEVEL - 1, "gain": 3 if name == "he_layer_norm" else LEVEL + 1, "bias": 3}.get(arg, LEVEL + 1)
        for bad in (ct(n, least - 1), ct(n, least, dtype=torch.int32), ct(n, least, dtype=torch.float64), ct(n, least)[..., :-1], ct(n, least).transpose(2, 3), ct(n, least)[:, :1],
                    words(n, 2, least, 2 * N)[..., ::2], words(2, least, N)):
            with pytest.raises(ValueError):
                CALLS[name](**{arg: bad})
    assert library.calls == []


def test_keys_and_constants(library):
    big = 1 << 63
    for bad in (dict(k=[1]), dict(rot_keys=[KEY]), dict(cross_keys=[KEY] * 3), dict(rot_keys=[KEY, None]), dict(cross_keys=[None, KEY]), dict(k=[1, big]), dict(k=[-big - 1, 1])):
        with pytest.raises(ValueError):
            scan(**bad)
        with pytest.raises(ValueError):
            back(**bad)
    for bad in (dict(states=None), dict(back_rot=None), dict(back_cross=None)):
        with pytest.raises(ValueError):
            back(**bad)
    for bad in (dict(k=big), dict(k=-big - 1)):
        with pytest.raises(ValueError):
            step(**bad)
    for bad in (dict(k_eps=big), dict(k_slope=big), dict(k_start=-big - 1), dict(k_bias=big), dict(k_newton=(big,)), dict(gain=None), dict(gain=None, bias=None, out=ct(limbs=2))):
        with pytest.raises(ValueError):
            norm(**bad)
    for bad in (dict(k_grad=big), dict(k_norm=-big - 1), dict(sum_keys=[[None]]), dict(inv=ct(1))):
        with pytest.raises(ValueError):
            grad(**bad)
    assert library.calls == []


def test_what_is_not_wanted_is_not_needed(library):
    dx, dgate = back(want_gate=False, states=None, back_rot=None, back_cross=None)
    assert dgate is None and tuple(dx.shape) == (CHANNELS, 2, LEVEL - 1, N)
    dx, dgain, dbias = grad(want_gain=False, want_bias=False, sum_keys=())
    assert dgain is None and dbias is None
    assert norm(gain=None, bias=None)[2] is None
    step(x=None)
    assert library.calls == ["he_scan_gated_backward", "he_layer_norm_backward", "he_layer_norm", "he_scan_step"]
