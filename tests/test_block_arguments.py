"""Arguments of the transformer block's operators that have to be refused before the library is called, on the CPU: the binding is given CPU
tensors and a library that notes its calls."""
from types import SimpleNamespace

import pytest
import torch

import paper_2604_16834_amd as hx
from paper_2604_16834_amd.block import linear_scale, quantise_weights

N, LEVEL = 16, 3


class Library:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            if name.endswith("_bytes"):
                return 256
            self.calls.append(name)
            return 0
        return call


@pytest.fixture
def library(monkeypatch):
    lib = Library()
    monkeypatch.setattr(hx.binding, "_expect_device", "cpu")
    monkeypatch.setattr(hx.binding, "_lib", lib)
    return lib


def words(*shape, dtype=torch.int64):
    return torch.zeros(*shape, dtype=dtype)


def calls(out=None, bias=None, cos=None, sin=None, ws=None):
    """The three operators with well-formed arguments but for those given."""
    ctx = SimpleNamespace(handle=None, N=N, _check=lambda rc: None, workspace=lambda n: words(n, dtype=torch.uint8))
    x, w = words(1, 4, 2, LEVEL + 1, N), words(1, 4, 4, dtype=torch.int8)
    table = words(2, LEVEL + 1, N)
    return {
        "he_linear_grouped": lambda: hx.he_linear_grouped(ctx, LEVEL, (1,), x, w, 3, bias=words(1, 4, LEVEL + 1) if bias is None else bias,
                                                          out=words(1, 4, 2, LEVEL, N) if out is None else out, ws=ws),
        "he_rope_axes": lambda: hx.he_rope_axes(ctx, LEVEL, x, table if cos is None else cos, table if sin is None else sin,
                                                out=words(1, 4, 2, LEVEL, N) if out is None else out, ws=ws),
        "he_norm_gate": lambda: hx.he_norm_gate(ctx, LEVEL, x[0], 1, 1, 1, (), SimpleNamespace(handle=None),
                                                out=words(4, 2, LEVEL - 2, N) if out is None else out, ws=ws),
    }


def out_of(name, dtype):
    return words(4, 2, LEVEL - 2, N, dtype=dtype) if name == "he_norm_gate" else words(1, 4, 2, LEVEL, N, dtype=dtype)


@pytest.mark.parametrize("name", ["he_linear_grouped", "he_rope_axes", "he_norm_gate"])
def test_well_formed_arguments_reach_the_library(library, name):
    calls(ws=words(512, dtype=torch.uint8))[name]()
    calls(out=out_of(name, torch.uint64))[name]()
    assert library.calls == [name, name]


# As many elements as there are words, of a type that is shorter, would be read or written past their end; doubles are not residues.
@pytest.mark.parametrize("dtype", [torch.uint8, torch.int32, torch.float64])
@pytest.mark.parametrize("name", ["he_linear_grouped", "he_rope_axes", "he_norm_gate"])
def test_outputs_have_to_be_words(library, name, dtype):
    with pytest.raises(ValueError):
        calls(out=out_of(name, dtype))[name]()
    assert library.calls == []


@pytest.mark.parametrize("dtype", [torch.uint8, torch.int32, torch.float64])
def test_biases_and_tables_have_to_be_words(library, dtype):
    with pytest.raises(ValueError):
        calls(bias=words(1, 4, LEVEL + 1, dtype=dtype))["he_linear_grouped"]()
    for table in ("cos", "sin"):
        with pytest.raises(ValueError):
            calls(**{table: words(2, LEVEL + 1, N, dtype=dtype)})["he_rope_axes"]()
    assert library.calls == []


def test_operands_of_other_calls_have_eight_byte_elements(library):
    ctx = SimpleNamespace(handle=None, N=N, _check=lambda rc: None, workspace=lambda n: words(n, dtype=torch.uint8))
    ct = words(2, LEVEL + 1, N)
    hx.ckks_rescale(ctx, ct, LEVEL, out=words(2, LEVEL, N), ws=words(512, dtype=torch.uint8))
    with pytest.raises(ValueError):
        hx.ckks_rescale(ctx, ct, LEVEL, out=words(2, LEVEL, N, dtype=torch.uint8))
    with pytest.raises(ValueError):
        hx.ckks_rescale(ctx, ct.to(torch.uint8), LEVEL)
    assert library.calls == ["ckks_rescale"]


@pytest.mark.parametrize("gain", [0.0, -1.0, float("nan"), float("inf"), float("-inf")])
def test_a_gain_has_to_be_positive_and_finite(gain):
    """A negative or zero gain would leave the multiplier at one: outputs at a scale far below the noise, and no error."""
    with pytest.raises(ValueError):
        quantise_weights([[0.5, -0.25]], (1 << 50) - 27, 16, gain=gain)


def test_a_multiplier_is_at_least_one_and_its_scale_is_told():
    """Where step * q_level * gain is below one the scale grows instead; linear_scale follows the multiplier that is used."""
    q = (1 << 20) - 3
    qw = quantise_weights([[1.0, -0.5]], q, 32)
    assert qw.multiplier == 1 and qw.step * q < 0.5
    assert linear_scale(2.0 ** 30, qw, q) == 2.0 ** 30 / qw.step / q
