"""What the Python calls of the drafting operators hand to the library, without a GPU: the
library, the device and its tensors are stand-ins."""

import weakref
from types import SimpleNamespace

import pytest
import torch

import paper_2512_04752_amd as sv
from paper_2512_04752_amd import binding as B


@pytest.fixture
def made(monkeypatch):
    """Workspaces that calls make, as weak references, and whether each lived when the library
    was called."""
    got = SimpleNamespace(refs=[], alive=[], asked=[])

    def make(nbytes, index, stream):
        t = torch.empty(nbytes, dtype=torch.uint8)
        got.refs.append(weakref.ref(t))
        return t

    def launch(*args):
        got.alive.append(got.refs[-1]() is not None)
        return 0

    fake = SimpleNamespace(spec_w4_product_bytes=lambda *a: got.asked.append(a) or 4096, spec_w4_linear=launch, spec_w4_gate_up=launch,
                           spec_beam_workspace_bytes=lambda *a: 4096, spec_beam_select=launch,
                           spec_kv4_reorder_bytes=lambda *a: 4096, spec_kv4_reorder=launch)
    monkeypatch.setattr(B, "lib", lambda: fake)
    monkeypatch.setattr(B, "_made_workspace", make)
    monkeypatch.setattr(B, "_device_rows", lambda t, *a: t.shape[1])
    monkeypatch.setattr(B, "_device_workspace", lambda t, index: (t.data_ptr(), t.numel()))
    monkeypatch.setattr(B, "_device_stream", lambda index, stream: None)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    return got


def matrix(rows, cols):
    return SimpleNamespace(index=0, rows=rows, cols=cols, needs={}, struct=B.spec_w4(0, rows, cols))


def test_products_hold_their_workspace_until_they_are_launched(made):
    m, x = matrix(48, 64), torch.zeros(3, 64, dtype=torch.bfloat16)
    sv.spec_w4_linear(m, x, torch.zeros(3, 48))
    sv.spec_w4_gate_up(m, m, x, torch.zeros(3, 48, dtype=torch.bfloat16))
    assert made.alive == [True, True]
    assert all(ref() is None for ref in made.refs)         # and no longer


def test_products_ask_for_their_own_rows_alone(made):
    """One plan, not a search over all numbers of rows up to theirs, and once."""
    m = matrix(48, 64)
    for n in (3, 700, 3):
        x = torch.zeros(n, 64, dtype=torch.bfloat16)
        sv.spec_w4_linear(m, x, torch.zeros(n, 48))
        sv.spec_w4_gate_up(m, m, x, torch.zeros(n, 48, dtype=torch.bfloat16))
    assert made.asked == [(48, 64, 3, 0), (48, 64, 3, 1), (48, 64, 700, 0), (48, 64, 700, 1)]


@pytest.mark.parametrize("rows,cols", [(16, 32), (293, 1088), (4096, 14336), (2048, 2048), (40, 70016)])
def test_a_product_needs_what_the_search_finds(rows, cols):
    most = 0
    for n in range(1, 150):
        most = max(most, *(sv.spec_w4_product_bytes(rows, cols, n, pair) for pair in (False, True)))
        if n in (1, 2, 16, 17, 64, 149):
            assert sv.spec_w4_workspace_bytes(rows, cols, n) == most
    assert sv.spec_w4_product_bytes(rows, cols, 5000) == 0                # so many rows are not split


def test_a_product_s_bytes_of_invalid_arguments():
    for bad in ((0, 32, 1, 0), (1, 40, 1, 0), (48, 64, 0, 0), (48, 64, -1, 0), (48, 64, (1 << 20) + 1, 0), (48, 64, 1, 2)):
        assert B.lib().spec_w4_product_bytes(*bad) == 0


def test_a_matrix_reads_back_into_its_own_shape(monkeypatch):
    """Another shape of as many bytes would be read as another layout."""
    calls = []
    monkeypatch.setattr(B, "spec_w4_unpack", lambda data, out, stream=None: calls.append(tuple(out.shape)))
    m = sv.W4Matrix.__new__(sv.W4Matrix)
    m.rows, m.cols, m.data = 32, 256, None
    for shape in ((64, 128), (32, 128), (16, 256), (256, 32), (8192,)):
        with pytest.raises(ValueError, match="32"):
            m.unpack(torch.empty(shape, dtype=torch.bfloat16))
    m.unpack(torch.empty(32, 256, dtype=torch.bfloat16))
    assert calls == [(32, 256)]


class Matrix:
    """Stands in for a matrix of W4Weights; a tensor's device is what it is said to be."""

    devices = {}

    def __init__(self, w, stream=None):
        self.index = self.devices.get(w.data_ptr(), -1)
        self.struct = B.spec_w4(0, *w.shape)


@pytest.mark.parametrize("field", [None, "wo", "w_gate", "w_up", "w_down"])
@pytest.mark.parametrize("layer", [0, 1])
def test_weights_lie_on_one_device(monkeypatch, layer, field):
    """A step's kernels run on one device, and read every matrix."""
    def bf16(*shape):
        return torch.zeros(shape, dtype=torch.bfloat16)

    W = dict(tok_embed=bf16(128, 64), final_norm=bf16(64), lm_head=bf16(128, 64), layers=[
        dict(attn_norm=bf16(64), ffn_norm=bf16(64), wq=bf16(64, 64), wk=bf16(64, 64), wv=bf16(64, 64), wo=bf16(64, 64),
             w_gate=bf16(96, 64), w_up=bf16(96, 64), w_down=bf16(64, 96)) for _ in range(2)])
    monkeypatch.setattr(B, "W4Matrix", Matrix)
    monkeypatch.setattr(Matrix, "devices", {} if field is None else {W["layers"][layer][field].data_ptr(): 1})
    if field is None:
        assert sv.W4Weights(W).shape == (2, 64, 128)
    else:
        with pytest.raises(ValueError, match="device"):
            sv.W4Weights(W)
