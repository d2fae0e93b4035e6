"""The microscaled calls without a GPU: everything the host refuses before it touches CUDA."""
import ctypes

import pytest
import torch

import paper_2604_14156_b200 as cs
from paper_2604_14156_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return cs.load_library()


P = 1 << 20       # an aligned address that no refused call reads


def test_calls_are_declared_and_exported(lib):
    names = {"cs_mx_quantize", "cs_mx_dequantize", "cs_mx_pack", "cs_mx_norm", "cs_mx_ffn", "cs_mx_ffn_shared"}
    assert names <= set(cs.exported_symbols())


@pytest.mark.parametrize("change,code", [
    (dict(w=None), 1), (dict(codes=None), 1), (dict(scales=None), 1), (dict(dtype=2), 3), (dict(dtype=-1), 3), (dict(rows=0), 2),
    (dict(cols=0), 2), (dict(rows=-1), 2), (dict(ld=95), 2), (dict(codes=P + 8), 3), (dict(w=P + 2), 3),
    (dict(rows=1 << 30), 2), (dict(transpose=1, rows=(1 << 24) - 255, cols=1, ld=1), 2),
    (dict(transpose=1, rows=1 << 30, cols=1 << 10, ld=1 << 10), 2),
])
def test_quantize_refusals(lib, change, code):
    a = dict(w=P, dtype=0, rows=64, cols=96, ld=96, transpose=0, codes=P, scales=P)
    a.update(change)
    assert lib.cs_mx_quantize(a["w"], a["dtype"], a["rows"], a["cols"], a["ld"], a["transpose"], a["codes"], a["scales"], None) == code


@pytest.mark.parametrize("change,code", [
    (dict(w=None), 1), (dict(codes=None), 1), (dict(scales=None), 1), (dict(dtype=2), 3), (dict(rows=0), 2), (dict(cols=0), 2),
    (dict(ld=95), 2), (dict(codes=P + 4), 3), (dict(w=P + 1), 3), (dict(rows=1 << 30), 2),
])
def test_dequantize_refusals(lib, change, code):
    a = dict(w=P, dtype=1, rows=64, cols=96, ld=96, codes=P, scales=P)
    a.update(change)
    assert lib.cs_mx_dequantize(a["codes"], a["scales"], a["rows"], a["cols"], a["dtype"], a["w"], a["ld"], None) == code


def test_null_plans_and_layers_are_reported(lib):
    m, layer = binding._MxMatrix(P, P), binding._MxLayer(P, P, P, P)
    assert lib.cs_mx_pack(None, ctypes.byref(m), ctypes.byref(m), ctypes.byref(m), P, P, P, P, None) == 1
    assert lib.cs_mx_norm(None, P, 0, None, 0, None, 1, None, None, P, P, None) == 1
    assert lib.cs_mx_ffn(None, ctypes.byref(layer), P, P, P, 1, P, None) == 1
    assert lib.cs_mx_ffn_shared(None, ctypes.byref(layer), P, P, P, 1, P, None) == 1


@pytest.mark.parametrize("kw", [dict(group=64), dict(d=320)])
def test_plan_shapes(kw):
    args = dict(d=256, d_ff=1024, group=128, m=8, k=4, T=10, w_dtype="mx4", max_tokens=4)
    args.update(kw)
    with pytest.raises(cs.CSError) as e:
        cs.Plan(**args)
    assert e.value.code == 3


def test_binding_refuses_cpu_and_foreign_types():
    with pytest.raises(TypeError):
        binding._matrix(torch.zeros(4, 32), binding._FLOATS, "w", 0)
    with pytest.raises(TypeError):
        binding._checked(torch.zeros(4), binding._BYTES, "q", (4,), 0)
    with pytest.raises(TypeError):
        binding._checked(torch.zeros(4, dtype=torch.uint8), binding._BYTES, "q", (4,), 0)
    assert binding._checked(None, binding._BYTES, "q", (4,), 0, True) is None
    with pytest.raises(TypeError):
        binding._dtype_code(torch.zeros(4, dtype=torch.float16), "x")


class _HostPlan:
    """What the binding itself looks at of a plan."""

    def __init__(self, d=256, k=2):
        self.d, self.k, self.device, self._templates = d, k, 0, {}

        def call(*args):
            raise AssertionError("a refused call reached the library")
        self.lib = type("lib", (), dict(cs_mx_ffn=call, cs_mx_ffn_shared=call, cs_mx_norm=call))
        self.handle = None


@pytest.mark.parametrize("shared", [False, True])
def test_a_refused_ffn_call_leaves_no_output_template(monkeypatch, shared):
    """The next call would allocate its output from it, on the refused tensor's device."""
    monkeypatch.setattr(binding, "_device_index", lambda: 0)
    plan, layer = _HostPlan(), type("layer", (), dict(ref=None))
    q = torch.zeros((8, 256), dtype=torch.float8_e4m3fn)
    s = torch.zeros((1, 2, 32, 4, 4), dtype=torch.float8_e8m0fnu)
    support = torch.zeros((2,) if shared else (8, 2), dtype=torch.int32)
    with pytest.raises((TypeError, ValueError)):
        (binding.cs_mx_ffn_shared if shared else binding.cs_mx_ffn)(plan, layer, q, s, support)
    assert plan._templates == {}


def test_refused_norm_and_matrix_calls_leave_no_output_template(monkeypatch):
    monkeypatch.setattr(binding, "_device_index", lambda: 0)
    plan, before = _HostPlan(), dict(binding._matrix_templates)
    x, codes = torch.zeros((8, 256)), torch.zeros((8, 128), dtype=torch.uint8)
    for call in (lambda: binding.cs_mx_norm(plan, x), lambda: binding.cs_mx_quantize(x),
                 lambda: binding.cs_mx_dequantize(codes, torch.zeros((8, 8), dtype=torch.uint8), 256)):
        with pytest.raises((TypeError, ValueError)):
            call()
    assert plan._templates == {} and binding._matrix_templates == before


def test_a_plan_of_another_device_is_refused(monkeypatch):
    """Its scratch is there, while stream and tensors would be here."""
    monkeypatch.setattr(binding, "_device_index", lambda: 1)
    monkeypatch.setattr(binding, "_checked", lambda *args: 1 << 20)      # tensors of the current device
    plan, layer = _HostPlan(), type("layer", (), dict(ref=None))
    plan.d_ff = 512
    q = torch.zeros((8, 256), dtype=torch.float8_e4m3fn)
    pair = (torch.zeros((512, 128), dtype=torch.uint8), torch.zeros((512, 8), dtype=torch.uint8))
    for call in (lambda: binding.cs_mx_norm(plan, torch.zeros((8, 256))), lambda: binding.cs_mx_ffn(plan, layer, q, None, None, stream=0),
                 lambda: binding.cs_mx_ffn_shared(plan, layer, q, None, None, stream=0), lambda: binding.MxLayer(plan, pair, pair, pair)):
        with pytest.raises(ValueError, match="plan is on"):
            call()
