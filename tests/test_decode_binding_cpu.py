"""Argument checks of the binding's decode calls that need no device: tensors are stand-ins that answer what the checks ask."""
import ctypes as C
import os
import subprocess
import sys

import pytest
import torch

PAGE_BYTES = 26624


class FakeTensor:
    """A tensor on CUDA device `index` as far as the binding looks at one; its address is never dereferenced."""

    def __init__(self, index, dtype, *shape):
        self.index, self.dtype, self.shape, self.is_cuda = index, dtype, torch.Size(shape), True
        self.device = torch.device("cuda", index)

    def get_device(self):
        return self.index

    def is_contiguous(self):
        return True

    def numel(self):
        return self.shape.numel()

    def data_ptr(self):
        return 1 << 20


@pytest.fixture()
def on(monkeypatch):
    """The binding, a context without a handle (the library answers RK_ERR_NULL to it), and a switch of the current device."""
    from paper_2609_07008_b200 import binding
    ctx = object.__new__(binding.Context)
    ctx.handle, ctx.n_heads = C.c_void_p(), 16
    now = [0]
    monkeypatch.setattr(binding, "_current_device", lambda: now[0])
    monkeypatch.setattr(binding, "_quick_stream", lambda: 0)
    monkeypatch.setattr(binding, "_empty", lambda shape, dtype, device: FakeTensor(device.index, dtype, *(
        (shape,) if type(shape) is int else shape)))

    def at(index):
        now[0] = index

    return binding, ctx, at


def kept(binding, index):
    """A table, a plan and weights whose tensors are on device `index` (the current one)."""
    i32, u8 = torch.int32, torch.uint8
    table = binding.CacheTable(FakeTensor(index, i32, 2), FakeTensor(index, i32, 3), FakeTensor(index, i32, 4))
    plan = binding.DecodePlan(binding.rk_decode_shape(1, 1, 1, 1), 4, FakeTensor(index, u8, 4096))
    w4 = binding.W4(1, 16, 64, 32, FakeTensor(index, u8, 512), FakeTensor(index, torch.bfloat16, 32))
    return table, plan, w4


def calls(ctx, index, table, plan, w4):
    """Every decode call with its own tensors on device `index`."""
    bf, i32 = torch.bfloat16, torch.int32
    pages = FakeTensor(index, torch.uint8, 4, PAGE_BYTES)
    t = lambda dtype, *shape: FakeTensor(index, dtype, *shape)
    items = (t(i32, 2), t(i32, 1), t(i32, 1), t(i32, 1, 1))
    return {
        "append": lambda: ctx.rk_cache4_append(pages, table, t(bf, 3, 512), t(bf, 3, 64), t(i32, 3)),
        "read": lambda: ctx.rk_cache4_read(pages, table, t(i32, 3), 3, kv=t(bf, 3, 576)),
        "plan": lambda: ctx.rk_decode_plan(table, 4, *items, max_tiles=1),
        "attn": lambda: ctx.rk_cache4_attn(pages, plan, t(bf, 1, 1, 16, 576)),
        "quant4": lambda: ctx.rk_quant4(t(bf, 1, 16, 64), 32, w4),
        "matvec4": lambda: ctx.rk_matvec4(w4, t(bf, 1, 1, 64)),
    }


@pytest.mark.parametrize("name", ["append", "read", "plan", "attn", "quant4", "matvec4"])
def test_kept_tables_plans_and_weights_of_another_device_are_refused(on, name):
    binding, ctx, at = on
    mine = kept(binding, 0)
    with pytest.raises(binding.RKError) as ei:                    # all on one device: the call reaches the library
        calls(ctx, 0, *mine)[name]()
    assert ei.value.status == 1
    at(1)
    with pytest.raises(ValueError, match="device"):               # the kept object's memory is on device 0
        calls(ctx, 1, *mine)[name]()


def test_plan_buffer_of_another_device_is_not_filled_anew(on):
    binding, ctx, at = on
    plan = kept(binding, 0)[1]
    at(1)
    table = kept(binding, 1)[0]
    i32 = torch.int32
    with pytest.raises(ValueError, match="device"):
        ctx.rk_decode_plan(table, 4, FakeTensor(1, i32, 2), FakeTensor(1, i32, 1), FakeTensor(1, i32, 1), FakeTensor(1, i32, 1, 1),
                           max_tiles=1, plan=plan)


def test_plan_buffer_has_to_be_bytes_in_a_row(on):
    binding, _, _ = on
    shape = binding.rk_decode_shape(1, 1, 1, 1)
    with pytest.raises(TypeError):
        binding.DecodePlan(shape, 4, FakeTensor(0, torch.int32, 1024))
    with pytest.raises(ValueError):
        binding.DecodePlan(shape, 4, FakeTensor(0, torch.uint8, 4, 1024))


def test_import_needs_no_private_function_of_torch():
    """A torch without the two private look-ups (one built without CUDA has neither): the binding imports, and the public
    functions take their place."""
    code = """
import torch
for name in ("_cuda_getDevice", "_cuda_getCurrentRawStream"):
    if hasattr(torch._C, name):
        delattr(torch._C, name)
class Stream:
    cuda_stream = 77
torch.cuda.current_device = lambda: 3
torch.cuda.current_stream = lambda device=None: Stream() if device == 3 else None
from paper_2609_07008_b200 import binding
assert binding._current_device() == 3 and binding._quick_stream() == 77
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr


@pytest.mark.parametrize("dtype", [torch.float16, torch.float64, torch.int32])
def test_products_refuse_output_types_they_do_not_have(on, dtype):
    binding, ctx, _ = on
    w4 = kept(binding, 0)[2]
    x = FakeTensor(0, torch.bfloat16, 1, 1, 64)
    with pytest.raises(TypeError, match="bfloat16 or float32"):
        ctx.rk_matvec4(w4, x, out_dtype=dtype)
    with pytest.raises(TypeError, match="bfloat16 or float32"):
        ctx.rk_matvec4(w4, x, y=FakeTensor(0, dtype, 1, 1, 16))
