"""Argument checks of the calls behind the attention that need no device: tensors are stand-ins that answer what the checks ask."""
import pytest
import torch

from tests.test_decode_binding_cpu import FakeTensor, on  # noqa: F401  (the fixture)

BF, F32, I32, U8, I8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8, torch.int8


class Rows(FakeTensor):
    def dim(self):
        return len(self.shape)


def t(dtype, *shape, index=0):
    return Rows(index, dtype, *shape)


@pytest.fixture()
def calls(on, monkeypatch):  # noqa: F811
    binding, ctx, at = on
    monkeypatch.setattr(binding, "_empty", lambda shape, dtype, device: t(dtype, *((shape,) if type(shape) is int else shape), index=device.index))
    w, x = binding.Q8(t(I8, 2, 32, 64), t(F32, 2, 32), 60), binding.Q8(t(I8, 5, 64), t(F32, 5), 60)
    good = {
        "route": lambda **k: ctx.rk_moe_route(k.pop("logits", t(F32, 4, 16)), k.pop("k", 2), **k),
        "group": lambda **k: ctx.rk_moe_group(k.pop("ids", t(I32, 4, 2)), 16, **k),
        "quant": lambda **k: ctx.rk_quant8(k.pop("x", t(BF, 5, 60)), **k),
        "matmul": lambda **k: ctx.rk_matmul8(k.pop("w", w), k.pop("x", x), **k),
        "experts": lambda **k: ctx.rk_matmul8_experts(k.pop("w", w), x, k.pop("row_off", t(I32, 3)), k.pop("rows", t(I32, 10)), 2, **k),
        "sample": lambda **k: ctx.rk_sample(k.pop("logits", t(F32, 3, 10)), k.pop("u", t(F32, 3)), **k),
    }
    return binding, at, good, w, x


def test_well_formed_calls_reach_the_library(calls):
    binding, _, good, _, _ = calls
    for name, call in good.items():
        with pytest.raises(binding.RKError) as ei:
            call()
        assert ei.value.status == 1, name                           # the context has no handle


@pytest.mark.parametrize("name, change, error", [
    ("route", dict(logits=t(torch.float16, 4, 16)), TypeError),
    ("route", dict(logits=t(F32, 4, 16, 1)), ValueError),
    ("route", dict(score="relu"), ValueError),
    ("route", dict(bias=t(F32, 15)), ValueError),
    ("route", dict(bias=t(BF, 16)), TypeError),
    ("route", dict(ids=t(torch.int64, 4, 2)), TypeError),
    ("route", dict(weights=t(F32, 4, 3)), ValueError),
    ("group", dict(ids=t(torch.int64, 4, 2)), TypeError),
    ("group", dict(keep=t(U8, 5)), ValueError),
    ("group", dict(row_off=t(I32, 16)), ValueError),
    ("group", dict(rows=t(I32, 7)), ValueError),
    ("quant", dict(x=t(F32, 5, 60)), TypeError),
    ("quant", dict(x=t(F32, 2, 5, 60)), TypeError),
    ("quant", dict(x=t(BF, 60)), ValueError),
    ("matmul", dict(out_dtype=torch.float16), TypeError),
    ("matmul", dict(y=t(torch.float16, 5, 32)), TypeError),
    ("matmul", dict(y=t(BF, 4, 32)), ValueError),
    ("matmul", dict(y=t(BF, 5, 31)), ValueError),
    ("experts", dict(row_off=t(I32, 2)), ValueError),
    ("experts", dict(rows=t(torch.int64, 10)), TypeError),
    ("experts", dict(y=t(F32, 9, 32)), ValueError),
    ("sample", dict(logits=t(torch.float16, 3, 10)), TypeError),
    ("sample", dict(u=t(F32, 4)), ValueError),
    ("sample", dict(temperature=t(F32, 2)), ValueError),
    ("sample", dict(top_k=t(F32, 3)), TypeError),
    ("sample", dict(top_p=t(torch.float64, 3)), TypeError),
    ("sample", dict(tokens=t(torch.int64, 3)), TypeError),
    ("sample", dict(probs=t(F32, 3, index=1)), ValueError),
])
def test_wrong_tensors_are_refused(calls, name, change, error):
    with pytest.raises(error):
        calls[2][name](**change)


def test_rows_of_another_device_are_refused(calls):
    binding, at, good, w, x = calls
    at(1)
    for call in (good["matmul"], good["experts"]):
        with pytest.raises(ValueError, match="device"):
            call()
    with pytest.raises(ValueError, match="device"):
        good["quant"](x=t(BF, 5, 60, index=1), q8=x)


def test_q8_checks_what_it_keeps(on):  # noqa: F811
    binding = on[0]
    binding.Q8(t(I8, 4, 64), t(F32, 4), 49)
    for codes, scales, k, error in ((t(I8, 4, 60), t(F32, 4), 60, ValueError), (t(U8, 4, 64), t(F32, 4), 64, TypeError),
                                    (t(I8, 4, 64), t(F32, 5), 64, ValueError), (t(I8, 4, 64), t(BF, 4), 64, TypeError),
                                    (t(I8, 64), t(F32, 1), 64, ValueError), (t(I8, 2, 4, 64), t(F32, 8), 64, ValueError)):
        with pytest.raises(error):
            binding.Q8(codes, scales, k)


def test_a_quantised_result_shows_its_codes_and_scales(monkeypatch):
    """The one allocation behind a result: codes in front, scales behind them, each where the C ABI is told."""
    from paper_2609_07008_b200 import binding
    monkeypatch.setattr(binding, "_empty", lambda shape, dtype, device: torch.zeros(shape, dtype=dtype))
    for rows, k in (((3,), 17), ((2, 5), 64), ((0,), 8), ((1,), 1)):
        q = binding.Q8._new(rows, k, torch.device("cpu"))
        pad = (k + 15) // 16 * 16
        assert q.codes.shape == rows + (pad,) and q.codes.dtype == torch.int8 and q.codes.is_contiguous()
        assert q.scales.shape == rows and q.scales.dtype == torch.float32
        if q.n_rows:
            assert q.codes.data_ptr() == q.struct.codes and q.scales.data_ptr() == q.struct.scales
        assert (q.struct.n_mat, q.struct.n_rows, q.struct.k) == (rows[0] if len(rows) == 2 else 1, rows[-1], k)
