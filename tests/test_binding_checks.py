"""What the binding refuses before the library sees it, with a library that only counts its calls: no GPU needed, and none of
the bad arguments can reach one."""
import ctypes

import pytest
import torch

import paper_2501_14183_amd as vd
from paper_2501_14183_amd import binding

F32, BF16, I32, I64 = torch.float32, torch.bfloat16, torch.int32, torch.int64


class OnGpu(torch.Tensor):
    """A tensor that says it is on device 0."""

    def get_device(self):
        return 0


def gpu(*shape, dtype=F32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu)


class Library:
    """Counts the calls that get through; sizes come from the real library."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        if name.endswith("_bytes"):
            return getattr(vd.load_library(), name)
        return lambda *args: self.calls.append(name) or 0


class Ctx:
    def __init__(self):
        self._lib, self.handle, self.device = Library(), None, torch.device("cuda", 0)

    def check(self, rc, where):
        assert rc == 0


def a_list():
    """A TensorList that was not built."""
    tensors = object.__new__(vd.TensorList)
    tensors.device, tensors.table, tensors.struct = 0, gpu(256, dtype=torch.uint8), binding._TensorListStruct()
    tensors.pointer = ctypes.addressof(tensors.struct)
    return tensors


def test_a_clipping_norm_that_single_precision_takes_for_none_is_refused():
    """max_norm 0 means no clipping, so what rounds to 0 must not pass for it."""
    ctx, tensors = Ctx(), a_list()
    for max_norm in (1e-46, 1e-300):
        for call in (lambda: vd.vardrop_adamw(ctx, tensors, 0.1, 1, norm=gpu(1), max_norm=max_norm, stream=0),
                     lambda: vd.vardrop_adamw_dev(ctx, tensors, gpu(1), gpu(1, dtype=I64), norm=gpu(1), max_norm=max_norm, stream=0)):
            with pytest.raises(vd.VarDropError) as e:
                call()
            assert e.value.code == -1
    assert ctx._lib.calls == []
    for max_norm in (0.0, 1e-45, 1.0):
        vd.vardrop_adamw(ctx, tensors, 0.1, 1, norm=gpu(1), max_norm=max_norm, stream=0)
        vd.vardrop_adamw_dev(ctx, tensors, gpu(1), gpu(1, dtype=I64), norm=gpu(1), max_norm=max_norm, stream=0)
    assert ctx._lib.calls == ["vardrop_adamw", "vardrop_adamw_dev"] * 3


# what may stand in the place of a device scalar of the given type
def bad_scalars(dtype):
    other = {F32: torch.float64, I32: I64, I64: I32}[dtype]
    return [torch.zeros(1, dtype=dtype), gpu(1, dtype=other), gpu(1, dtype=BF16), gpu(0, dtype=dtype)]


def optimiser_calls():
    """The library that counts, and (call, its device scalars with their types)."""
    ctx, tensors = Ctx(), a_list()
    return ctx._lib, [
        (lambda **k: vd.vardrop_grad_norm(ctx, tensors, stream=0, **k), dict(out=F32)),
        (lambda **k: vd.vardrop_clip_grads(ctx, tensors, max_norm=1.0, stream=0, **k), dict(norm=F32, status=I32)),
        (lambda **k: vd.vardrop_adamw(ctx, tensors, 0.1, 1, max_norm=1.0, stream=0, **k), dict(norm=F32, status=I32)),
        (lambda **k: vd.vardrop_adamw_dev(ctx, tensors, max_norm=1.0, stream=0, **k),
         dict(lr_dev=F32, step_dev=I64, norm=F32, status=I32)),
    ]


def test_device_scalars_of_the_optimiser():
    library, calls = optimiser_calls()
    for call, scalars in calls:
        good = {name: gpu(1, dtype=dtype) for name, dtype in scalars.items()}
        for name, dtype in scalars.items():
            for bad in bad_scalars(dtype):
                with pytest.raises(TypeError):
                    call(**{**good, name: bad})
    assert library.calls == []
    for call, scalars in calls:
        call(**{name: gpu(3, dtype=dtype)[1:] for name, dtype in scalars.items()})
    assert library.calls == ["vardrop_grad_norm", "vardrop_clip_grads", "vardrop_adamw", "vardrop_adamw_dev"]
