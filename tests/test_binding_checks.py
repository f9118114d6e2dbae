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


def norm_arguments(B=2, n=3, d=8):
    """Everything the two calls take, on the GPU: (forward, backward), results and gradients under their own names."""
    tokens = lambda: gpu(B, n, d)
    forward = dict(x=tokens(), f=tokens(), w=gpu(d), b=gpu(d), wp=gpu(d), bp=gpu(d), gate=gpu(B, d), r=tokens(), h=tokens(),
                   stats=gpu(B * n, 4), n_dev=gpu(1, dtype=I32), status=gpu(1, dtype=I32))
    backward = dict(dr=tokens(), dh=tokens(), r=tokens(), f=tokens(), stats=gpu(B * n, 4), w=gpu(d), wp=gpu(d), bp=gpu(d), gate=gpu(B, d),
                    ws=gpu(vd.vardrop_block_norm_workspace_bytes(B, n, d, B), dtype=torch.uint8), n_dev=gpu(1, dtype=I32),
                    status=gpu(1, dtype=I32), dx=tokens(), df=tokens(), dw=gpu(d), db=gpu(d), dwp=gpu(d), dbp=gpu(d), dgate=gpu(B, d))
    return forward, backward


def call_norm(ctx, arguments):
    a = dict(arguments)
    kinds = dict(pre=vd.NORM_LAYER, post=vd.NORM_RMS, stream=0)
    if "x" in a:
        out = tuple(a.pop(k) for k in ("r", "h", "stats"))
        return vd.vardrop_block_norm_fwd(ctx, out=out, **a, **kinds)
    out = tuple(a.pop(k) for k in ("dx", "df", "dw", "db", "dwp", "dbp", "dgate"))
    return vd.vardrop_block_norm_bwd(ctx, out=out, **a, **kinds)


@pytest.mark.parametrize("which,name", [(i, k) for i, a in enumerate(norm_arguments()) for k in a])
def test_every_tensor_of_the_block_norms_has_to_be_on_the_device(which, name):
    ctx, arguments = Ctx(), norm_arguments()[which]
    call_norm(ctx, arguments)
    assert len(ctx._lib.calls) == 1
    with pytest.raises(TypeError):
        call_norm(ctx, {**arguments, name: torch.zeros_like(arguments[name].as_subclass(torch.Tensor))})
    assert len(ctx._lib.calls) == 1


@pytest.mark.parametrize("which,name", [(i, k) for i in (0, 1) for k in ("n_dev", "status")])
def test_device_scalars_of_the_block_norms(which, name):
    ctx, arguments = Ctx(), norm_arguments()[which]
    for bad in bad_scalars(I32):
        with pytest.raises(TypeError):
            call_norm(ctx, {**arguments, name: bad})
    assert ctx._lib.calls == []


def test_a_workspace_that_is_smaller_than_it_says_is_refused():
    """An expanded view counts its elements, not the memory behind them."""
    ctx, arguments = Ctx(), norm_arguments()[1]
    size = arguments["ws"].numel()
    for bad in (gpu(1, dtype=torch.uint8).expand(size), gpu(2 * size, dtype=torch.uint8)[::2]):
        with pytest.raises(TypeError):
            call_norm(ctx, {**arguments, "ws": bad})
    assert ctx._lib.calls == []


def test_a_backward_without_dr_and_r_is_refused():
    ctx, arguments = Ctx(), norm_arguments()[1]
    with pytest.raises(TypeError):
        call_norm(ctx, {**arguments, "dr": None, "r": None})
    assert ctx._lib.calls == []


def counted_calls():
    """The library that counts, and every older call that reads a count or a counter on the device with its scalars' types."""
    ctx = Ctx()
    B, N, n, d, L, H = 2, 6, 4, 8, 12, 2
    tok, few, x, index = gpu(B, N, d), gpu(B, n, d), gpu(B, N, L), gpu(N, dtype=I32)
    We, room, W, dW = gpu(L, d), gpu(4096, dtype=torch.uint8), [gpu(d, d)] * 4, [gpu(d, d) for _ in range(4)]
    counts = dict(n_dev=I32, status=I32)
    return ctx._lib, [
        (lambda step_dev: vd.vardrop_sample_dev(ctx, gpu(N, dtype=I64), 4, 1, 10, 1, step_dev, True, (index, index, gpu(2, dtype=I32)), stream=0),
         dict(step_dev=I64)),
        (lambda n_dev, status: vd.vardrop_gather_dev(ctx, tok, index, n_dev, n, few, status=status, stream=0), counts),
        (lambda n_dev, status: vd.vardrop_scatter_dev(ctx, few, index, n_dev, n, tok, status=status, stream=0), counts),
        (lambda n_dev, status: vd.vardrop_gather_attn_fwd_dev(ctx, tok, index, n_dev, n, *W, H, few, few, room, status=status, stream=0), counts),
        (lambda n_dev, status: vd.vardrop_attn_fwd_dev(ctx, few, n_dev, n, *W, H, few, room, status=status, stream=0), counts),
        (lambda n_dev, status: vd.vardrop_attn_bwd_dev(ctx, few, few, n_dev, n, *W, H, room, room, (few, *dW), status=status, stream=0), counts),
        (lambda n_dev, status: vd.vardrop_embed_fwd_dev(ctx, x, index, n_dev, n, We, gpu(d), few, room, status=status, stream=0), counts),
        (lambda n_dev: vd.vardrop_embed_bwd_dev(ctx, few, n_dev, n, L, room, room, (We, gpu(d)), stream=0), dict(n_dev=I32)),
    ]


def test_device_scalars_of_the_older_calls():
    library, calls = counted_calls()
    for call, scalars in calls:
        good = {name: gpu(1, dtype=dtype) for name, dtype in scalars.items()}
        for name, dtype in scalars.items():
            for bad in bad_scalars(dtype):
                with pytest.raises(TypeError):
                    call(**{**good, name: bad})
    assert library.calls == []
    for call, scalars in calls:
        call(**{name: gpu(3, dtype=dtype)[1:] for name, dtype in scalars.items()})
        if "status" in scalars:
            call(n_dev=gpu(1, dtype=I32), status=None)
    assert len(library.calls) == 2 * len(calls) - 2
