"""What the binding of the feed-forward block and the 8-bit operators hands to the library, with a library that only records its calls: no
GPU needed, and none of the bad arguments can reach one."""
import pytest
import torch

import paper_2501_14183_amd as vd

F32, BF16, I8, U8 = torch.float32, torch.bfloat16, torch.int8, torch.uint8


class OnGpu(torch.Tensor):
    """A tensor that says it is on device 0."""

    def get_device(self):
        return 0


def gpu(*shape, dtype=F32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu)


class Library:
    """Records the calls that get through with their arguments; sizes come from the real library."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        if name.endswith("_bytes"):
            return getattr(vd.load_library(), name)
        return lambda *args: self.calls.append((name, args)) or 0


class Ctx:
    def __init__(self):
        self._lib, self.handle, self.device = Library(), None, torch.device("cuda", 0)

    def check(self, rc, where):
        assert rc == 0


def weight(N, K):
    """Codes and scales as vardrop_quantize_weight makes them."""
    return gpu(N, vd.load_library().vardrop_i8_pitch(K), dtype=I8), gpu(N)


def product_of_codes(ctx, q, sx, rows, N=5, K=128):
    return vd.vardrop_linear_i8(ctx, (q, sx), *weight(N, K), out=gpu(rows, N, dtype=BF16), stream=0)


@pytest.mark.parametrize("shape,rows", [((6, 128), 6), ((2, 3, 128), 6), ((2, 1, 3, 128), 6), ((128,), 1), ((0, 128), 0)])
def test_codes_of_any_rank_have_a_scale_for_each_row(shape, rows):
    """The rows that the library is told are the rows whose scales were counted."""
    ctx, q = Ctx(), gpu(*shape, dtype=I8)
    for wrong in {rows - 1, rows + 1, shape[0], 128} - {rows, -1}:
        with pytest.raises(TypeError):
            product_of_codes(ctx, q, gpu(wrong), rows)
    assert ctx._lib.calls == []
    product_of_codes(ctx, q, gpu(rows), rows)
    (name, args), = ctx._lib.calls
    assert name == "vardrop_linear_i8" and args[3:5] == (rows, 128)


@pytest.mark.parametrize("K", [1, 96, 127, 129, 250])
def test_rows_of_codes_that_end_before_the_pitch_are_refused(K):
    """The kernels read whole pitches of 128 bytes, behind the end of a buffer of shorter rows."""
    ctx = Ctx()
    with pytest.raises(TypeError):
        product_of_codes(ctx, gpu(4, K, dtype=I8), gpu(4), 4, K=K)
    assert ctx._lib.calls == []


MORE = 2 ** 32 + 3            # 3 in 32 bits


def test_sizes_that_32_bits_cut_have_no_bytes():
    for call, sizes in ((vd.vardrop_pack8_bytes, (1, 2, 64)), (vd.vardrop_ffn_saved_bytes, (1, 2, 64, 64)),
                        (vd.vardrop_linear_i8_workspace_bytes, (2, 64, 64)),
                        (lambda *s: vd.vardrop_ffn_workspace_bytes(*s, BF16), (1, 2, 64, 64)),
                        (lambda *s: vd.vardrop_ffn_workspace_bytes(*s, F32), (1, 2, 64, 64))):
        assert call(*sizes) > 0
        for at in range(len(sizes)):
            for more in (MORE, 2 ** 32 + 64, 2 ** 31, 2 ** 63 + 64, -1):
                assert call(*sizes[:at], more, *sizes[at + 1:]) == 0


def far(*shape, dtype=BF16):
    """A tensor of that shape without memory."""
    return torch.empty(*shape, dtype=dtype, device="meta").as_subclass(OnGpu)


def far_calls():
    room, saved = gpu(1 << 12, dtype=U8), gpu(1 << 12, dtype=U8)
    block = dict(ws=room, stream=0)
    return {
        "pack8": lambda c: vd.vardrop_pack8(c, far(MORE, 1, 64), out=saved, stream=0),
        "pack8, tokens": lambda c: vd.vardrop_pack8(c, far(1, MORE, 64), out=saved, stream=0),
        "pack8, channels": lambda c: vd.vardrop_pack8(c, far(1, 1, MORE), out=saved, stream=0),
        "pack8, none": lambda c: vd.vardrop_pack8(c, far(MORE, 0, 64), out=saved, stream=0),
        "unpack8": lambda c: vd.vardrop_unpack8(c, saved, far(MORE, 1, 64), stream=0),
        "ffn_fwd": lambda c: vd.vardrop_ffn_fwd(c, far(MORE, 1, 64), far(64, 64), far(64, 64), train=False, out=far(MORE, 1, 64), **block),
        "ffn_fwd, tokens": lambda c: vd.vardrop_ffn_fwd(c, far(1, MORE, 64), far(64, 64), far(64, 64), saved=saved, out=far(1, MORE, 64), **block),
        "ffn_fwd, channels": lambda c: vd.vardrop_ffn_fwd(c, far(1, 1, 64), far(64, 2 ** 32 + 64), far(2 ** 32 + 64, 64), train=False,
                                                          out=far(1, 1, 64), **block),
        "ffn_bwd": lambda c: vd.vardrop_ffn_bwd(c, far(MORE, 1, 64), far(64, 64), far(64, 64), saved, out=(None, far(64, 64), far(64, 64), None, None),
                                                **block),
        "quantize_rows": lambda c: vd.vardrop_quantize_rows(c, far(MORE, 64), out=(far(MORE, 128, dtype=I8), far(MORE, dtype=F32)), stream=0),
        "quantize_rows, channels": lambda c: vd.vardrop_quantize_rows(c, far(1, MORE), out=(far(1, 128, dtype=I8), far(1, dtype=F32)), stream=0),
        "quantize_weight": lambda c: vd.vardrop_quantize_weight(c, far(64, MORE), out=(far(MORE, 128, dtype=I8), far(MORE, dtype=F32)), stream=0),
        "linear_i8": lambda c: vd.vardrop_linear_i8(c, far(MORE, 64), *weight(5, 64), ws=room, out=far(MORE, 5), stream=0),
        "linear_i8, channels": lambda c: vd.vardrop_linear_i8(c, far(1, MORE), *weight(5, 64), ws=room, out=far(1, 5), stream=0),
        "linear_i8, results": lambda c: vd.vardrop_linear_i8(c, far(1, 64), far(MORE, 128, dtype=I8), far(MORE, dtype=F32), ws=room, out=far(1, MORE),
                                                             stream=0),
        "linear_i8, codes": lambda c: vd.vardrop_linear_i8(c, (far(MORE, 128, dtype=I8), far(MORE, dtype=F32)), *weight(5, 128), out=far(MORE, 5),
                                                           stream=0),
    }


@pytest.mark.parametrize("name", list(far_calls()))
def test_calls_whose_sizes_32_bits_cut_are_refused(name):
    """The library takes 32-bit sizes: a larger one has to be refused before it becomes another."""
    ctx = Ctx()
    with pytest.raises(vd.VarDropError) as e:
        far_calls()[name](ctx)
    assert e.value.code == -4 and ctx._lib.calls == []


def test_more_rows_of_codes_than_the_products_take_are_refused():
    """2^30 rows, or channels, as vardrop_linear_i8 takes them; the address of a context is looked at before anything behind it."""
    lib, most = vd.load_library(), 1 << 30
    context = torch.zeros(64, dtype=U8).data_ptr()
    for rows in (most + 1, 2 ** 31 - 1):
        assert lib.vardrop_quantize_rows(context, None, rows, 8, vd.F32, None, None, None) == -4
        assert lib.vardrop_quantize_weight(context, None, 8, rows, vd.F32, None, None, None) == -4
        assert lib.vardrop_linear_i8_workspace_bytes(rows, 8, 8) == 0 and lib.vardrop_linear_i8_workspace_bytes(8, 8, rows) == 0
    assert lib.vardrop_quantize_rows(context, None, most, 8, vd.F32, None, None, None) == -1
    assert lib.vardrop_quantize_weight(context, None, 8, most, vd.F32, None, None, None) == -1
    assert lib.vardrop_linear_i8_workspace_bytes(most, 8, most) == most * 128 + most * 4


def test_weight_gradients_that_are_missing_are_a_type_error():
    ctx, W1, W2, saved, ws = Ctx(), gpu(64, 128), gpu(128, 64), gpu(1 << 14, dtype=U8), gpu(1 << 20, dtype=U8)
    for missing in ((1,), (2,), (1, 2)):
        out = [gpu(1, 4, 64), gpu(64, 128), gpu(128, 64), None, None]
        for k in missing:
            out[k] = None
        with pytest.raises(TypeError):
            vd.vardrop_ffn_bwd(ctx, gpu(1, 4, 64), W1, W2, saved, ws=ws, out=tuple(out), stream=0)
    assert ctx._lib.calls == []
