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
