"""Host side of the block norms and tensor lists: sizes and refusals that need no GPU (ctx NULL is refused first everywhere)."""
import ctypes

import pytest

import paper_2501_14183_amd as vd
from paper_2501_14183_amd import binding


@pytest.fixture(scope="module")
def lib():
    return vd.load_library()


def test_workspace_of_the_block_norm_backward(lib):
    size = lib.vardrop_block_norm_workspace_bytes
    # four fp32 sums of d columns for every range of rows: eight rows at least, 512 ranges in all, 256 for wide rows
    assert size(1, 8, 512, 0) == 4 * 512 * 4
    assert size(1, 16, 512, 1) == 2 * 4 * 512 * 4
    assert size(8, 8192, 768, 8) == 512 * 4 * 768 * 4
    assert size(8, 8192, 2048, 8) == 256 * 4 * 2048 * 4
    assert size(32, 1, 512, 32) == 32 * 4 * 512 * 4                      # a range for every gate row
    assert size(4, 0, 64, 0) == 4 * 64 * 4 and size(0, 4, 64, 0) == 4 * 64 * 4
    for bad in ((-1, 4, 64, 0), (4, -1, 64, 0), (4, 4, 0, 0), (4, 4, 8193, 0), (4, 4, 64, -1), (4, 4, 64, 3), (70000, 1, 64, 70000)):
        assert size(*bad) == 0
    assert vd.vardrop_block_norm_workspace_bytes(4, 4, 8193, 0) == 256


def test_workspace_grows_with_the_tokens(lib):
    """A workspace for a bound serves every smaller count (the _dev forms rely on the bound alone)."""
    for d in (16, 64, 512, 1500, 4096):
        for gates in (0, 4):
            sizes = [lib.vardrop_block_norm_workspace_bytes(4, n, d, gates) for n in range(0, 3000, 37)]
            assert sizes == sorted(sizes)


def test_size_of_a_list(lib):
    def size(*numel):
        return lib.vardrop_tensor_list_bytes(len(numel), (ctypes.c_int64 * max(1, len(numel)))(*numel))

    empty = size()
    assert empty > 0 and empty % 256 == 0 and size(0, 0) == empty
    assert size(1, 4096) == empty + 256                                  # two chunks of 64 bytes, rounded up
    assert size(4097) == empty + 256 and size(*[4096 * 4] * 5) == empty + 5 * 256
    assert size(-1) == 0 and size(1 << 41) == 0 and lib.vardrop_tensor_list_bytes(-1, None) == 0 and lib.vardrop_tensor_list_bytes(2, None) == 0


def test_no_context_is_refused(lib):
    n = None
    assert lib.vardrop_block_norm_fwd(n, n, n, 1, 1, 8, 0, 0, 0, n, n, n, 0, 1.0, 1.0, 1, n, n, 1e-5, n, n, n, n) == -1
    assert lib.vardrop_block_norm_bwd(n, n, n, n, n, n, 1, 1, 8, 0, 0, 0, n, n, n, 0, 1.0, 1.0, 1, n, n, n, n, n, n, n, n, n, 0, n) == -1
    assert lib.vardrop_tensor_list_build(n, 0, n, n, n, n, n, n, n, n, n, n, n, 0, n, n) == -1
    struct = binding._TensorListStruct()
    at = ctypes.addressof(struct)
    assert lib.vardrop_grad_norm(n, at, n, n) == -1
    assert lib.vardrop_clip_grads(n, at, n, 1.0, n, n) == -1
    assert lib.vardrop_adamw(n, at, 0.1, 0.9, 0.999, 1e-8, 1, n, 0.0, n, n) == -1
    assert lib.vardrop_adamw_dev(n, at, n, 0.9, 0.999, 1e-8, n, 1, n, 0.0, n, n) == -1


def test_kernel_ids_have_names(lib):
    names = [vd.vardrop_kernel_name(k) for k in range(64)]
    for name in ("block_norm_fwd", "block_norm_bwd", "block_norm_vectors", "grad_norm", "clip", "adamw"):
        assert names.count(name) == 1


def test_tensors_that_are_not_on_the_gpu_are_refused(lib):
    import torch

    class Ctx:
        _lib, handle = lib, None

    x = torch.zeros(2, 3, 8)
    with pytest.raises(TypeError):
        vd.vardrop_block_norm_fwd(Ctx, x, x)
    with pytest.raises(TypeError):
        vd.vardrop_block_norm_bwd(Ctx, x, x, x, x, torch.zeros(6, 4))
