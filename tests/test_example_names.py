"""examples/train_encoder.py: every weight of a deep encoder has a name of its own (built on the CPU, no call of the library is made)."""
import pytest
import torch

import examples.train_encoder as ex
import paper_2501_14183_amd as vd


class Lists:
    """Stands for the list of tensors that the optimiser takes."""

    def __init__(self, ctx, grads, **kw):
        self.grads = grads


@pytest.fixture
def on_the_cpu(monkeypatch):
    def here(make):
        return lambda *a, **kw: make(*a, **{**kw, **({"device": "cpu"} if "device" in kw else {})})

    monkeypatch.setattr(ex.vd, "TensorList", Lists)
    for name in ("randn", "zeros", "empty"):
        monkeypatch.setattr(torch, name, here(getattr(torch, name)))
    generator = torch.Generator
    monkeypatch.setattr(torch, "Generator", lambda device=None: generator())


class Ctx:
    _lib = vd.load_library()


@pytest.mark.parametrize("layers,ffn", [(2, 0), (2, 128), (6, 128), (6, 64), (12, 192), (30, 64), (120, 0)])
def test_every_weight_is_there_once(on_the_cpu, layers, ffn):
    d = 64
    enc = ex.Encoder(Ctx, 1, 24, 2, d, 1, layers, seed=1, ffn=ffn)
    blocks = layers * (2 if ffn else 1)
    # embedding, the norm before the first block; a post norm, a gate and a norm for each block; four matrices, or two and two biases
    assert len(enc.params) == 4 + 4 * blocks + 4 * layers * (2 if ffn else 1)
    assert len({t.data_ptr() for t in enc.params.values()}) == len(enc.params) == len(enc.grads) == len(enc.list.grads)
    for k, kind in enumerate(enc.blocks):
        if kind == "ffn":
            W1, W2, b1, b2 = enc.feed_forward(k)
            assert W1.shape == (d, ffn) and W2.shape == (ffn, d) and b1.shape == (ffn,) and b2.shape == (d,)
            mine = {t.data_ptr() for t in (W1, W2, b1, b2)}
        else:
            mine = {t.data_ptr() for t in enc.attention(k)}
        for other in range(len(enc.blocks) + 1):
            assert not mine & {v.data_ptr() for v in enc.around(other).values() if torch.is_tensor(v)}
            assert enc.norm_bias(other).data_ptr() not in mine and enc.norm_bias(other).shape == (d,)


def test_names_of_few_blocks_are_the_plain_ones(on_the_cpu):
    enc = ex.Encoder(Ctx, 1, 24, 2, 64, 1, 2, seed=1, ffn=64)
    assert {"We", "be", "w0", "b0", "b4", "W11", "b11", "W23", "b23", "Wo2", "gate3", "wp0"} <= set(enc.params)
