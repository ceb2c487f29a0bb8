"""The distillation's kernels that calls of more tokens take, against the oracle with the bounds of
test_gpu_distill: dhidden from a transposed W, logits tiles cut into pieces, the narrow last column after all
others, the larger float32 tiles."""
import pytest
import torch

from tests.test_gpu_distill import DEV, Case, _compare

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def fr():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_36932_amd as m
    return m


# (tokens modulo 256: 56, 128, 192 one, two, three narrow columns; 255 and 0 none, and so cut tiles)
@pytest.mark.parametrize("T, d, V, k", [(6200, 8, 600, 9), (6272, 64, 600, 33), (6336, 16, 300, 128), (6399, 24, 600, 5),
                                        (6200, 264, 300, 16)])
def test_many_tokens(fr, T, d, V, k):
    c = Case(T + d, T, d, V, k, BF16, gathered=T % 2 == 0, tau=(1.0, 2.0)[d % 3 == 0])
    _compare(c, c.call(fr), c.ref())


def test_many_tokens_each_output(fr):
    c = Case(41, 6200, 16, 500, 12, BF16, weighted=True, tail=True)
    ref = c.ref()
    for k in (dict(dW_dtype=F32), dict(need_dhidden=False), dict(need_dW=False), dict(slab_tokens=3000),
              dict(slab_tokens=3000, dW_dtype=F32, dhidden_dtype=F32), dict(need_dW=False, need_dhidden=False)):
        _compare(c, c.call(fr, **k), ref)
    dW = 1e-3 * torch.randn(500, 16)
    _compare(c, c.call(fr, dW=dW.to(DEV), dW_accumulate=True), ref, dW0=dW.double().numpy())


def test_dhidden_alone_from_a_transposed_weight(fr):
    c = Case(42, 20500, 8, 300, 6, BF16)
    _compare(c, c.call(fr, need_dW=False), c.ref())


# one or two columns of four blocks: 4 and 8 tiles cut into four pieces; 80 and 120 into two; 460 = 256 + 204
@pytest.mark.parametrize("T, d, V, k", [(256, 64, 770, 40), (512, 40, 770, 7), (460, 64, 1000, 20), (512, 16, 10200, 64),
                                        (768, 16, 10200, 20), (250, 32, 20000, 128), (3300, 16, 600, 8), (4000, 16, 600, 8)])
def test_cut_tiles_and_late_columns(fr, T, d, V, k):
    c = Case(T + d + 1, T, d, V, k, BF16, dup=True, tau=0.5)
    _compare(c, c.call(fr), c.ref())
    _compare(c, c.call(fr, need_dW=False, need_dhidden=False), c.ref())


@pytest.mark.parametrize("T, d, V, k", [(4200, 2048, 300, 5), (40, 2048, 4200, 30), (129, 64, 8193, 17), (600, 64, 3000, 9)])
def test_float32_tiles(fr, T, d, V, k):
    c = Case(T + d + 2, T, d, V, k, F32, h_std=0.5)
    _compare(c, c.call(fr), c.ref())
