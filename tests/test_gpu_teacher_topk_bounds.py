"""Top logits where a first part of the vocabulary gives each token a bound for the rest: calls of 112 to 256
tokens, whose first part goes by estimated time, and the largest K."""
import pytest
import torch

from tests.test_gpu_teacher_topk import _check, _head

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fr():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_36932_amd as m
    return m


@pytest.mark.parametrize("T", [111, 112, 128, 193, 256])
@pytest.mark.parametrize("V, d, k", [(36001, 24, 1), (60000, 16, 20), (36001, 200, 20)])
def test_one_column_of_tiles(fr, T, V, d, k):
    g = torch.Generator().manual_seed(T + V)
    H = torch.randn(T, d, generator=g).to(torch.bfloat16)
    w, ws = _head(V + k, V, d)
    _check(fr, H, w, ws, k, tau=(0.5, 1.0, 2.0)[T % 3])


@pytest.mark.parametrize("T", [130, 300])
def test_the_largest_k(fr, T):
    g = torch.Generator().manual_seed(T)
    H = torch.randn(T, 16, generator=g)
    w, ws = _head(T, 111001, 16)
    _check(fr, H, w, ws, 128)


@pytest.mark.parametrize("kind", ["rising", "falling", "equal", "last", "barred"])
def test_orders_of_the_vocabulary(fr, kind):
    T, V, d, k = 193, 36001, 16, 20
    g = torch.Generator().manual_seed(len(kind))
    H = torch.randn(T, d, generator=g)
    w, ws = _head(3, V, d)
    if kind in ("rising", "falling"):
        H, w = H.abs(), w.abs()
        ws = torch.linspace(0.01, 1.0, V)
        ws = ws if kind == "rising" else ws.flip(0)
    elif kind == "equal":
        w[:] = 0
        w[::7, 0] = 1
        ws[:] = 0.5
    elif kind == "last":
        ws[:V - 30] *= 1e-3
    else:
        H, w = 0.5 + H.abs(), w.abs() + 1 - w.abs() // 127
        ws[:V - 40] = float("-inf")
    H[5] = 0
    H[6, 3] = float("nan")
    _check(fr, H, w, ws, k)
