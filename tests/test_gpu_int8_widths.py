"""Operands whose widths do not belong together are refused, the wide side as the narrow one."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def fr():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_36932_amd as m
    return m


def _codes(fr, rows, cols):
    return fr.quantize_rows(torch.randn(rows, cols, device=DEV))


@pytest.mark.parametrize("T", [1, 9, 40])
@pytest.mark.parametrize("K, width", [(20, 48), (16, 17), (48, 112), (33, 64), (20, 16), (33, 32)])
def test_a_weight_of_another_width(fr, T, K, width):
    w, ws = _codes(fr, 40, width)
    x = torch.randn(T, K, device=DEV)
    for call in (lambda: fr.linear_i8(x, w, ws), lambda: fr.teacher_topk(x, w, ws, 2)):
        with pytest.raises(fr.FastRLError, match="codes"):
            call()


@pytest.mark.parametrize("a, b", [(32, 64), (64, 32), (16, 17)])
def test_codes_of_two_widths(fr, a, b):
    (x, xs), (w, ws) = _codes(fr, 5, a), _codes(fr, 40, b)
    with pytest.raises(fr.FastRLError, match="codes"):
        fr.matmul_i8(x, xs, w, ws)
    with pytest.raises(fr.FastRLError, match="codes"):
        fr.matmul_i8(x, xs, w, ws, K=max(a, b))


def test_widths_that_belong_together(fr):
    """Rows padded to 16 codes, more of them as a view, and a stated number of columns."""
    x = torch.randn(6, 20, device=DEV)
    w, ws = _codes(fr, 40, 20)
    ref = fr.linear_i8(x, w, ws)
    wide = torch.full((40, 96), 3, dtype=torch.int8, device=DEV)
    wide[:, 32:64] = w
    assert torch.equal(fr.linear_i8(x, wide[:, 32:64], ws), ref)
    q, s = fr.quantize_rows(x)
    assert torch.equal(fr.matmul_i8(q, s, w, ws), ref)
    assert torch.equal(fr.matmul_i8(q, s, wide[:, 32:], ws, K=20), ref)


@pytest.mark.parametrize("T", [3, 40, 300])
def test_codes_past_the_stated_columns(fr, T):
    """Those up to the next multiple of 16 count unless they are 0 in one operand; later ones never do."""
    g = torch.Generator().manual_seed(T)
    x, w = (torch.randint(-128, 128, (n, 64), generator=g, dtype=torch.int32).to(torch.int8) for n in (T, 70))
    one = torch.ones(300, device=DEV)
    def product(x, w):
        return fr.matmul_i8(x.to(DEV), one[:T], w.to(DEV), one[:70], K=20, out_dtype=torch.float32).cpu()
    exp = lambda n: (x[:, :n].double() @ w[:, :n].double().t()).float()
    assert torch.equal(product(x, w), exp(32))
    for a, b in ((x.clone(), w), (x, w.clone())):
        (a if b is w else b)[:, 20:32] = 0
        assert torch.equal(product(a, b), exp(20))
