"""linear_i8 on rows that are gathered, strided and unaligned, into strided rows, in one launch (up to 16 tokens)
and in two: the oracle's bits, and nothing between the output's rows."""
import numpy as np
import pytest
import torch

from tests.test_gpu_int8 import DEV, _expected, _rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fr():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_36932_amd as m
    return m


@pytest.mark.parametrize("T", [1, 3, 4, 5, 9, 16, 17, 300])
@pytest.mark.parametrize("K, N", [(7, 40), (100, 33), (1001, 300), (2056, 70)])
@pytest.mark.parametrize("dtype, out", [(torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32),
                                        (torch.float32, torch.bfloat16)])
def test_gathered_strided_unaligned(fr, T, K, N, dtype, out):
    g = torch.Generator().manual_seed(T + K)
    base = _rows(T * K + N, 37, K + 6, dtype)
    rows = torch.randint(0, 37, (T,), generator=g, dtype=torch.int32)
    rows[-1] = 36
    Kp = (K + 15) // 16 * 16
    wq, ws = fr.quantize_rows(_rows(T + K + N, N, K, torch.float32, 0.02).to(DEV))
    wide = torch.full((N, Kp + 32), 5, dtype=torch.int8, device=DEV)
    wide[:, 16:16 + Kp] = wq
    x = base.to(DEV)
    for lo in (0, 1, 3):
        exp = _expected(base[rows.long(), lo:lo + K], wq.cpu().numpy()[:, :K], ws.cpu().numpy(), out)
        for off, pad in ((0, 5), (3, 6)):
            buf = torch.full((T, N + pad), 7.0, dtype=out, device=DEV)
            fr.linear_i8(x[:, lo:lo + K], wide[:, 16:16 + Kp], ws, row_index=rows.to(DEV), out=buf[:, off:off + N])
            assert np.array_equal(buf[:, off:off + N].float().cpu().numpy(), exp)
            assert (buf[:, :off] == 7).all() and (buf[:, off + N:] == 7).all()
    if T <= 37:  # without an index
        exp = _expected(base[:T, 2:2 + K], wq.cpu().numpy()[:, :K], ws.cpu().numpy(), out)
        assert np.array_equal(fr.linear_i8(x[:T, 2:2 + K], wq, ws, out_dtype=out).float().cpu().numpy(), exp)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T", [1, 2, 4, 5, 12, 16])
@pytest.mark.parametrize("K", [40, 600, 2100, 3200])
def test_few_rows_that_are_not_finite(fr, T, K, dtype):
    """A row that is not finite gives NaN, the others what they give alone."""
    g = torch.Generator().manual_seed(T * K)
    x = torch.randn(T, K, generator=g).to(dtype)
    for t, v in ((0, "nan"), (1, "inf"), (3, "-inf"), (11, "nan")):
        if t < T:
            x[t, (K - 1, 0, K // 2)[t % 3]] = float(v)
    wq, ws = fr.quantize_rows(torch.randn(20, K, generator=g).to(DEV))
    z = fr.linear_i8(x.to(DEV), wq, ws, out_dtype=torch.float32).cpu().numpy()
    bad = ~torch.isfinite(x.float()).all(1).numpy()
    exp = _expected(x, wq.cpu().numpy()[:, :K], ws.cpu().numpy(), torch.float32)
    assert np.isnan(z[bad]).all() and np.array_equal(z[~bad], exp[~bad])
