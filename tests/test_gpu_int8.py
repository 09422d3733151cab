"""Rows in 8 bits (ap_quantize_rows) and scores against them (ap_scores_int8): the 8-bit values equal the formula's in IEEE f32, the scores
are the integer sums times two scales, off by at most the sum's and the products' three roundings (2^-24 each)."""
import numpy as np
import pytest
import torch

from paper_2511_00855_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


def rounded(x):
    """(8-bit values with zeros up to a multiple of 16 columns, scales) by numpy, whose f32 division is the IEEE one."""
    x = x.float().cpu().numpy()
    scale = np.abs(x).max(1) / np.float32(127)
    q = np.zeros((len(x), -(-x.shape[1] // 16) * 16), np.int8)
    with np.errstate(invalid="ignore", divide="ignore"):
        q[:, :x.shape[1]] = np.where(scale[:, None] > 0, np.rint(x / scale[:, None]), 0).astype(np.int8)
    return q, scale


def matrix(rng, rows, dim, dtype, stride=0):
    m = torch.full((rows, dim + stride), float("nan"), dtype=dtype, device=DEV)
    m[:, :dim] = torch.from_numpy((rng.standard_normal((rows, dim)) * np.exp(rng.uniform(-3, 3, (rows, 1)))).astype(np.float32)).to(DEV, dtype)
    return m[:, :dim]


def expected(qx, sx, q, s):
    return (qx.astype(np.int64) @ q.astype(np.int64).T).astype(np.float64) * sx.astype(np.float64)[:, None] * s.astype(np.float64)


@pytest.mark.parametrize("dtype,rows,dim,stride", [(F32, 1, 4, 0), (F32, 77, 260, 4), (BF16, 130, 264, 8), (F32, 9, 8192, 0), (BF16, 33, 1000, 0), (F32, 70_000, 20, 0)])
def test_rows(dtype, rows, dim, stride):
    rng = np.random.default_rng(dim)
    x = matrix(rng, rows, dim, dtype, stride)
    if rows > 5:
        x[1], x[3] = 0.0, 1.0
        x[4] = torch.arange(dim, device=DEV).to(dtype) - dim // 2   # many ties
    q, s = B.quantize_rows(x)
    want, scale = rounded(x)
    assert q.shape == want.shape and np.array_equal(q.cpu().numpy(), want) and np.array_equal(s.cpu().numpy(), scale)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_that_are_no_numbers(dtype):
    """Infinity or NaN: the scale is NaN, and so is every score of the row; the others are what they were."""
    rng = np.random.default_rng(1)
    x = matrix(rng, 5, 48, dtype)
    clean = B.quantize_rows(x)
    docs = B.quantize_rows(matrix(rng, 40, 48, F32))
    want = B.scores_int8(x, *docs)
    x[1, 7], x[3, 40] = float("inf"), float("nan")
    q, s = B.quantize_rows(x)
    assert torch.isnan(s[[1, 3]]).all() and (q[[1, 3]] == 0).all() and torch.equal(q[[0, 2, 4]], clean[0][[0, 2, 4]])
    got = B.scores_int8(x, *docs)
    assert torch.isnan(got[[1, 3]]).all() and torch.equal(got[[0, 2, 4]], want[[0, 2, 4]])


def test_tiny_rows():
    """Scales among the denormals: values stay within 127."""
    x = torch.tensor([[1e-44, -1e-44, 3e-45, 0.0], [1.2e-38, -6e-39, 1e-45, 0.0]], device=DEV)
    q, s = B.quantize_rows(x)
    assert int(q.abs().max()) <= 127 and torch.isfinite(s).all()


@pytest.mark.parametrize("dtype,rows,n,dim,stride", [
    (F32, 1, 1, 4, 0), (BF16, 1, 1000, 1024, 0), (F32, 7, 333, 260, 4), (BF16, 16, 17, 40, 0), (F32, 17, 5001, 100, 0), (BF16, 33, 700, 520, 8), (F32, 64, 1201, 768, 0),
    (F32, 65, 999, 36, 0), (BF16, 130, 3001, 264, 0), (F32, 40, 300, 4096, 0), (BF16, 700, 1030, 1000, 0)])
def test_scores(dtype, rows, n, dim, stride):
    rng = np.random.default_rng(rows + n)
    x, docs = matrix(rng, rows, dim, dtype, stride), matrix(rng, n, dim, F32)
    q, s = B.quantize_rows(docs)
    got = B.scores_int8(x, q, s)
    qx, sx = rounded(x)
    want = expected(qx, sx, *rounded(docs))
    assert got.shape == (rows, n) and got.dtype is F32
    assert (np.abs(got.cpu().numpy() - want) <= 3.01 * 2.0 ** -24 * np.abs(want) + 1e-44).all()
    # 8-bit queries with their scales: the same bits
    again = B.scores_int8(torch.from_numpy(qx).to(DEV), q, s, torch.from_numpy(sx).to(DEV))
    assert torch.equal(got, again)


def test_tiles_of_256():
    rng = np.random.default_rng(2)
    x, docs = matrix(rng, 3_001, 48, BF16), matrix(rng, 5_003, 48, F32)
    got = B.scores_int8(x, *B.quantize_rows(docs)).cpu().numpy()
    want = expected(*rounded(x), *rounded(docs))
    assert (np.abs(got - want) <= 3.01 * 2.0 ** -24 * np.abs(want) + 1e-44).all()


@pytest.mark.parametrize("rows", [5, 300])
def test_largest_sums_are_exact(rows):
    """All values 127 or -127 in 8,192 columns: sums beyond 24 bits, exact until the one rounding to f32."""
    q = torch.full((40, 8192), 127, dtype=torch.int8, device=DEV)
    q[1::2] = -127
    x = torch.full((rows, 8192), -127, dtype=torch.int8, device=DEV)
    one = torch.ones(300, device=DEV)
    got = B.scores_int8(x, q, one[:40], one[:rows])
    assert (got[:, 0] == float(np.float32(-8192 * 127 * 127))).all() and (got[:, 1] == float(np.float32(8192 * 127 * 127))).all()


def test_documents_apart_and_outputs_past_32_bits():
    """Rows of documents that lie further apart than they are long, and scores of more than 2^32 bytes."""
    rng = np.random.default_rng(4)
    wide = torch.full((700, 96), -128, dtype=torch.int8, device=DEV)
    docs = matrix(rng, 700, 64, F32)
    q, s = B.quantize_rows(docs)
    wide[:, :64] = q
    x = matrix(rng, 20, 64, F32)
    assert torch.equal(B.scores_int8(x, wide[:, :64], s), B.scores_int8(x, q, s))
    n, rows = 1_200_000, 1_000
    one = torch.ones(n, device=DEV)
    many = torch.zeros((n, 16), dtype=torch.int8, device=DEV)
    many[:, 0] = 1
    many[n - 1, 1] = 5
    y = torch.zeros((rows, 16), dtype=torch.int8, device=DEV)
    y[:, 0] = 3
    y[rows - 1, 1] = 2
    got = B.scores_int8(y, many, one, one[:rows])
    assert got[rows - 1, n - 1] == 13 and got[0, 0] == 3 and got[rows - 1, 0] == 3 and got[0, n - 1] == 3


def test_no_queries():
    q, s = B.quantize_rows(torch.ones((3, 16), device=DEV))
    assert B.scores_int8(torch.ones((0, 16), device=DEV), q, s).shape == (0, 3)
    assert B.quantize_rows(torch.ones((0, 16), device=DEV))[0].shape == (0, 16)


def test_refusals():
    x = torch.ones((3, 16), device=DEV)
    q, s = B.quantize_rows(x)
    with pytest.raises(ValueError, match="columns"):
        B.scores_int8(torch.ones((3, 20), device=DEV), q, s)
    with pytest.raises(ValueError, match="x_scale"):
        B.scores_int8(q, q, s)
    with pytest.raises(ValueError, match="q_scale"):
        B.scores_int8(x, q, s[:2])
    with pytest.raises(ValueError, match="int8"):
        B.scores_int8(x, x, s)
    with pytest.raises(B.ApError, match="multiple of 4"):
        B.quantize_rows(torch.ones((3, 6), device=DEV))
    with pytest.raises(B.ApError, match="row to row"):
        B.scores_int8(x, torch.ones(16, dtype=torch.int8, device=DEV).expand(3, 16), s)
