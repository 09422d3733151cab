"""Dense rows out of token lists and their gradients (ap_embed, ap_embed_grad, ap_embed_grad_weights) against the formula in 64 bits.

Bounds: a sum of L products in f32, each of two roundings, is off by at most (L + 3) 2^-24 of the sum of the products' magnitudes, and
a result rounded to bf16 by 2^-8 of itself more (f32: 2^-24)."""
import numpy as np
import pytest
import torch

from paper_2511_00855_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


def lists_of(rng, rows, vocab, longest, hot=False):
    """Lists of 0 to `longest` tokens, unused slots among them; hot: half of the tokens are one."""
    lengths = rng.integers(0, longest + 1, rows)
    lengths[rng.random(rows) < 0.2] = 0
    indptr = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)
    n = int(indptr[-1])
    tokens = rng.integers(0, vocab, n).astype(np.int32)
    if hot:
        tokens[rng.random(n) < 0.5] = vocab // 2
    tokens[rng.random(n) < 0.05] = -1
    tokens[rng.random(n) < 0.02] = vocab   # outside as well
    return torch.from_numpy(indptr), torch.from_numpy(tokens), torch.from_numpy(rng.standard_normal(n).astype(np.float32))


def matrix(rng, rows, dim, dtype, stride=0):
    """rows x dim on the GPU, `stride` more elements from row to row (NaN between them)."""
    m = torch.full((rows, dim + stride), float("nan"), dtype=dtype, device=DEV)
    m[:, :dim] = torch.from_numpy(rng.standard_normal((rows, dim)).astype(np.float32)).to(DEV, dtype)
    return m[:, :dim]


def plain(table, indptr, tokens, weights, scale, grad=None):
    """(rows, sum of magnitudes) of the lists; with grad also both gradients and their magnitudes.  All in 64 bits on the CPU."""
    t = table.double().cpu()
    n = len(tokens)
    row = torch.arange(n) if indptr is None else torch.searchsorted(indptr, torch.arange(n), right=True) - 1
    rows = n if indptr is None else len(indptr) - 1
    used = (tokens >= 0) & (tokens < t.shape[0])
    w = (torch.ones(n, dtype=torch.float64) if weights is None else weights.double()) * scale * used
    at = torch.where(used, tokens.long(), 0)
    e = t[at] * w[:, None]
    out = [torch.zeros((rows, t.shape[1]), dtype=torch.float64).index_add_(0, row, v) for v in (e, e.abs())]
    if grad is None:
        return out
    g = grad.double().cpu()[row]
    gt = [torch.zeros_like(t).index_add_(0, at, v) for v in (g * w[:, None], (g * w[:, None]).abs())]
    dots = t[at] * g * scale * used[:, None]
    return out, gt, [dots.sum(1), dots.abs().sum(1)]


def near(got, want, size, terms, dtype):
    bound = (terms + 3) * 2.0 ** -24 * size + (2.0 ** -8 if dtype is BF16 else 2.0 ** -24) * want.abs() + 1e-37
    off = (got.double().cpu() - want).abs()
    assert torch.isfinite(got).all()
    assert (off <= bound).all(), float((off / bound).max())


@pytest.mark.parametrize("dtype,out_dtype,dim,rows,longest,weighted,stride", [
    (F32, F32, 4, 5, 3, True, 0), (F32, F32, 260, 33, 40, True, 4), (F32, BF16, 264, 33, 9, False, 0), (BF16, BF16, 8, 100, 20, True, 0),
    (BF16, F32, 1000, 21, 70, True, 24), (BF16, BF16, 2048, 3, 300, False, 0), (F32, F32, 96, 2000, 5, True, 32), (F32, F32, 8192, 2, 30, True, 0)])
def test_lists(dtype, out_dtype, dim, rows, longest, weighted, stride):
    rng = np.random.default_rng(dim + rows)
    table = matrix(rng, 50, dim, dtype, stride)
    indptr, tokens, weights = lists_of(rng, rows, 50, longest)
    w = weights if weighted else None
    got = B.embed(table, tokens.to(DEV), None if w is None else w.to(DEV), indptr.to(DEV), scale=0.37, out_dtype=out_dtype)
    want, size = plain(table, indptr, tokens, w, 0.37)
    assert got.dtype is out_dtype
    near(got, want, size, longest, out_dtype)
    assert (got[indptr.diff() == 0] == 0).all()


@pytest.mark.parametrize("dtype,dim,n", [(F32, 100, 1), (BF16, 128, 777), (F32, 768, 64)])
def test_one_token_a_row(dtype, dim, n):
    rng = np.random.default_rng(n)
    table = matrix(rng, 31, dim, dtype)
    tokens = torch.from_numpy(rng.integers(0, 31, n).astype(np.int32))
    got = B.embed(table, tokens.to(DEV), scale=1.5)
    want, size = plain(table, None, tokens, None, 1.5)
    near(got, want, size, 1, dtype)


@pytest.mark.parametrize("few", [0, 1])
@pytest.mark.parametrize("dtype,table_dtype,dim,vocab,rows,longest,weighted,hot,stride", [
    (F32, F32, 4, 3, 7, 3, True, False, 0), (F32, F32, 260, 50, 90, 30, True, True, 4), (F32, BF16, 264, 1000, 33, 9, False, False, 0),
    (BF16, BF16, 1000, 70_000, 60, 40, True, False, 8), (BF16, F32, 128, 513, 150, 30, True, True, 0), (BF16, BF16, 520, 2, 200, 20, True, True, 0)])
def test_gradient_of_the_table(debug_knobs, few, dtype, table_dtype, dim, vocab, rows, longest, weighted, hot, stride):
    """Both ways: entries that find their equals (up to 4,096), and sorted ones."""
    debug_knobs("embed_few", few)
    rng = np.random.default_rng(vocab + rows)
    indptr, tokens, weights = lists_of(rng, rows, vocab, longest, hot)
    w = weights if weighted else None
    grad = matrix(rng, rows, dim, dtype, stride)
    table = torch.zeros((vocab, dim), device=DEV)
    args = (grad, tokens.to(DEV), vocab, None if w is None else w.to(DEV), indptr.to(DEV))
    got = B.embed_grad(*args, scale=-2.5, dtype=table_dtype)
    _, (want, size), _ = plain(table, indptr, tokens, w, -2.5, grad)
    count = torch.bincount(tokens[(tokens >= 0) & (tokens < vocab)].long(), minlength=vocab)
    near(got, want, size, int(count.max()), table_dtype)
    assert (got[(count == 0).to(DEV)] == 0).all()
    assert torch.equal(got, B.embed_grad(*args, scale=-2.5, dtype=table_dtype))


@pytest.mark.parametrize("vocab,n,dim", [(300, 4_097, 132), (250_002, 9_000, 64), (1, 5_000, 256), (1 << 19, 70_000, 8)])
def test_gradient_of_many_tokens(vocab, n, dim):
    """More entries than are compared with each other: keys of one to three passes, tokens over many runs."""
    rng = np.random.default_rng(n)
    tokens = torch.from_numpy(np.minimum(rng.zipf(1.2, n) - 1, vocab).astype(np.int32))   # some past the end
    grad = matrix(rng, n, dim, F32)
    got = B.embed_grad(grad, tokens.to(DEV), vocab, scale=0.5)
    _, (want, size), _ = plain(torch.zeros((vocab, dim)), None, tokens, None, 0.5, grad)
    near(got, want, size, n, F32)


@pytest.mark.parametrize("counts,dim,table_dtype", [
    ([64, 128, 64 * 16, 64 * 17, 64 * 18, 63, 1, 65], 72, F32),           # tokens that end with a run, of up to and over 16 runs
    ([1, 64 * 17 - 1, 64 * 17, 64 * 17 + 1, 2, 64 * 40 + 5], 520, BF16),
    ([32, 32 * 16, 31, 32 * 17, 1, 32 * 18 - 1, 33, 32 * 50], 24, F32), ([5] * 800 + [32 * 16 + 1] * 2, 1000, BF16),
    ([30_000] * 10 + [3] * 100, 8, F32)])                                  # longer blocks of the sort
def test_gradient_of_tokens_over_many_runs(counts, dim, table_dtype):
    rng = np.random.default_rng(len(counts))
    tokens = np.repeat(np.arange(len(counts), dtype=np.int32), counts)
    tokens = torch.from_numpy(rng.permutation(tokens))
    grad = matrix(rng, len(tokens), dim, F32)
    got = B.embed_grad(grad, tokens.to(DEV), len(counts) + 2, scale=2.0, dtype=table_dtype)
    _, (want, size), _ = plain(torch.zeros((len(counts) + 2, dim)), None, tokens, None, 2.0, grad)
    near(got, want, size, max(counts), table_dtype)
    assert torch.equal(got, B.embed_grad(grad, tokens.to(DEV), len(counts) + 2, scale=2.0, dtype=table_dtype))


@pytest.mark.parametrize("dtype,grad_dtype,dim,stride", [(F32, F32, 4, 0), (F32, F32, 260, 4), (BF16, BF16, 264, 8), (F32, BF16, 1000, 0), (BF16, F32, 2048, 0)])
def test_gradient_of_the_weights(dtype, grad_dtype, dim, stride):
    rng = np.random.default_rng(dim)
    indptr, tokens, weights = lists_of(rng, 41, 60, 17)
    table, grad = matrix(rng, 60, dim, dtype, stride), matrix(rng, 41, dim, grad_dtype, stride)
    got = B.embed_grad_weights(grad, table, tokens.to(DEV), indptr.to(DEV), scale=3.0)
    _, _, (want, size) = plain(table, indptr, tokens, weights, 3.0, grad)
    near(got, want, size, dim, F32)


@pytest.mark.parametrize("dtype,grad_dtype,dim,rows,lists", [(F32, F32, 260, 4_500, True), (BF16, BF16, 264, 9, False), (BF16, F32, 72, 33_001, False), (BF16, BF16, 136, 4_500, True)])
def test_gradient_of_many_weights(dtype, grad_dtype, dim, rows, lists):
    rng = np.random.default_rng(dim)
    indptr, tokens, weights = lists_of(rng, rows, 60, 19 if rows > 9 else 20_000)
    if not lists:
        indptr, rows = None, len(tokens)
    table, grad = matrix(rng, 60, dim, dtype), matrix(rng, rows, dim, grad_dtype)
    assert len(tokens) > 32_768
    got = B.embed_grad_weights(grad, table, tokens.to(DEV), None if indptr is None else indptr.to(DEV), scale=3.0)
    _, _, (want, size) = plain(table, indptr, tokens, weights, 3.0, grad)
    near(got, want, size, dim, F32)


@pytest.mark.parametrize("few", [0, 1])
def test_lists_with_broken_offsets_have_no_gradient(debug_knobs, few):
    debug_knobs("embed_few", few)
    tokens, indptr = torch.arange(5, dtype=torch.int32, device=DEV), torch.tensor([0, 2, 1, 9], device=DEV)
    table, grad = torch.ones((8, 8), device=DEV), torch.ones((3, 8), device=DEV)
    assert B.embed_grad(grad, tokens, 8, None, indptr)[:, 0].tolist() == [1.0, 1.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0]
    assert B.embed_grad_weights(grad, table, tokens, indptr).tolist() == [8.0, 8.0, 0.0, 0.0, 0.0]


def test_gradients_are_the_rows_differences():
    """out is linear in the table and in the weights: <G, out(T + D) - out(T)> = <dT, D>, and so for the weights."""
    rng = np.random.default_rng(3)
    indptr, tokens, weights = (t.to(DEV) for t in lists_of(rng, 20, 30, 12))
    table, grad, step = matrix(rng, 30, 64, F32), matrix(rng, 20, 64, F32), matrix(rng, 30, 64, F32)
    step_w = torch.randn(len(weights), device=DEV)
    a = B.embed(table, tokens, weights, indptr, scale=0.7).double()
    b = B.embed(table + step, tokens, weights, indptr, scale=0.7).double()
    c = B.embed(table, tokens, weights + step_w, indptr, scale=0.7).double()
    size = (grad.double().abs() * (a.abs() + b.abs() + c.abs())).sum()   # every output is off by at most 16 roundings of its own magnitude's sum
    tol = 16 * 40 * 2.0 ** -24 * size
    assert abs((grad.double() * (b - a)).sum() - (B.embed_grad(grad, tokens, 30, weights, indptr, scale=0.7).double() * step.double()).sum()) <= tol
    assert abs((grad.double() * (c - a)).sum() - (B.embed_grad_weights(grad, table, tokens, indptr, scale=0.7).double() * step_w.double()).sum()) <= tol


def test_unused_rows_and_slots_do_not_show():
    """NaN in rows that no token names, infinite weights of unused slots, gradients of empty lists."""
    table = torch.full((6, 16), float("nan"), device=DEV)
    table[2] = 1.0
    tokens = torch.tensor([2, -1, 6, 2], dtype=torch.int32, device=DEV)
    weights = torch.tensor([1.0, float("inf"), float("nan"), 2.0], device=DEV)
    indptr = torch.tensor([0, 3, 3, 4], device=DEV)
    assert B.embed(table, tokens, weights, indptr).tolist() == [[1.0] * 16, [0.0] * 16, [2.0] * 16]
    grad = torch.ones((3, 16), device=DEV)
    grad[1] = float("nan")
    for few in (0, 1):
        B.debug_set("embed_few", few)
        got = B.embed_grad(grad, tokens, 6, weights, indptr)
        B.debug_reset()
        assert got[2].tolist() == [3.0] * 16 and (got[[0, 1, 3, 4, 5]] == 0).all()
    assert B.embed_grad_weights(grad, table, tokens, indptr).tolist() == [16.0, 0.0, 0.0, 16.0]


def test_lists_with_broken_offsets_are_empty():
    table = torch.ones((4, 8), device=DEV)
    tokens = torch.zeros(5, dtype=torch.int32, device=DEV)
    indptr = torch.tensor([0, 2, 1, 9], device=DEV)   # the second descends, the third ends past the tokens
    assert B.embed(table, tokens, None, indptr)[:, 0].tolist() == [2.0, 0.0, 0.0]


def test_no_rows_and_no_tokens():
    table = torch.ones((4, 8), device=DEV)
    none = torch.zeros(0, dtype=torch.int32, device=DEV)
    assert B.embed(table, none).shape == (0, 8)
    assert B.embed(table, none, None, torch.zeros(4, dtype=torch.int64, device=DEV)).tolist() == [[0.0] * 8] * 3
    assert B.embed_grad(torch.ones((3, 8), device=DEV), none, 4, None, torch.zeros(4, dtype=torch.int64, device=DEV)).abs().sum() == 0
    assert B.embed_grad(torch.ones((0, 8), device=DEV), none, 4).abs().sum() == 0


def test_offsets_past_32_bits():
    """A table of more than 2^32 bytes: its last rows are found, and the gradient reaches them."""
    vocab, dim = 1_100_003, 1024
    table = torch.zeros((vocab, dim), device=DEV)
    table[vocab - 1] = torch.arange(dim, device=DEV).float()
    tokens = torch.tensor([vocab - 1, 5, vocab - 1], dtype=torch.int32, device=DEV)
    assert torch.equal(B.embed(table, tokens)[2], table[vocab - 1])
    got = B.embed_grad(torch.ones((3, dim), device=DEV), tokens, vocab)
    assert (got[vocab - 1] == 2).all() and (got[5] == 1).all() and got.sum() == 3 * dim


def test_refusals():
    table = torch.ones((4, 16), device=DEV)
    tokens = torch.zeros(3, dtype=torch.int32, device=DEV)
    with pytest.raises(B.ApError, match="multiple of 4"):
        B.embed(torch.ones((4, 6), device=DEV), tokens)
    with pytest.raises(B.ApError, match="aligned"):
        B.embed(torch.ones(65, device=DEV)[1:].view(4, 16), tokens)
    with pytest.raises(B.ApError, match="row to row"):
        B.embed(torch.ones(16, device=DEV).expand(4, 16), tokens)
    with pytest.raises(ValueError, match="rows are contiguous"):
        B.embed(torch.ones((16, 4), device=DEV).T, tokens)
    with pytest.raises(ValueError, match="f32 or bf16"):
        B.embed(table.double(), tokens)
    with pytest.raises(ValueError, match="tokens"):
        B.embed(table, tokens.long())
    with pytest.raises(ValueError, match="weights"):
        B.embed(table, tokens, torch.ones(2, device=DEV))
    with pytest.raises(ValueError, match="rows for"):
        B.embed_grad(torch.ones((2, 16), device=DEV), tokens, 4)
    with pytest.raises(B.ApError, match="vocab"):
        B.embed_grad(torch.ones((3, 16), device=DEV), tokens, 0)
