"""The softmax loss over all documents and its gradients (ap_softmax_loss, ap_softmax_loss_grad) against the formula in 64 bits.

Bounds.  A logit is a sum of dim products: off by at most (dim + 8) 2^-24 of scale sum |x_k w_k|, the sum's rounding, and f32 rows, which are
multiplied as two parts of 11 bits, by 2^-21 of it more; call the largest of a query E.  lse and the loss are off by at most 2 E, and by 2^-19
of 1 + |lse| for the exponentials, the sums and the roundings of the results.  A coefficient is off by (2 E + 2^-18 (1 + |lse|)) of p, and by
its rounding: 2^-8 of itself in one bf16 part (more than 128 queries), 2^-16 in two, 2^-21 in two f16 parts (and 2^-38, where f16 has no
smaller numbers, of the largest weight).  A gradient is off by the coefficients' bounds times the magnitudes that they multiply, (terms + 8)
2^-24 of the sum of magnitudes, and its own rounding, 2^-8 in bf16."""
import numpy as np
import pytest
import torch

from paper_2511_00855_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


def make(rng, rows, n, dim, dtype, stride=0, size=1.0):
    def m(r):
        t = torch.full((r, dim + stride), float("nan"), dtype=dtype, device=DEV)
        t[:, :dim] = torch.from_numpy((rng.standard_normal((r, dim)) * size * dim ** -0.5).astype(np.float32)).to(DEV, dtype)
        return t[:, :dim]
    labels = torch.from_numpy(rng.integers(0, n, rows).astype(np.int32)).to(DEV)
    return m(rows), m(n), labels


def check(x, docs, labels, scale, row_grad, want=(True, True)):
    dtype, (rows, dim), n = x.dtype, x.shape, docs.shape[0]
    loss, lse = B.softmax_loss(x, docs, labels, scale=scale)
    gx, gd = B.softmax_loss_grad(x, docs, labels, lse, row_grad, scale=scale, want_x=want[0], want_docs=want[1])
    X, D, lab, g = x.double().cpu(), docs.double().cpu(), labels.long().cpu(), row_grad.double().cpu()
    known = (lab >= 0) & (lab < n) & (g != 0)
    has = (lab >= 0) & (lab < n)
    at = torch.where(has, lab, 0)
    logits = scale * (X @ D.T)
    e = scale * (X.abs() @ D.abs().T) * ((dim + 8) * 2.0 ** -24 + (2.0 ** -21 if dtype is F32 else 0.0))   # of each logit
    E = e.amax(1)
    L = torch.logsumexp(logits, 1)
    r = torch.arange(rows)
    tol = 2 * E + 2.0 ** -19 * (1 + L.abs())
    assert ((lse.double().cpu() - L).abs() <= tol).all()
    assert ((loss.double().cpu() - torch.where(has, L - logits[r, at], 0.0)).abs() <= tol).all()
    assert (loss.cpu()[~has] == 0).all()
    p = torch.exp(logits - L[:, None])
    c = p.clone()
    c[r, at] -= 1.0
    c *= torch.where(known, g, 0.0)[:, None]
    rounding = 2.0 ** -21 if dtype is F32 else 2.0 ** -16 if rows <= 128 else 2.0 ** -8
    most = float(g[known].abs().max()) if known.any() else 1.0
    dc = p * (g.abs() * known * (2 * E + 2.0 ** -18 * (1 + L.abs())))[:, None] + c.abs() * rounding + most * 2.0 ** -38 * known[:, None]
    out = 2.0 ** -8 if dtype is BF16 else 2.0 ** -23
    inner = 2.0 ** -21 if dtype is F32 else 0.0   # the other factor's parts
    if want[0]:
        ref, bound = scale * (c @ D), scale * (dc @ D.abs() + (c.abs() @ D.abs()) * ((n + 8) * 2.0 ** -24 + inner))
        off = (gx.double().cpu() - ref).abs()
        assert gx.dtype is dtype and (off <= bound + out * ref.abs() + 1e-37).all(), float((off / (bound + out * ref.abs() + 1e-37)).max())
        assert (gx.cpu()[~known] == 0).all()
    else:
        assert gx is None
    if want[1]:
        X0 = torch.where(known[:, None], X, 0.0)
        ref, bound = scale * (c.T @ X0), scale * (dc.T @ X0.abs() + (c.T.abs() @ X0.abs()) * ((rows + 8) * 2.0 ** -24 + inner))
        off = (gd.double().cpu() - ref).abs()
        assert gd.dtype is dtype and (off <= bound + out * ref.abs() + 1e-37).all(), float((off / (bound + out * ref.abs() + 1e-37)).max())
    else:
        assert gd is None
    return loss, lse, gx, gd


@pytest.mark.parametrize("dtype,rows,n,dim,stride", [
    (F32, 1, 1, 4, 0), (BF16, 1, 1, 8, 0), (F32, 1, 1001, 260, 0), (BF16, 3, 777, 264, 8), (F32, 16, 64, 100, 4), (BF16, 17, 513, 1000, 0),
    (F32, 33, 300, 1024, 0), (BF16, 64, 2000, 128, 0), (F32, 65, 257, 36, 0), (BF16, 100, 1000, 520, 16), (F32, 129, 700, 500, 12),
    (BF16, 129, 255, 40, 0), (BF16, 300, 3000, 72, 0), (F32, 520, 1030, 64, 0), (BF16, 600, 4097, 264, 0), (F32, 40, 90, 2048, 0), (BF16, 5, 40, 8192, 0)])
@pytest.mark.parametrize("uneven", [False, True])
def test_loss_and_gradients(dtype, rows, n, dim, stride, uneven):
    rng = np.random.default_rng(rows * 7 + n)
    x, docs, labels = make(rng, rows, n, dim, dtype, stride)
    if rows > 8:
        labels[2], labels[5] = -1, n
    g = torch.from_numpy(rng.uniform(0.1, 1.0, rows).astype(np.float32)).to(DEV) if uneven else torch.full((rows,), 1.0 / rows, device=DEV)
    check(x, docs, labels, 7.0, g)


@pytest.mark.parametrize("dtype,rows,n,dim", [(BF16, 1100, 50_000, 136), (F32, 260, 60_001, 64)])
def test_tiles_of_256(dtype, rows, n, dim):
    rng = np.random.default_rng(n)
    x, docs, labels = make(rng, rows, n, dim, dtype)
    check(x, docs, labels, 10.0, torch.full((rows,), 1.0 / rows, device=DEV))


@pytest.mark.parametrize("dtype,rows,n,dim", [(BF16, 20, 3001, 72), (F32, 70, 1500, 100), (BF16, 300, 2600, 264)])
def test_pieces_of_the_documents(debug_knobs, dtype, rows, n, dim):
    """Coefficients of 256 or 512 documents at a time, with a short last piece, as with millions of them."""
    rng = np.random.default_rng(n)
    x, docs, labels = make(rng, rows, n, dim, dtype)
    g = torch.full((rows,), 0.5, device=DEV)
    whole = check(x, docs, labels, 5.0, g)
    for piece in (256, 512):
        debug_knobs("loss_piece", piece)
        got = check(x, docs, labels, 5.0, g)
        assert all(torch.equal(a, b) for a, b in zip(whole[:2], got[:2]))


@pytest.mark.parametrize("form", [1, 2])
@pytest.mark.parametrize("few", [0, 1])
@pytest.mark.parametrize("rows,n,dim", [(20, 300, 68), (64, 515, 260), (150, 700, 100), (1, 64, 8192)])
def test_forms_of_f32_products(debug_knobs, form, few, rows, n, dim):
    """The f32 instruction and the two f16 parts, tiles and passes over the documents, whatever the sizes would choose."""
    debug_knobs("loss_form", form)
    debug_knobs("loss_few", few)
    rng = np.random.default_rng(n)
    x, docs, labels = make(rng, rows, n, dim, F32)
    check(x, docs, labels, 6.0, torch.full((rows,), 1.0 / rows, device=DEV))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_queries_by_the_ten_thousand(dtype):
    """More queries than every workgroup looks through for the largest weight."""
    rng = np.random.default_rng(8)
    x, docs, labels = make(rng, 17_000, 90, 24, dtype)
    labels[5], labels[16_999] = -1, 90
    check(x, docs, labels, 5.0, torch.from_numpy(rng.uniform(-1.0, 1.0, 17_000).astype(np.float32)).to(DEV))


@pytest.mark.parametrize("rows", [3, 130])
def test_documents_past_32_bits(rows):
    """Documents of more than 2^32 bytes: labels among the last are found, and the gradient reaches them."""
    n, dim = 2_100_003, 1024
    docs = torch.zeros((n, dim), dtype=BF16, device=DEV)
    g = torch.Generator(DEV).manual_seed(1)
    docs[-300:] = (torch.randn((300, dim), generator=g, device=DEV) * dim ** -0.5).to(BF16)
    x = (docs[-rows:].float() * 0.5).to(BF16)
    labels = torch.arange(n - rows, n, dtype=torch.int32, device=DEV)
    loss, lse = B.softmax_loss(x, docs, labels, scale=20.0)
    gx, gd = B.softmax_loss_grad(x, docs, labels, lse, torch.ones(rows, device=DEV), scale=20.0)
    logits = 20.0 * (x.double() @ docs[-300:].double().T)
    want = torch.logsumexp(torch.cat([logits, torch.full((rows, 1), float(np.log(n - 300)), device=DEV, dtype=torch.float64)], 1), 1)
    own = logits[torch.arange(rows), 300 - rows + torch.arange(rows)]
    assert (lse.double() - want).abs().max() < 2e-5 and (loss.double() - (want - own)).abs().max() < 2e-5   # 2^-19 (1 + |lse|), twice the logits' sums
    c = torch.exp(logits - want[:, None])
    c[torch.arange(rows), 300 - rows + torch.arange(rows)] -= 1.0
    size = 20.0 * (c.abs() @ docs[-300:].double().abs())
    assert ((gx.double() - 20.0 * (c @ docs[-300:].double())).abs() <= 2.0 ** -7 * size).all()
    wd = 20.0 * (c.T @ x.double())
    assert ((gd[-300:].double() - wd).abs() <= 2.0 ** -7 * 20.0 * (c.T.abs() @ x.double().abs())).all()
    assert torch.isfinite(gd[:1000]).all() and (gd[:1000].double() - 20.0 * (torch.exp(-want) @ x.double())).abs().max() <= 2.0 ** -7 * 20.0 * float((torch.exp(-want) @ x.double().abs()).max())


@pytest.mark.parametrize("want", [(True, False), (False, True)])
@pytest.mark.parametrize("dtype,rows", [(BF16, 200), (F32, 9)])
def test_one_gradient_alone(dtype, rows, want):
    rng = np.random.default_rng(rows)
    x, docs, labels = make(rng, rows, 900, 96, dtype)
    both = check(x, docs, labels, 3.0, torch.ones(rows, device=DEV))
    one = check(x, docs, labels, 3.0, torch.ones(rows, device=DEV), want)
    assert all(b is None or torch.equal(a, b) for a, b in zip(both, one))


@pytest.mark.parametrize("dtype,rows", [(BF16, 6), (BF16, 150), (F32, 6), (F32, 150)])
def test_queries_without_a_part_do_not_show(dtype, rows):
    """NaN and infinities in queries that have no label or no weight reach no result but their own lse."""
    rng = np.random.default_rng(rows)
    x, docs, labels = make(rng, rows, 500, 64, dtype)
    g = torch.ones(rows, device=DEV)
    labels[1], g[3], labels[4] = -1, 0.0, 500
    clean = B.softmax_loss(x, docs, labels, scale=4.0)
    want = B.softmax_loss_grad(x, docs, labels, clean[1], g, scale=4.0)
    y = x.clone()
    y[1], y[3], y[4] = float("nan"), float("inf"), -float("inf")
    loss, lse = B.softmax_loss(y, docs, labels, scale=4.0)
    keep = [i for i in range(rows) if i not in (1, 3, 4)]
    assert torch.equal(loss[keep], clean[0][keep]) and torch.equal(lse[keep], clean[1][keep]) and loss[1] == 0 and loss[4] == 0
    got = B.softmax_loss_grad(y, docs, labels, lse, g, scale=4.0)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype,rows", [(BF16, 10), (BF16, 140), (F32, 10), (F32, 140)])
def test_nothing_is_asked_for(dtype, rows):
    rng = np.random.default_rng(rows)
    x, docs, labels = make(rng, rows, 300, 32, dtype)
    labels[:] = -1
    loss, lse = B.softmax_loss(x, docs, labels)
    assert (loss == 0).all() and torch.isfinite(lse).all()
    assert all((t == 0).all() for t in B.softmax_loss_grad(x, docs, labels, lse, torch.ones(rows, device=DEV)))


@pytest.mark.parametrize("size", [1e-12, 1e-4, 300.0, 1e12])
@pytest.mark.parametrize("rows", [4, 130])
def test_f32_rows_of_any_size(size, rows):
    """The two f16 parts come with a power of two of their own: tiny and huge rows, with a scale that brings the logits to size."""
    rng = np.random.default_rng(rows)
    x, docs, labels = make(rng, rows, 400, 60, F32, size=size)
    check(x, docs, labels, float(np.float32(4.0 / size ** 2)), torch.full((rows,), 1.0 / rows, device=DEV))


@pytest.mark.parametrize("rows", [3, 200])
def test_large_logits_and_a_sure_query(rows):
    """Logits of several hundred; a query whose label has all of the probability; one whose label has none."""
    rng = np.random.default_rng(5)
    x, docs, labels = make(rng, rows, 600, 128, BF16, size=6.0)
    x[0] = docs[labels[0].long()] * 4
    x[1] = -docs[labels[1].long()] * 4
    check(x, docs, labels, 3.0, torch.ones(rows, device=DEV))


@pytest.mark.parametrize("dtype,rows", [(F32, 12), (F32, 140)])
def test_gradients_are_the_losses_differences(dtype, rows):
    """Central differences of the summed loss along a direction.  With steps of h along unit directions, logits change by at most scale |w| h:
    the third derivative is at most (scale |w|)^3 a query, and the loss is off by 2^-19 (1 + |lse|) a query on either side."""
    rng = np.random.default_rng(rows)
    n, dim, scale, h = 300, 32, 2.0, 2.0 ** -5
    x, docs, labels = make(rng, rows, n, dim, dtype)
    loss, lse = B.softmax_loss(x, docs, labels, scale=scale)
    gx, gd = B.softmax_loss_grad(x, docs, labels, lse, torch.ones(rows, device=DEV), scale=scale)
    v = torch.from_numpy(rng.standard_normal((rows, dim)).astype(np.float32)).to(DEV)
    v /= v.norm(dim=1, keepdim=True)
    u = torch.from_numpy(rng.standard_normal((n, dim)).astype(np.float32)).to(DEV)
    u /= u.norm(dim=1, keepdim=True)
    most = float(max(x.norm(dim=1).max(), docs.norm(dim=1).max()))
    tol = rows * ((scale * most) ** 3 * h * h / 6 * 2 + 2 * 2.0 ** -19 * (1 + float(lse.abs().max())) / h)
    for a, b, grad, along in ((v, 0 * docs, gx, v), (0 * x, u, gd, u)):
        up = B.softmax_loss(x + h * a, docs + h * b, labels, scale=scale)[0].double().sum()
        down = B.softmax_loss(x - h * a, docs - h * b, labels, scale=scale)[0].double().sum()
        assert abs((up - down) / (2 * h) - (grad.double() * along.double()).sum()) <= tol


@pytest.mark.parametrize("dtype,rows", [(BF16, 5), (BF16, 200), (F32, 200)])
def test_same_bits_on_another_stream_and_in_a_graph(dtype, rows):
    rng = np.random.default_rng(rows)
    x, docs, labels = make(rng, rows, 1500, 64, dtype)
    g = torch.full((rows,), 0.01, device=DEV)

    def step():
        loss, lse = B.softmax_loss(x, docs, labels, scale=9.0)
        return (loss, lse, *B.softmax_loss_grad(x, docs, labels, lse, g, scale=9.0))
    want = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(3):
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out)), i
        step()


def test_no_queries():
    docs = torch.ones((5, 8), device=DEV)
    x = torch.ones((0, 8), device=DEV)
    labels = torch.zeros(0, dtype=torch.int32, device=DEV)
    loss, lse = B.softmax_loss(x, docs, labels)
    assert loss.shape == lse.shape == (0,)
    gx, gd = B.softmax_loss_grad(x, docs, labels, lse, lse)
    assert gx.shape == (0, 8) and (gd == 0).all()


def test_bf16_rows_of_device_vecs():
    """int16 holds bf16 as DeviceVecs keeps it."""
    rng = np.random.default_rng(1)
    x, docs, labels = make(rng, 20, 100, 64, BF16)
    want = B.softmax_loss(x, docs, labels)
    got = B.softmax_loss(x, docs.view(torch.int16), labels)
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_refusals():
    x, docs, labels = torch.ones((3, 16), device=DEV), torch.ones((5, 16), device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV)
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(B.ApError, match="scale"):
            B.softmax_loss(x, docs, labels, scale=scale)
    with pytest.raises(ValueError, match="type"):
        B.softmax_loss(x, docs.bfloat16(), labels)
    with pytest.raises(ValueError, match="columns"):
        B.softmax_loss(x, docs[:, :8], labels)
    with pytest.raises(ValueError, match="labels"):
        B.softmax_loss(x, docs, labels[:2])
    with pytest.raises(B.ApError, match="multiple of 4"):
        B.softmax_loss(x[:, :6], docs[:, :6], labels)
    with pytest.raises(B.ApError, match="aligned"):
        B.softmax_loss(torch.ones(49, device=DEV)[1:].view(3, 16), docs, labels)
    with pytest.raises(B.ApError, match="neither"):
        B.softmax_loss_grad(x, docs, labels, torch.ones(3, device=DEV), torch.ones(3, device=DEV), want_x=False, want_docs=False)
