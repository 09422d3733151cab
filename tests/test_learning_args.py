"""What the calls on dense rows refuse on the host, before any device work (no GPU needed): sizes, types, strides, alignment, workspaces."""
import ctypes as C

import pytest

from paper_2511_00855_amd import binding as B

A = 1 << 12   # an address that is never read


def refused(rc, word):
    assert rc == -1 and word in B.lib().ap_last_error().decode(), (rc, B.lib().ap_last_error())


def test_workspaces_grow_with_the_work():
    L, out = B.lib(), C.c_size_t()
    got = []
    for rows, n in ((1, 1), (64, 1000), (300, 10_000), (4096, 250_002)):
        for dtype in (B.AP_F32, B.AP_BF16):
            assert L.ap_softmax_loss_bytes(rows, n, 768, dtype, C.byref(out)) == 0
            got.append(out.value)
            assert L.ap_softmax_loss_grad_bytes(rows, n, 768, dtype, 1, C.byref(out)) == 0
            got.append(out.value)
    assert all(0 < v < 4 << 30 for v in got)
    # the logits of the largest would take 4 GB
    assert got[-1] < 1 << 30
    assert L.ap_embed_grad_bytes(100_000, 30_522, 768, C.byref(out)) == 0 and out.value > 0
    assert L.ap_scores_int8_bytes(1, 768, B.AP_F32, C.byref(out)) == 0 and out.value == 0
    for fn, args in ((L.ap_softmax_loss_bytes, (1, 1, 4, 0, None)), (L.ap_softmax_loss_grad_bytes, (1, 1, 4, 0, 1, None)), (L.ap_embed_grad_bytes, (1, 1, 4, None)),
                     (L.ap_scores_int8_bytes, (1, 4, 0, None))):
        refused(fn(*args), "out is NULL")


@pytest.mark.parametrize("change,word", [
    (dict(dtype=2), "dtype"), (dict(dim=6), "dim"), (dict(dim=0), "dim"), (dict(dim=8196, ldx=8196, ldd=8196), "dim"), (dict(rows=-1), "rows"), (dict(rows=(1 << 24) + 1), "rows"),
    (dict(n=0), "n ="), (dict(n=1 << 30), "n ="), (dict(ldx=12), "row to row"), (dict(ldd=18), "row to row"), (dict(ldd=(1 << 20) + 4), "row to row"), (dict(x=0), "x is NULL"),
    (dict(docs=0), "docs is NULL"), (dict(x=A + 4), "aligned"), (dict(labels=0), "labels"), (dict(scale=0.0), "scale"), (dict(scale=float("nan")), "scale"), (dict(bytes=16), "workspace"),
    (dict(ws=0), "workspace")])
def test_softmax_loss(change, word):
    a = dict(x=A, ldx=16, rows=3, docs=A, ldd=16, n=5, dim=16, dtype=0, scale=1.0, labels=A, ws=A, bytes=1 << 30) | change
    head = (a["x"], a["ldx"], a["rows"], a["docs"], a["ldd"], a["n"], a["dim"], a["dtype"], a["scale"], a["labels"])
    refused(B.lib().ap_softmax_loss(*head, A, A, a["ws"], a["bytes"], None), word)
    refused(B.lib().ap_softmax_loss_grad(*head, A, A, A, A, a["ws"], a["bytes"], None), word)


def test_softmax_loss_grad_of_nothing():
    head = (A, 16, 3, A, 16, 5, 16, 0, 1.0, A)
    refused(B.lib().ap_softmax_loss_grad(*head, A, A, None, None, A, 1 << 30, None), "neither")
    refused(B.lib().ap_softmax_loss_grad(*head, None, A, A, A, A, 1 << 30, None), "NULL")
    refused(B.lib().ap_softmax_loss_grad(*head, A, A, A + 4, A, A, 1 << 30, None), "aligned")
    refused(B.lib().ap_softmax_loss(*head, None, A, A, 1 << 30, None), "NULL")


def test_embed():
    L = B.lib()
    lists = B._Lists(2, 3, A, A, None)
    ok = dict(table=A, ld=16, dtype=0, vocab=9, dim=16, lists=C.byref(lists), out=A, out_dtype=0)

    def call(**change):
        a = ok | change
        return L.ap_embed(a["table"], a["ld"], a["dtype"], a["vocab"], a["dim"], a["lists"], 1.0, a["out"], a["out_dtype"], None)
    for change, word in ((dict(table=None), "NULL"), (dict(ld=8), "row to row"), (dict(dtype=3), "dtype"), (dict(vocab=0), "vocab"), (dict(dim=18), "dim"), (dict(lists=None), "lists"),
                         (dict(out=None), "NULL"), (dict(out=A + 8), "aligned"), (dict(out_dtype=3), "dtype"), (dict(dim=12, ld=12, out_dtype=1), "multiple of 8"),
                         (dict(lists=C.byref(B._Lists(2, 3, None, A, None))), "indptr"), (dict(lists=C.byref(B._Lists(2, 3, A, None, None))), "tokens"),
                         (dict(lists=C.byref(B._Lists(1 << 28, 3, A, A, None))), "rows")):
        refused(call(**change), word)
    refused(L.ap_embed_grad(A, 16, 0, 16, C.byref(lists), 9, 1.0, None, 0, None, 0, None), "NULL")
    refused(L.ap_embed_grad(A, 16, 7, 16, C.byref(lists), 9, 1.0, A, 0, None, 0, None), "dtype")
    refused(L.ap_embed_grad(A, 16, 0, 16, C.byref(B._Lists(100_000, 100_000, None, A, None)), 9, 1.0, A, 0, A, 64, None), "workspace")
    refused(L.ap_embed_grad_weights(A, 16, 0, A, 16, 0, 9, 16, C.byref(lists), 1.0, None, A, 64, None), "NULL")
    refused(L.ap_embed_grad_weights(A, 12, 0, A, 16, 0, 9, 16, C.byref(lists), 1.0, A, A, 64, None), "row to row")
    refused(L.ap_embed_grad_weights(A, 256, 0, A, 256, 0, 9, 256, C.byref(B._Lists(100_000, 100_000, None, A, None)), 1.0, A, A, 16, None), "workspace")


def test_eight_bits():
    L = B.lib()
    refused(L.ap_quantize_rows(A, 16, 3, 16, 3, A, 16, A, None), "dtype")
    refused(L.ap_quantize_rows(A, 20, 3, 20, 0, A, 20, A, None), "row to row")
    refused(L.ap_quantize_rows(A, 16, 3, 16, 0, A + 4, 16, A, None), "aligned")
    refused(L.ap_quantize_rows(A, 16, 3, 16, 0, A, 16, None, None), "scale")
    ok = (A, 16, A, 3, 16, 3, A, 16, A, 5, A, 5, A, 1 << 20, None)
    for at, value, word in ((0, None, "NULL"), (1, 8, "row to row"), (2, None, "x_scale"), (4, 24, "dim"), (5, 9, "dtype"), (6, None, "NULL"), (7, 8, "row to row"), (9, 0, "n ="),
                            (10, None, "out"), (11, 4, "ld_out")):
        refused(L.ap_scores_int8(*ok[:at], value, *ok[at + 1:]), word)
    refused(L.ap_scores_int8(A, 16, None, 300, 16, 0, A, 16, A, 5, A, 5, A, 8, None), "workspace")
