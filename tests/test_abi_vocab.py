"""Refusals of the vocabulary's and the clipping's entry points, without a GPU: every call stops at a host check."""
import ctypes

import pytest

from paper_1805_08899_amd import binding as eb

A = 0x10000  # a fake, aligned, never dereferenced device address


def _embed_fwd(desc, **kw):
    args = dict(tokens=A, table=A, scale=1.0, out=A)
    args.update(kw)
    return eb.echo_embed_fwd(desc, **args)


def _embed_bwd(desc, call="echo_embed_bwd", **kw):
    args = dict(tokens=A, dout=A, scale=1.0, dtable=A, workspace=A, workspace_bytes=1 << 50)
    args.update(kw)
    return getattr(eb, call)(desc, **args)


def _loss_fwd(desc, **kw):
    args = dict(h=A, W=A, labels=A, label_smoothing=0.1, loss=A, lse=A, workspace=A, workspace_bytes=1 << 50)
    args.update(kw)
    return eb.echo_vocab_loss_fwd(desc, **args)


def _loss_bwd(desc, **kw):
    args = dict(dloss=A, lse=A, h=A, W=A, labels=A, label_smoothing=0.1, dh=A, dW=A, workspace=A, workspace_bytes=1 << 50)
    args.update(kw)
    return eb.echo_vocab_loss_bwd(desc, **args)


CALLS = {
    "fwd": (_embed_fwd, ("tokens", "table", "out")),
    "bwd": (_embed_bwd, ("tokens", "dout", "dtable", "workspace")),
    "acc": (lambda d, **kw: _embed_bwd(d, "echo_embed_bwd_accumulate", **kw), ("tokens", "dout", "dtable", "workspace")),
    "loss": (_loss_fwd, ("h", "W", "labels", "loss", "lse", "workspace")),
    "dloss": (_loss_bwd, ("dloss", "lse", "h", "W", "labels", "workspace")),
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_pointers_types_and_limits(name):
    call, pointers = CALLS[name]
    good = eb.make_vocab_desc(5, 7, 9)
    stop = {pointers[0]: None}                            # stops at the check behind those of the descriptor
    for p in pointers:
        assert call(good, **{p: None}) == eb.ECHO_ERR_NULL, p
        assert call(good, **{p: A + 4}) == eb.ECHO_ERR_ALIGN, p
    most = eb.make_vocab_desc(eb.ECHO_VOCAB_MAX_ROWS, eb.ECHO_VOCAB_MAX_ROWS, eb.ECHO_VOCAB_MAX_D)
    assert call(most, **stop) == eb.ECHO_ERR_NULL
    for field, limit in (("N", eb.ECHO_VOCAB_MAX_ROWS), ("V", eb.ECHO_VOCAB_MAX_ROWS), ("D", eb.ECHO_VOCAB_MAX_D)):
        for value in (0, -1, limit + 1, -2 ** 31):
            d = eb.make_vocab_desc(5, 7, 9)
            setattr(d, field, value)
            assert call(d) == eb.ECHO_ERR_SHAPE, (field, value)
    for field in ("in_dtype", "out_dtype"):
        for value in (-1, 2):
            d = eb.make_vocab_desc(5, 7, 9)
            setattr(d, field, value)
            assert call(d) == eb.ECHO_ERR_DTYPE, (field, value)
    with pytest.raises(TypeError):
        call(eb.make_desc(1, 1, 1, 1, 4))


def test_types_that_go_together():
    assert _loss_fwd(eb.make_vocab_desc(5, 7, 9, "f32", "bf16")) == eb.ECHO_ERR_DTYPE
    assert _loss_bwd(eb.make_vocab_desc(5, 7, 9, "f32", "bf16")) == eb.ECHO_ERR_DTYPE
    assert _loss_bwd(eb.make_vocab_desc(5, 7, 9, "bf16", "bf16"), h=None) == eb.ECHO_ERR_NULL
    assert _embed_fwd(eb.make_vocab_desc(5, 7, 9, "f32", "bf16"), out=None) == eb.ECHO_ERR_NULL


def test_numbers():
    good = eb.make_vocab_desc(5, 7, 9)
    for s in (float("nan"), float("inf"), float("-inf")):
        assert _embed_fwd(good, scale=s) == eb.ECHO_ERR_SHAPE and _embed_bwd(good, scale=s) == eb.ECHO_ERR_SHAPE
    for e in (-0.1, 1.0, 2.0, float("nan")):
        assert _loss_fwd(good, label_smoothing=e) == eb.ECHO_ERR_SHAPE and _loss_bwd(good, label_smoothing=e) == eb.ECHO_ERR_SHAPE
    assert _loss_bwd(good, dh=None, dW=None) == eb.ECHO_ERR_NULL
    assert _loss_bwd(good, dh=None, dW=A + 2) == eb.ECHO_ERR_ALIGN


def test_workspaces():
    good = eb.make_vocab_desc(50, 70, 90)
    for query, call in ((eb.echo_embed_bwd_workspace_bytes, _embed_bwd), (eb.echo_vocab_loss_fwd_workspace_bytes, _loss_fwd),
                        (eb.echo_vocab_loss_bwd_workspace_bytes, _loss_bwd)):
        need = query(good)
        assert need > 0 and call(good, workspace_bytes=need - 1) == eb.ECHO_ERR_WORKSPACE
        assert query(eb.make_vocab_desc(0, 7, 9)) == 0
    L = eb.lib()
    assert L.echo_vocab_loss_fwd_workspace_bytes(None) == 0
    assert L.echo_embed_fwd(None, A, A, 1.0, A, None) == eb.ECHO_ERR_NULL
    # nothing of the size of the logits: 8 GB of them, a twentieth for the backward pass
    d = eb.make_vocab_desc(16384, 131072, 1024, "bf16", "f32")
    logits = 4 * 16384 * 131072
    assert eb.echo_vocab_loss_fwd_workspace_bytes(d) < logits // 16 and eb.echo_vocab_loss_bwd_workspace_bytes(d) < logits // 8
    # sizes stay sums of 64-bit numbers at the limits
    most = eb.make_vocab_desc(eb.ECHO_VOCAB_MAX_ROWS, eb.ECHO_VOCAB_MAX_ROWS, eb.ECHO_VOCAB_MAX_D)
    assert eb.echo_vocab_loss_bwd_workspace_bytes(most) > 1 << 40 and eb.echo_embed_bwd_workspace_bytes(most) > 1 << 36


def _grads(*entries):
    a = (eb.echo_grad_t * len(entries))()
    for e, (grad, clipped, n, dtype) in zip(a, entries):
        e.grad, e.clipped, e.n, e.dtype = grad, clipped, n, dtype
    return a


def test_clipping_refuses():
    ok = (A, A, 10, eb.ECHO_F32)

    def clip(*entries, count=None, max_norm=1.0, norm=A, workspace=A, workspace_bytes=1 << 20):
        g = _grads(*entries)
        return eb.echo_grad_clip(g, len(g) if count is None else count, max_norm, norm, workspace, workspace_bytes)

    def norm_(*entries, norm=A, workspace=A, workspace_bytes=1 << 20):
        g = _grads(*entries)
        return eb.echo_grad_norm(g, len(g), norm, workspace, workspace_bytes)

    for call in (clip, norm_):
        assert call(ok, norm=None) == eb.ECHO_ERR_NULL and call(ok, workspace=None) == eb.ECHO_ERR_NULL
        assert call(ok, norm=A + 4) == eb.ECHO_ERR_ALIGN and call(ok, workspace=A + 8) == eb.ECHO_ERR_ALIGN
        assert call(ok, (None, A, 1, eb.ECHO_F32)) == eb.ECHO_ERR_NULL
        assert call(ok, (A + 2, A, 1, eb.ECHO_BF16)) == eb.ECHO_ERR_ALIGN
        assert call(ok, (A, A, -1, eb.ECHO_F32)) == eb.ECHO_ERR_SHAPE
        assert call(ok, (A, A, (1 << 40) + 1, eb.ECHO_F32)) == eb.ECHO_ERR_SHAPE
        assert call(ok, (A, A, 1, 2)) == eb.ECHO_ERR_DTYPE
        assert call(ok, workspace_bytes=eb.echo_grad_workspace_bytes(_grads(ok), 1) - 1) == eb.ECHO_ERR_WORKSPACE
    assert clip((A, None, 1, eb.ECHO_F32)) == eb.ECHO_ERR_NULL
    assert clip((A, A + 4, 1, eb.ECHO_F32)) == eb.ECHO_ERR_ALIGN
    for m in (0.0, -1.0, float("nan")):
        assert clip(ok, max_norm=m) == eb.ECHO_ERR_SHAPE
    assert clip(ok, count=0) == eb.ECHO_ERR_SHAPE
    with pytest.raises(ValueError):
        clip(ok, count=2)
    with pytest.raises(TypeError):
        eb.echo_grad_clip(A, 1, 1.0, A, A, 1 << 20)
    assert eb.echo_grad_workspace_bytes(_grads(ok), 0) == 0
    many = _grads(*[ok] * (eb.ECHO_GRAD_MAX_COUNT + 1))
    assert eb.echo_grad_clip(many, len(many), 1.0, A, A, 1 << 20) == eb.ECHO_ERR_SHAPE
    L = eb.lib()
    assert L.echo_grad_clip(None, 1, 1.0, A, A, 1 << 20, None) == eb.ECHO_ERR_NULL


def test_make_grads():
    import torch
    a, b = torch.zeros(6), torch.zeros(2, 3, dtype=torch.bfloat16)
    g = eb.make_grads([a, b])
    assert [(e.grad, e.clipped, e.n, e.dtype) for e in g] == [(a.data_ptr(), a.data_ptr(), 6, 0), (b.data_ptr(), b.data_ptr(), 6, 1)]
    out = torch.zeros(6)
    assert eb.make_grads([a], [out])[0].clipped == out.data_ptr()
    for bad in (([b.t()], None), ([a], [b]), ([a], [torch.zeros(5)]), ([a.half()], None), ([a], [])):
        with pytest.raises(ValueError):
            eb.make_grads(*bad)
    assert ctypes.sizeof(eb.echo_grad_t) == 32 and ctypes.sizeof(eb.echo_vocab_desc_t) == 20
