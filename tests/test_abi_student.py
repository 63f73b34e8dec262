"""Refusals of the recurrence, the distillation and the verification, without a GPU: every call stops at a host check."""
import ctypes

import pytest

from paper_1805_08899_amd import binding as eb
from test_abi_index_types import FORMS

A = 0x10000  # a fake, aligned, never dereferenced device address
BIG = 1 << 60


def _call(name, **given):
    def call(desc, m=eb, **kw):
        return getattr(m, name)(desc, **{**given, **kw})
    return call


scan = lambda: eb.make_scan_desc(3, 5, 7)
vocab = lambda: eb.make_vocab_desc(6, 7, 8)
draft = lambda: eb.make_draft_desc(3, 4, 9)
CALLS = {
    # call, a good descriptor, pointers that may not be NULL, those that may
    "scan_fwd": (_call("echo_scan_fwd", G=A, c0=A, len=A, h=A, c_last=A, states=A, workspace=A, workspace_bytes=BIG), scan,
                 ("G", "h"), ("c0", "len", "c_last", "states")),
    "scan_bwd": (_call("echo_scan_bwd", dh=A, dc_last=A, G=A, len=A, states=A, dG=A, dc0=A, workspace=A, workspace_bytes=BIG), scan,
                 ("dh", "G", "states", "dG"), ("dc_last", "len", "dc0")),
    "distill_fwd": (_call("echo_distill_fwd", h=A, W=A, words=A, logits=A, K=3, T=2.0, loss=A, lse=A, workspace=A, workspace_bytes=BIG), vocab,
                    ("h", "W", "words", "logits", "loss", "lse", "workspace"), ()),
    "distill_bwd": (_call("echo_distill_bwd", dloss=A, lse=A, h=A, W=A, words=A, logits=A, K=3, T=2.0, dh=A, dW=A, workspace=A, workspace_bytes=BIG),
                    vocab, ("dloss", "lse", "h", "W", "words", "logits", "workspace"), ("dh", "dW")),
    "verify": (_call("echo_draft_verify", drafted=A, n_drafted=A, draft=A, target=A, u=A, r=A, tokens=A, taken=A, workspace=A, workspace_bytes=BIG),
               draft, ("drafted", "draft", "target", "u", "r", "tokens", "taken"), ("n_drafted",)),
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_pointers(name):
    call, good, needed, optional = CALLS[name]
    for p in needed:
        assert call(good(), **{p: None}) == eb.ECHO_ERR_NULL, p
    for p in needed + optional:
        assert call(good(), **{p: A + 4}) == eb.ECHO_ERR_ALIGN, p
    for p in optional:                                    # taken, and then stopped behind it
        assert call(good(), **{p: None, needed[0]: None}) == eb.ECHO_ERR_NULL, p
    assert call(good(), workspace=A + 8) == eb.ECHO_ERR_ALIGN
    with pytest.raises(TypeError):
        call(eb.make_desc(1, 1, 1, 1, 4))
    with pytest.raises(TypeError):
        call(good(), nonsense=1)


LIMITS = {
    "scan_fwd": {"B": eb.ECHO_SCAN_MAX_ROWS, "T": eb.ECHO_SCAN_MAX_ROWS, "H": eb.ECHO_SCAN_MAX_H},
    "distill_fwd": {"N": eb.ECHO_VOCAB_MAX_ROWS, "V": eb.ECHO_VOCAB_MAX_ROWS, "D": eb.ECHO_VOCAB_MAX_D},
    "verify": {"B": eb.ECHO_DRAFT_MAX_B, "K": eb.ECHO_DRAFT_MAX_K, "V": eb.ECHO_DRAFT_MAX_V},
}
LIMITS["scan_bwd"], LIMITS["distill_bwd"] = LIMITS["scan_fwd"], LIMITS["distill_fwd"]


@pytest.mark.parametrize("name", sorted(CALLS))
def test_limits_and_types(name):
    call, good, needed, _ = CALLS[name]
    for field, limit in LIMITS[name].items():
        for value in (0, -1, limit + 1, -2 ** 31):
            d = good()
            setattr(d, field, value)
            assert call(d) == eb.ECHO_ERR_SHAPE, (field, value)
        d = good()
        setattr(d, field, limit)
        assert call(d, **{needed[0]: None}) == eb.ECHO_ERR_NULL, (field, limit)
    for field in ("dtype",) if name in ("scan_fwd", "scan_bwd", "verify") else ("in_dtype", "out_dtype"):
        for value in (-1, 2):
            d = good()
            setattr(d, field, value)
            assert call(d) == eb.ECHO_ERR_DTYPE, (field, value)


def test_other_refusals():
    for name in ("scan_fwd", "scan_bwd"):
        for value in (-1, 2):
            d = scan()
            d.reverse = value
            assert CALLS[name][0](d) == eb.ECHO_ERR_SHAPE
        assert CALLS[name][0](eb.make_scan_desc(1 << 24, 1 << 16, 2)) == eb.ECHO_ERR_SHAPE
    for name in ("distill_fwd", "distill_bwd"):
        call = CALLS[name][0]
        for K in (0, -1, eb.ECHO_DISTILL_MAX_K + 1):
            assert call(vocab(), K=K) == eb.ECHO_ERR_SHAPE, K
        for T in (0.0, -1.0, float("nan"), float("inf"), 2.0 ** -65, 2.0 ** 65):
            assert call(vocab(), T=T) == eb.ECHO_ERR_SHAPE, T
        assert call(eb.make_vocab_desc(6, 7, 8, "f32", "bf16")) == eb.ECHO_ERR_DTYPE
    assert CALLS["distill_bwd"][0](vocab(), dh=None, dW=None) == eb.ECHO_ERR_NULL


def test_workspaces():
    d = eb.make_vocab_desc(50, 700, 90)
    for query, name, vocab_query in ((eb.echo_distill_fwd_workspace_bytes, "distill_fwd", eb.echo_vocab_loss_fwd_workspace_bytes),
                                     (eb.echo_distill_bwd_workspace_bytes, "distill_bwd", eb.echo_vocab_loss_bwd_workspace_bytes)):
        need = query(d, 9)
        assert need > vocab_query(d) and CALLS[name][0](d, K=9, workspace_bytes=need - 1) == eb.ECHO_ERR_WORKSPACE
        assert query(d, 0) == query(d, 129) == query(eb.make_vocab_desc(0, 7, 8), 9) == 0
        # a hundredth of the logits' size for the lists
        big = eb.make_vocab_desc(16384, 131072, 1024, "bf16", "f32")
        assert query(big, 64) - vocab_query(big) < 4 * 16384 * 131072 // 100
        most = eb.make_vocab_desc(eb.ECHO_VOCAB_MAX_ROWS, eb.ECHO_VOCAB_MAX_ROWS, eb.ECHO_VOCAB_MAX_D)
        assert query(most, 128) > 1 << 40
    for d in (scan(), eb.make_scan_desc(2, 1000, 70, "bf16")):
        for query, name in ((eb.echo_scan_fwd_workspace_bytes, "scan_fwd"), (eb.echo_scan_bwd_workspace_bytes, "scan_bwd")):
            need = query(d)
            if need:
                assert CALLS[name][0](d, workspace_bytes=need - 1) == eb.ECHO_ERR_WORKSPACE
                assert CALLS[name][0](d, workspace=None) == eb.ECHO_ERR_NULL
        assert eb.echo_scan_states_bytes(d) == d.B * -(-d.T // eb.ECHO_SCAN_CHUNK) * d.H * 4
    for d in (draft(), eb.make_draft_desc(1, 4, 100000)):
        need = eb.echo_draft_verify_workspace_bytes(d)
        if need:
            assert CALLS["verify"][0](d, workspace_bytes=need - 1) == eb.ECHO_ERR_WORKSPACE
            assert CALLS["verify"][0](d, workspace=None) == eb.ECHO_ERR_NULL
    L = eb.lib()
    for f in (L.echo_scan_states_bytes, L.echo_scan_fwd_workspace_bytes, L.echo_scan_bwd_workspace_bytes, L.echo_draft_verify_workspace_bytes):
        assert f(None) == 0
    assert L.echo_distill_fwd_workspace_bytes(None, 3) == 0 and L.echo_distill_bwd_workspace_bytes(None, 3) == 0
    assert eb.echo_scan_states_bytes(eb.make_scan_desc(0, 1, 1)) == 0
    assert L.echo_scan_fwd(None, *[A] * 7, BIG, None) == eb.ECHO_ERR_NULL and L.echo_scan_bwd(None, *[A] * 8, BIG, None) == eb.ECHO_ERR_NULL
    assert L.echo_draft_verify(None, *[A] * 9, BIG, None) == eb.ECHO_ERR_NULL
    assert ctypes.sizeof(eb.echo_scan_desc_t) == 20 and ctypes.sizeof(eb.echo_draft_desc_t) == 16


@pytest.mark.parametrize("form", sorted(FORMS))
def test_index_tensors(form):
    """Lengths and words are int32 tensors of at least as many numbers as the call reads."""
    import torch
    m = FORMS[form]()
    # descriptors of the form's own module; the first pointer is NULL, so that a taken tensor ends in an error
    s, v, d = m.make_scan_desc(3, 5, 7), m.make_vocab_desc(3, 7, 8), m.make_draft_desc(3, 4, 9)
    arguments = {
        "scan_fwd": ("len", 3, s, dict(G=None)), "scan_bwd": ("len", 3, s, dict(dh=None)),
        "distill_fwd": ("words", 12, v, dict(h=None, K=4)), "distill_bwd": ("words", 12, v, dict(dloss=None, K=4)),
        "verify": ("drafted", 12, d, dict(draft=None)), "verify ": ("n_drafted", 3, d, dict(draft=None)),
    }
    for name, (argument, count, desc, null) in arguments.items():
        call = CALLS[name.strip()][0]
        for x in (torch.zeros(count, dtype=torch.int32), torch.zeros(2, count, dtype=torch.int32), A):
            assert call(desc, m, **null, **{argument: x}) == eb.ECHO_ERR_NULL, name
        for x in (torch.zeros(count, dtype=torch.int64), torch.zeros(count), torch.zeros(count - 1, dtype=torch.int32),
                  torch.zeros(2 * count, dtype=torch.int32)[::2]):
            with pytest.raises(ValueError):
                call(desc, m, **null, **{argument: x})
                pytest.fail(f"{name} took {x.dtype}, {tuple(x.shape)}")
    for K in (0, -1, 129):                                # refused by the library, not by the size of the tensor
        assert CALLS["distill_fwd"][0](v, m, K=K, words=torch.zeros(3 * 129, dtype=torch.int32)) == eb.ECHO_ERR_SHAPE
