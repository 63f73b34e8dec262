"""Every tile kernel of the vocabulary loss, by the names of the launches: which rows and words take 128 x 128 or 256 x 256 tiles, or go straight to
the matrix cores, is decided by rules of the time they take, so that a test's sizes alone do not say what it runs.  Tolerances: test_gpu_vocab_loss.py."""
import numpy as np
import pytest

from test_gpu_vocab_loss import Problem, _torch

pytestmark = pytest.mark.gpu

CASES = [
    # N, V, D, storage, gradients, label smoothing, share of rows without a label, tile of: logits, dz, gradients.  All have several row tiles and
    # k axes of several steps of 64 and a rest.
    (1500, 6000, 136, "f32", "f32", 0.1, 0.3, 256, 256, 256),
    (1500, 9001, 200, "f32", "f32", 0.0, 0.3, 256, 256, 256),
    (5000, 9100, 136, "f32", "f32", 0.1, 0.6, 256, 128, 256),         # two pieces of the vocabulary
    (2000, 4000, 520, "f32", "f32", 0.1, 0.2, 128, 128, 128),
    (900, 2003, 129, "f32", "f32", 0.0, 0.1, 128, 128, 128),          # rows that no 16-byte load can take
    (1000, 9001, 520, "bf16", "f32", 0.1, 0.2, 256, 256, 256),
    (20000, 6000, 200, "bf16", "f32", 0.1, 0.85, 256, 256, 256),      # two pieces
    (1300, 2500, 130, "bf16", "f32", 0.0, 0.1, 128, 128, 128),        # rows that no 16-byte load can take
    (1000, 9001, 520, "bf16", "bf16", 0.0, 0.2, 256, 256, 256),
    (16000, 9001, 136, "bf16", "bf16", 0.1, 0.85, 256, 256, 256),     # two pieces
    (1500, 9001, 200, "bf16", "bf16", 0.1, 0.3, 256, 256, 128),
    (1300, 2500, 130, "bf16", "bf16", 0.1, 0.1, 128, 128, 128),
]
IDS = ["N%d_V%d_D%d_%s_%s" % c[:5] for c in CASES]


def _launches(p, **kw):
    torch, eb, types = _torch()
    eb.echo_attn_profile_enable(True)
    try:
        eb.echo_attn_profile_read()
        got = p.run(**kw)
        names = eb.echo_attn_profile_read()
    finally:
        eb.echo_attn_profile_enable(False)
    return got, names


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_tiles_against_the_oracle(case):
    N, V, D, store, out, eps, pad, logits, dlogits, grads = case
    print("tiles", case, flush=True)
    p = Problem(N, V, D, store, out, eps, pad=pad, seed=N + D)
    got, names = _launches(p)
    tiles = {n.rsplit("_", 1)[0]: int(n.rsplit("_", 1)[1]) for n in names if n.endswith(("_128", "_256"))}
    assert tiles == {"vocab_logits": logits, "vocab_dlogits": dlogits, "vocab_grads": grads}, names
    p.check(got)
    assert np.array_equal(p.run(want_dW=False)["dh"], got["dh"]) and np.array_equal(p.run(want_dh=False)["dW"], got["dW"])


@pytest.mark.parametrize("case", [CASES[i] for i in (0, 4, 5, 7, 8, 11)], ids=[IDS[i] for i in (0, 4, 5, 7, 8, 11)])
def test_infinities_and_nan_reach_their_rows(case):
    """In labelled rows: NaN and an infinity in h, in dloss.  Such a row's loss, lse and dh are not finite and no entry of dW is; what the other rows get is, bit
    for bit, what they get beside rows of other numbers."""
    torch, eb, types = _torch()
    N, V, D, store, out, eps, pad, logits, dlogits, grads = case
    p = Problem(N, V, D, store, out, eps, pad=pad, seed=N + V)
    rows = np.flatnonzero((p.labels >= 0) & (p.labels < V))
    clean, names = _launches(p)
    assert {"vocab_logits_%d" % logits, "vocab_dlogits_%d" % dlogits, "vocab_grads_%d" % grads} <= set(names)
    bad = rows[[0, 200, 300, len(rows) - 1]]
    others = np.setdiff1d(np.arange(N), bad)
    for what in ("h", "dloss"):
        for value in (np.nan, np.inf):
            q = Problem(N, V, D, store, out, eps, pad=pad, seed=N + V)
            if what == "h":
                q.h[bad, 3] = value
            else:
                q.dloss[bad] = value
            got = q.run()
            for k in ("loss", "lse", "dh"):
                assert np.array_equal(got[k][others], clean[k][others]), (what, value, k)
            if what == "h":
                assert not np.isfinite(got["loss"][bad]).any()
            else:
                assert np.array_equal(got["loss"], clean["loss"])
            assert not np.isfinite(got["dh"][bad]).any(), (what, value)
            assert not np.isfinite(got["dW"]).any(), (what, value)


@pytest.mark.parametrize("store,out", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
def test_bit_identical_from_run_to_run_in_large_tiles(store, out):
    p = Problem(1500, 6000, 136, store, out, 0.1, seed=8)
    (a, names), b = _launches(p), p.run()
    assert "vocab_logits_256" in names and "vocab_dlogits_256" in names
    for k in a:
        assert np.array_equal(a[k], b[k]), k
