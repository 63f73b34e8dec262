"""The vocabulary loss and its gradients against the float64 oracle.

Tolerances, for every entry, from the arithmetic.  u = 2^-24.
  z    is summed in fp32 over S = pairs x ceil(D / 16) matrix instructions, each of which rounds its own 16 products' sum and the running sum: at
       most 4 S u of sum_d |h W|; fp32 operands' six plane pairs leave out less than 4 u of it.              ->  ez(n, v)
  exp  the argument's product and difference round once each, the exponential is good to 2 u: (2 + 2 |argument|) u relative.
  lse  the largest ez of the row, the exponentials, sums over at most V terms in groups (a running sum of V / 64 + 80 terms), logarithm
       and two sums of fp32 numbers of the size of lse and of the label's logit.
  dz   p times (ez + e_lse + exponential), three roundings.  From bf16 storage it is fp16: one plane (bf16 gradients) rounds it by 2^-11, two
       (f32 gradients) by 2^-22.  It has 2^15 at p = 1 (for dh, dloss left out) or at least 2^14 at the largest dloss (for dW), and
       fp16's last place is 2^-24: one plane is off by up to 2^-40 of dloss, or 2^-39 of the largest dloss; the second plane holds 2^11 times
       what is left, to 2^-11 of that.  The other operand, scaled to at least 2^15, is off by at most 2^-40 of its largest value.
  dh   the errors of dz through |W|, and the sum's own 4 S u of sum |dz| |W|; the rounding of the result.  dW alike.
"""
import numpy as np
import pytest

from oracle import vocab_ref as vr

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _torch():
    import torch
    assert torch.cuda.is_available(), "needs the GPU"
    from paper_1805_08899_amd import binding as eb
    return torch, eb, {"f32": torch.float32, "bf16": torch.bfloat16}


def _guarded(torch, n_bytes, guard=256):
    whole = torch.full((n_bytes + 2 * guard + 16,), 0xFF, dtype=torch.uint8, device="cuda")
    inner = whole[guard:guard + n_bytes]

    def check():
        assert bool((whole[:guard] == 0xFF).all()) and bool((whole[guard + n_bytes:] == 0xFF).all()), "written outside its buffer"
    return inner, check


class Problem:
    def __init__(self, N, V, D, store="f32", out="f32", eps=0.0, pad=0.3, seed=0, scale=1.5):
        torch, eb, types = _torch()
        self.N, self.V, self.D, self.store, self.out, self.eps = N, V, D, store, out, eps
        r = np.random.default_rng(seed)
        W = r.standard_normal((V, D)) / np.sqrt(D)
        labels = np.minimum(np.exp(r.random(N) * np.log(V + 0.5)).astype(np.int64) - 1, V - 1)
        h = scale * r.standard_normal((N, D)) + r.random((N, 1)) * 12 * W[labels]
        none = r.random(N) < pad
        labels[none] = np.where(r.random(N) < 0.5, -1, V)[none]
        self.labels = labels.astype(np.int32)
        to = lambda x: torch.from_numpy(x.astype(np.float32)).to(types[store])
        self.h, self.W = to(h), to(W)
        self.dloss = torch.from_numpy(r.standard_normal(N).astype(np.float32))
        self.desc = eb.make_vocab_desc(N, V, D, store, out)

    def run(self, want_dh=True, want_dW=True, forward_only=False, h=None, stream=None):
        torch, eb, types = _torch()
        N, V, D, t = self.N, self.V, self.D, types[self.out]
        size = 4 if self.out == "f32" else 2
        bufs = {"loss": N * 4, "lse": N * 4, "dh": N * D * size, "dW": V * D * size,
                "ws_f": eb.echo_vocab_loss_fwd_workspace_bytes(self.desc), "ws_b": eb.echo_vocab_loss_bwd_workspace_bytes(self.desc)}
        b, checks = {}, []
        for k, n in bufs.items():
            b[k], c = _guarded(torch, n)
            checks.append(c)
        loss, lse = b["loss"].view(torch.float32), b["lse"].view(torch.float32)
        dh, dW = b["dh"].view(t).view(N, D), b["dW"].view(t).view(V, D)
        st = stream or torch.cuda.current_stream()
        x = (self.h if h is None else h).cuda(), self.W.cuda(), torch.from_numpy(self.labels).cuda()
        eb.check(eb.echo_vocab_loss_fwd(self.desc, *x, self.eps, loss, lse, b["ws_f"], stream=st))
        if not forward_only:
            eb.check(eb.echo_vocab_loss_bwd(self.desc, self.dloss.cuda(), lse, *x, self.eps, dh if want_dh else None,
                                            dW if want_dW else None, b["ws_b"], stream=st))
        torch.cuda.synchronize()
        for c in checks:
            c()
        r = {"loss": loss, "lse": lse}
        if not forward_only:
            r.update({k: x for k, x, w in (("dh", dh, want_dh), ("dW", dW, want_dW)) if w})
        return {k: x.double().cpu().numpy() for k, x in r.items()}

    def check(self, got):
        h, W = self.h.double().numpy(), self.W.double().numpy()
        V, D, eps, labels = self.V, self.D, self.eps, self.labels
        loss, lse = vr.loss_forward(h, W, labels, eps)
        rows = vr.labelled(labels, V)
        h_, y = h[rows], labels[rows]
        size = np.abs(h_) @ np.abs(W).T
        S = (6 if self.store == "f32" else 1) * -(-D // 16)
        ez = (4 * S + 4) * U * size
        z = h_ @ W.T
        worst, zy, ezy = ez.max(1, initial=0), z[np.arange(len(rows)), y], ez[np.arange(len(rows)), y]
        span = 2 + 2 * (z.max(1, initial=0) - z.min(1, initial=0)) if len(rows) else np.zeros(0)
        e_lse = worst + (np.minimum(span, 220) + V / 64 + 80) * U + 3 * U * (np.abs(lse[rows]) + np.abs(zy) + 1)
        e_loss = worst + ezy + e_lse + 3 * U * np.abs(loss[rows]) + eps * (worst + (V / 64 + 80) * U * np.abs(z).mean(1))
        for k, ref, e in (("lse", lse, e_lse), ("loss", loss, e_loss)):
            bound = np.zeros(self.N)
            bound[rows] = e
            assert (np.abs(got[k] - ref) <= bound).all(), (k, np.abs(got[k] - ref).max())
        if "dh" not in got and "dW" not in got:
            return
        dh, dW, dz = vr.loss_backward(self.dloss.double().numpy(), h, W, labels, eps)
        g = np.abs(self.dloss.double().numpy()[rows, None])
        p = np.exp(z - lse[rows, None])
        e_dz = g * (p * (ez + e_lse[:, None] + (4 + 2 * np.abs(z - lse[rows, None])) * U) + 3 * U) + 3 * U * np.abs(dz)
        planes, e_dh, e_dW = 3, 0.0, 0.0
        if self.store == "bf16" and len(rows):
            planes = 1 if self.out == "bf16" else 2
            e_dz = e_dz + 2.0 ** (-11 * planes) * np.abs(dz)
            low = 2.0 ** (11 - 11 * planes)
            e_dh = 2.0 ** -40 * (low * g * np.abs(W).sum(0) + np.abs(dz).sum(1, keepdims=True) * np.abs(W).max())
            e_dW = 2.0 ** -39 * low * g.max() * np.abs(h_).sum(0) + 2.0 ** -40 * np.abs(dz).sum(0)[:, None] * np.abs(h_).max()
        pairs = 6 if self.store == "f32" else planes
        half = 2.0 ** -8 if self.out == "bf16" else U
        if "dh" in got:
            bound = np.zeros_like(dh)
            bound[rows] = e_dz @ np.abs(W) + (4 * pairs * (V // 16 + 4) + 8) * U * (np.abs(dz) @ np.abs(W)) + half * np.abs(dh[rows]) + e_dh
            assert (np.abs(got["dh"] - dh) <= 1.01 * bound).all(), np.abs(got["dh"] - dh).max()
        if "dW" in got:
            bound = e_dz.T @ np.abs(h_) + (4 * pairs * (len(rows) // 16 + 4) + 8) * U * (np.abs(dz).T @ np.abs(h_)) + half * np.abs(dW) + e_dW
            assert (np.abs(got["dW"] - dW) <= 1.01 * bound).all(), np.abs(got["dW"] - dW).max()


CASES = [
    # N, V, D, storage, gradients, label smoothing
    (1, 1, 1, "f32", "f32", 0.0),
    (1, 2, 8, "bf16", "f32", 0.0),
    (1, 300, 64, "bf16", "bf16", 0.1),
    (3, 5, 7, "f32", "f32", 0.1),
    (5, 129, 9, "bf16", "bf16", 0.0),          # rows that no 16-byte load can take
    (31, 127, 63, "bf16", "f32", 0.3),
    (64, 128, 64, "f32", "f32", 0.0),
    (65, 257, 65, "f32", "f32", 0.0),
    (127, 1000, 72, "bf16", "bf16", 0.1),
    (128, 256, 512, "bf16", "f32", 0.0),
    (129, 2047, 100, "f32", "f32", 0.1),
    (200, 513, 520, "bf16", "f32", 0.0),
    (300, 3001, 1000, "bf16", "bf16", 0.1),
    (700, 1500, 260, "f32", "f32", 0.0),
    (2500, 70, 136, "bf16", "f32", 0.1),       # more rows than words
    (8, 2000, 16384, "f32", "f32", 0.0),       # words of f32 storage in two pieces; the widest rows
    (4100, 8200, 64, "bf16", "bf16", 0.1),     # tiles of 128 x 128 (those of 256 x 256: test_gpu_vocab_tiles.py)
    (4100, 11000, 40, "f32", "f32", 0.0),      # logits in tiles of 256 x 256, dz in two pieces
]
IDS = ["N%d_V%d_D%d_%s_%s_%g" % c for c in CASES]


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_against_the_oracle(case):
    print("vocab loss", case, flush=True)
    p = Problem(*case, seed=case[0] + case[1])
    p.check(p.run())


@pytest.mark.parametrize("store", ["f32", "bf16"])
@pytest.mark.parametrize("N", [2, 15, 16, 17, 32, 33, 48, 63, 64, 65, 127, 128, 129, 320, 383, 384, 385])
def test_forward_of_few_rows(N, store):
    """The words go straight to the matrix cores for few rows, in groups of 64: all ends of those, words that fill no block, widths that fill no step."""
    for V, D in ((1000, 72), (257, 1032), (64, 8), (4099, 4), (1, 40)):
        p = Problem(N, V, D, store, "f32", 0.1 if V > 300 else 0.0, seed=N + V)
        print("few rows", N, V, D, flush=True)
        p.check(p.run(forward_only=True))


@pytest.mark.parametrize("N", [2, 15, 17, 32, 33, 63, 64, 65, 129, 383, 384, 385])
def test_gradients_of_few_rows(N):
    """f32 rows straight to the matrix cores, as they are gathered: ends of groups and of their eights, one gradient alone."""
    for V, D, pad in ((1000, 72, 0.0), (257, 1032, 0.4), (64, 8, 0.9), (4099, 4, 0.2), (1, 40, 0.0)):
        p = Problem(N, V, D, "f32", "f32", 0.1 if V > 300 else 0.0, pad=pad, seed=N + V)
        print("few rows", N, V, D, flush=True)
        both = p.run()
        p.check(both)
        assert np.array_equal(p.run(want_dW=False)["dh"], both["dh"]) and np.array_equal(p.run(want_dh=False)["dW"], both["dW"])


@pytest.mark.parametrize("N,V,D", [(556, 2180, 936), (1500, 500, 256), (8192, 128, 64), (8193, 120, 32), (1100, 1000, 1024)])
def test_more_rows_of_few_words(N, V, D):
    """Where many groups of rows still make few blocks."""
    for store in ("f32", "bf16"):
        p = Problem(N, V, D, store, "f32", 0.1, seed=N + 1)
        p.check(p.run())


def test_gradients_of_few_rows_in_pieces():
    """Words turned in pieces of 512 MB: 5460 words of the widest rows."""
    p = Problem(70, 6000, 16384, "f32", "f32", 0.1, seed=50)
    p.check(p.run())


@pytest.mark.parametrize("types", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")], ids="_".join)
@pytest.mark.parametrize("N,V,D,pad", [(9000, 40, 72, 0.1), (20, 30000, 64, 0.0), (5, 20011, 520, 0.0), (3000, 9001, 36, 0.99), (700, 700, 1000, 0.5),
                                       (3000, 300, 68, 1.0)])
def test_gradients_cut_along_either_axis(N, V, D, pad, types):
    """Many rows and few words and the other way round: sums in up to 64 parts; rows of which few or none have a label."""
    p = Problem(N, V, D, *types, 0.1, pad=pad, seed=N)
    p.check(p.run())


@pytest.mark.parametrize("store", ["f32", "bf16"])
def test_no_row_has_a_label(store):
    p = Problem(40, 300, 64, store, "f32", 0.1, pad=1.1)
    p.labels[:] = -1
    p.labels[::3] = 300
    got = p.run()
    for k, x in got.items():
        assert not x.any(), k


def test_rows_without_a_label_may_hold_anything():
    torch, eb, types = _torch()
    p = Problem(150, 300, 72, "f32", "f32", 0.1, pad=0.5, seed=3)
    none = (p.labels < 0) | (p.labels >= 300)
    clean = p.run()
    p.h[torch.from_numpy(none)] = float("nan")
    p.dloss[torch.from_numpy(none)] = float("inf")
    got = p.run()
    for k in clean:
        assert np.array_equal(got[k], clean[k]), k


@pytest.mark.parametrize("scale", [0.0, 60.0, 1000.0])
def test_flat_and_steep_logits(scale):
    p = Problem(90, 400, 48, "f32", "f32", 0.1, seed=4, scale=scale)
    p.check(p.run())


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("power", [0, 60, -60])
def test_bf16_operands_and_dloss_of_any_size(power, out):
    """h up, W down by a power of two leave the logits as they are; the dloss of neighbouring rows differ by up to 2^60."""
    torch, eb, types = _torch()
    p = Problem(300, 900, 136, "bf16", out, 0.1, seed=12)
    p.dloss *= torch.exp2(torch.randint(-30, 31, (300,), generator=torch.Generator().manual_seed(13)).float())
    p.h, p.W = p.h * 2.0 ** power, p.W * 2.0 ** -power
    p.check(p.run())


@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_bf16_operands_and_a_dloss_far_below_another(out):
    """2^-34 of it, in a word to which the other row gives nothing: dz in fp16 has 2^-20 there, in steps of 2^-24."""
    torch, eb, types = _torch()
    p = Problem(2, 64, 64, "bf16", out, 0.0, pad=0.0, seed=15)
    p.W[:] = torch.eye(64)
    p.h[:] = 0.0
    p.h[0, 0], p.h[1, 1:] = 120.0, -1.0
    p.labels[:] = (0, 1)
    p.dloss[:] = torch.tensor([1.0, 2.0 ** -34])
    got = p.run()
    p.check(got)
    assert got["dW"][1].any()


def test_two_planes_of_a_dz_add_up():
    """Few rows, so that one product with a plane off by a place of fp16 (2^-11) stands out of a word's sum; many words, since only a dz within
    fp32's rounding of halfway between two fp16 numbers (one in 2^13) could be taken for either."""
    for seed in range(12):
        p = Problem(4, 20000, 16, "bf16", "f32", 0.0, pad=0.0, seed=40 + seed, scale=0.5)
        p.W *= 0.25
        h, W = p.h.double().numpy(), p.W.double().numpy()
        got = p.run(want_dh=False)
        # from the lse that was found, so that its error, which all words share, is none of this test's
        z = h @ W.T
        q = np.exp(z - got["lse"][:, None])
        dz = p.dloss.double().numpy()[:, None] * (q - (p.labels[:, None] == np.arange(20000)))
        size = np.abs(dz).T @ np.abs(h)
        # z: S = 1; exp: its argument is at most 16 here; dz: three roundings and the planes; the sum: two pairs of one step, the scaling
        e = 12 * U * (np.abs(h) @ np.abs(W).T).max() + 40 * U + 3 * U + 2.0 ** -22 + 20 * U
        assert np.abs(z).max() < 6 and (np.abs(got["dW"] - dz.T @ h) <= e * size + 3 * U * np.abs(p.dloss.numpy()).max() * (p.labels[:, None] == np.arange(20000)).T @ np.abs(h)
                + 2.0 ** -50 * np.abs(h).sum(0)).all(), seed


@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_bf16_rows_without_a_label_do_not_reach_the_gradients(out):
    torch, eb, types = _torch()
    p = Problem(150, 300, 72, "bf16", out, 0.1, pad=0.5, seed=3)
    none = torch.from_numpy((p.labels < 0) | (p.labels >= 300))
    clean = p.run()
    for h, g in ((float("nan"), float("inf")), (1e30, 1e30), (float("inf"), float("nan"))):
        p.h[none], p.dloss[none] = h, g
        got = p.run()
        for k in clean:
            assert np.array_equal(got[k], clean[k]), k


def test_bf16_gradients_of_nothing():
    """dloss of zero everywhere, then words and rows of zeros."""
    p = Problem(100, 260, 64, "bf16", "bf16", 0.0, seed=14)
    p.dloss.zero_()
    got = p.run()
    assert not got["dh"].any() and not got["dW"].any()
    p = Problem(100, 260, 64, "bf16", "bf16", 0.0, seed=14)
    p.h.zero_()
    p.W.zero_()
    got = p.run()
    assert not got["dh"].any() and not got["dW"].any()


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [60.0, 1000.0])
def test_steep_logits_of_bf16_operands(scale, out):
    p = Problem(90, 400, 48, "bf16", out, 0.1, seed=4, scale=scale)
    p.check(p.run())


def test_a_sure_label_keeps_the_digits_of_its_loss():
    """Losses of 1e-5 from logits of 20: the difference of lse and the label's logit would have errors of 1e-6."""
    torch, eb, types = _torch()
    N, V, D = 64, 1000, 32
    p = Problem(N, V, D, "f32", "f32", 0.0, pad=0.0, seed=5, scale=0.0)
    p.h.zero_()
    p.h[:, 0] = 20.0
    p.labels[:] = np.arange(N)
    for n in range(3):                                    # one word above the others in turn
        p.W.zero_()
        p.W[:, 0] = 1.0
        p.W[n, 0] = 2.0
        got = p.run(forward_only=True)["loss"][n]
        ref = vr.loss_forward(p.h.numpy(), p.W.numpy(), p.labels, 0.0)[0][n]
        assert abs(got - ref) <= 300 * U * ref


@pytest.mark.parametrize("store", ["f32", "bf16"])
def test_infinities_and_nan_reach_their_row(store):
    torch, eb, types = _torch()
    p = Problem(100, 200, 64, store, "f32", 0.0, pad=0.0, seed=6)
    clean = p.run(forward_only=True)
    p.h[17, 3] = float("nan")
    p.h[80, 5] = float("inf")
    got = p.run(forward_only=True)
    bad = np.zeros(100, bool)
    bad[[17, 80]] = True
    assert not np.isfinite(got["loss"][bad]).any()
    assert np.array_equal(got["loss"][~bad], clean["loss"][~bad])


def test_one_gradient_alone():
    for store, out in (("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")):
        p = Problem(140, 333, 80, store, out, 0.1, seed=7)
        both = p.run()
        assert np.array_equal(p.run(want_dW=False)["dh"], both["dh"])
        assert np.array_equal(p.run(want_dh=False)["dW"], both["dW"])


@pytest.mark.parametrize("store,out", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
def test_bit_identical_from_run_to_run(store, out):
    p = Problem(1000, 3000, 128, store, out, 0.1, seed=8)
    a, b = p.run(), p.run()
    for k in a:
        assert np.array_equal(a[k], b[k]), k


def test_gradient_is_the_difference_of_losses():
    """Central differences along a direction u: sum_n dloss (L(h + s u) - L(h - s u)) / 2 s against <dh, u>.  Bound: the losses'
    own errors over s, and what central differences of this step leave out, taken from the oracle."""
    torch, eb, types = _torch()
    p = Problem(60, 500, 40, "f32", "f32", 0.1, seed=9)
    u = torch.from_numpy(np.random.default_rng(10).standard_normal((60, 40)).astype(np.float32))
    s = 2.0 ** -6
    dloss, W = p.dloss.double().numpy(), p.W.double().numpy()
    diff, exact = [], []
    for sign in (1, -1):
        h = (p.h + sign * s * u)
        diff.append((dloss * p.run(forward_only=True, h=h)["loss"]).sum())
        exact.append((dloss * vr.loss_forward(h.double().numpy(), W, p.labels, 0.1)[0]).sum())
    got = (p.run()["dh"] * u.double().numpy()).sum()
    formula = (vr.loss_backward(dloss, p.h.double().numpy(), W, p.labels, 0.1)[0] * u.double().numpy()).sum()
    left_out = abs((exact[0] - exact[1]) / (2 * s) - formula)
    size = (np.abs(p.h.numpy()) @ np.abs(W).T).max()
    e_loss = 2 * (4 * 6 * 3 + 4) * U * size + 300 * U + 10 * U * 20
    assert abs((diff[0] - diff[1]) / (2 * s) - got) <= left_out + 2 * np.abs(dloss).sum() * e_loss / s


def test_replayed_from_a_graph_and_on_another_stream():
    torch, eb, types = _torch()
    N, V, D = 300, 700, 64
    desc = eb.make_vocab_desc(N, V, D, "bf16", "f32")
    h, W = torch.randn(N, D, device="cuda").bfloat16(), (torch.randn(V, D, device="cuda") / 8).bfloat16()
    labels = torch.randint(-1, V, (N,), device="cuda").int()
    dloss = torch.rand(N, device="cuda")
    outs = [torch.empty(N, device="cuda"), torch.empty(N, device="cuda"), torch.empty(N, D, device="cuda"), torch.empty(V, D, device="cuda")]
    ws = torch.empty(max(eb.echo_vocab_loss_fwd_workspace_bytes(desc), eb.echo_vocab_loss_bwd_workspace_bytes(desc)), dtype=torch.uint8,
                     device="cuda")

    def step():
        st = torch.cuda.current_stream()
        eb.check(eb.echo_vocab_loss_fwd(desc, h, W, labels, 0.1, outs[0], outs[1], ws, stream=st))
        eb.check(eb.echo_vocab_loss_bwd(desc, dloss, outs[1], h, W, labels, 0.1, outs[2], outs[3], ws, stream=st))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        labels.copy_(torch.randint(-1 if k else -V, V, (N,), device="cuda"))   # another number of rows each time
        h.copy_(torch.randn(N, D, device="cuda"))
        step()
        torch.cuda.synchronize()
        want = [x.clone() for x in outs]
        for x in outs:
            x.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), k


@pytest.mark.parametrize("store,out", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("scale", [1e6, 1e9])
def test_logits_whose_rounding_is_larger_than_one(store, out, scale):
    """The forward pass and the backward pass add a logit's products in another order."""
    p = Problem(64, 3000, 264, store, out, 0.1, pad=0.1, seed=35, scale=scale)
    got = p.run()
    g = np.abs(p.dloss.double().numpy())
    for k in ("loss", "lse", "dh", "dW"):
        assert np.isfinite(got[k]).all(), k
    assert (np.abs(got["dh"]) <= 1.02 * g[:, None] * 3001 * np.abs(p.W.double().numpy()).max()).all()


def test_two_calls_at_once_with_workspaces_of_their_own():
    torch, eb, types = _torch()
    ps = [Problem(1500, 4000, 128, "bf16", out, 0.1, seed=36) for out in ("f32", "bf16")]
    want = [p.run() for p in ps]
    streams, all_out = [torch.cuda.Stream() for _ in ps], []
    for p, out in zip(ps, ("f32", "bf16")):
        x = p.h.cuda(), p.W.cuda(), torch.from_numpy(p.labels).cuda()
        o = [torch.empty(1500, device="cuda"), torch.empty(1500, device="cuda"), torch.empty(1500, 128, dtype=types[out], device="cuda"),
             torch.empty(4000, 128, dtype=types[out], device="cuda")]
        ws = [torch.empty(f(p.desc), dtype=torch.uint8, device="cuda") for f in (eb.echo_vocab_loss_fwd_workspace_bytes, eb.echo_vocab_loss_bwd_workspace_bytes)]
        all_out.append((x, p.dloss.cuda(), o, ws))
    torch.cuda.synchronize()
    for _ in range(5):
        for p, st, (x, g, o, ws) in zip(ps, streams, all_out):
            eb.check(eb.echo_vocab_loss_fwd(p.desc, *x, 0.1, o[0], o[1], ws[0], stream=st))
            eb.check(eb.echo_vocab_loss_bwd(p.desc, g, o[1], *x, 0.1, o[2], o[3], ws[1], stream=st))
    torch.cuda.synchronize()
    for w, (x, g, o, ws) in zip(want, all_out):
        for k, got in zip(("loss", "lse", "dh", "dW"), o):
            assert np.array_equal(got.double().cpu().numpy(), w[k]), k


def _zeros_but(torch, rows, width, filled):
    x = torch.zeros(rows, width, dtype=torch.bfloat16, device="cuda")
    for at, value in filled.items():
        x[at] = torch.from_numpy(value.astype(np.float32)).bfloat16()
    return x


@pytest.mark.parametrize("N", [3, 70])
def test_words_past_32_bits(N):
    """4.4 GB of words of zeros but two: the others all have a logit of zero."""
    torch, eb, types = _torch()
    V, D = 270000, 8192
    r = np.random.default_rng(31)
    words = {V - 1: r.standard_normal(D) / 64, 7: r.standard_normal(D) / 64}
    W = _zeros_but(torch, V, D, words)
    h = torch.from_numpy(r.standard_normal((N, D)).astype(np.float32)).bfloat16().cuda()
    labels = torch.tensor([(V - 1, 7, V - 2)[n % 3] for n in range(N)], dtype=torch.int32, device="cuda")
    desc = eb.make_vocab_desc(N, V, D, "bf16", "bf16")
    loss, lse, dloss = torch.empty(N, device="cuda"), torch.empty(N, device="cuda"), torch.rand(N, device="cuda") + 0.5
    dh, dW = torch.empty(N, D, dtype=torch.bfloat16, device="cuda"), torch.full((V, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(max(eb.echo_vocab_loss_fwd_workspace_bytes(desc), eb.echo_vocab_loss_bwd_workspace_bytes(desc)), dtype=torch.uint8, device="cuda")
    st = torch.cuda.current_stream()
    eb.check(eb.echo_vocab_loss_fwd(desc, h, W, labels, 0.0, loss, lse, ws, stream=st))
    eb.check(eb.echo_vocab_loss_bwd(desc, dloss, lse, h, W, labels, 0.0, dh, dW, ws, stream=st))
    torch.cuda.synchronize()
    kept = [7, V - 1, V - 2, 0]
    h_, W_, g, y = (x.double().cpu().numpy() for x in (h, W[kept], dloss, labels))
    z = h_ @ W_.T
    ref = np.log(np.exp(z[:, :2]).sum(1) + V - 2)
    size = np.abs(h_) @ np.abs(W_).T
    e = (4 * D // 16 + 4) * U * size.max() + 400 * U + (V / 64 + 80) * U      # ez, the exponentials' arguments, the sums
    assert np.abs(lse.cpu().numpy() - ref).max() <= e
    zy = np.where(y == V - 1, z[:, 1], np.where(y == 7, z[:, 0], 0.0))
    assert np.abs(loss.cpu().numpy() - (ref - zy)).max() <= 2 * e
    dz = g[:, None] * (np.exp(z - ref[:, None]) - (y[:, None] == np.array(kept)))
    want = dz.T @ h_
    bound = (2.0 ** -8 + 1e-5) * np.abs(want) + (2.0 ** -11 + 3 * e) * (np.abs(dz).T @ np.abs(h_))
    assert (np.abs(dW[kept].double().cpu().numpy() - want) <= bound).all()
    assert bool(torch.isfinite(dW[1000]).all()) and bool(torch.isfinite(dW[V // 2]).all())
    want = dz[:, :2] @ W_[:2]                                # (the other words are zeros)
    bound = (2.0 ** -8 + 1e-5) * np.abs(want) + (2.0 ** -11 + 3 * e) * (np.abs(dz[:, :2]) @ np.abs(W_[:2]))
    assert (np.abs(dh.double().cpu().numpy() - want) <= bound).all()


@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_more_words_than_32_bit_offsets_of_rows_of_dz(out):
    """A row of dz of 4.5 million words; its 255 neighbours begin past 2^31 bytes."""
    torch, eb, types = _torch()
    N, V, D = 3, 4500003, 8
    p = Problem(N, V, D, "bf16", out, 0.0, pad=0.0, seed=33)
    p.check(p.run())


@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_more_rows_than_32_bit_offsets_of_words_of_dz(out):
    """The same of 4.5 million rows, most of them without a label: turned, dz has a row of them per word."""
    torch, eb, types = _torch()
    N, V, D = 4500003, 300, 8
    p = Problem(N, 300, D, "bf16", out, 0.0, pad=0.999, seed=34)
    p.check(p.run())
