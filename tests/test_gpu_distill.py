"""The distillation from a teacher's top logits and its gradients against the float64 oracle.

Tolerances, for every value, from the arithmetic; u = 2^-24.  What is the vocabulary loss's (test_gpu_vocab_loss.py): a logit is off by ez(n, v), plus u of it from
the temperature (divided by it: ez / T); lse, dz's planes and the gradients' sums as there, with T dloss in the place of dloss.  What is new:
  q     its argument (t - max) / T is rounded twice, the exponential is good to 2 u, the sum of K and the quotient to (K + 3) u; shares of one word
        add up with as many roundings as there are of them:               eq <= q (2 |x| + 2 K + 8) u
  own   sum q log q: eq |log q| + q u (3 |x| + 3 |log sum| + K)           with |x|, |log sum| <= |log q| + log K
  mean  sum q z, tile by tile (V / 64 + 80 terms, as for lse):             sum (eq |z| + q ez + (V / 64 + 80 + 4) u q |z|)
  loss  T^2 times own, lse and mean, three roundings."""
import numpy as np
import pytest

from oracle import student_ref as sr
from test_gpu_scan import Buffers, _torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


class Problem:
    def __init__(self, N, V, D, K, store="f32", out="f32", T=1.0, pad=0.3, seed=0, scale=1.5, twice=0.1):
        torch, eb, types = _torch()
        self.N, self.V, self.D, self.K, self.store, self.out, self.T = N, V, D, K, store, out, T
        r = np.random.default_rng(seed)
        W = r.standard_normal((V, D)) / np.sqrt(D)
        words = r.integers(0, V, (N, K))
        words[:, 1:][r.random((N, K - 1)) < twice] = words[0, 0]       # words more than once
        h = scale * r.standard_normal((N, D)) + r.random((N, 1)) * 12 * W[words[:, 0]]
        words[r.random((N, K)) < 0.1] = -1
        words[r.random((N, K)) < 0.05] = V
        words[r.random(N) < pad] = -1
        logits = 8 * r.random((N, 1)) - 3 * r.random((N, K)) * np.arange(K)
        logits[r.random((N, K)) < 0.05] = -np.inf
        self.words, to = words.astype(np.int32), lambda x: torch.from_numpy(x.astype(np.float32))
        self.logits, self.dloss = to(logits), to(r.standard_normal(N))
        self.h, self.W = to(h).to(types[store]), to(W).to(types[store])
        self.desc = eb.make_vocab_desc(N, V, D, store, out)

    def rows(self):
        return {n: rest for n, *rest in sr.teacher_rows(self.words, self.logits.numpy(), self.V, self.T)}

    def run(self, want_dh=True, want_dW=True, forward_only=False, stream=None):
        torch, eb, types = _torch()
        N, V, D, K, t, b = self.N, self.V, self.D, self.K, types[self.out], Buffers(torch)
        loss, lse = b.of(torch.float32, N), b.of(torch.float32, N)
        st = stream or torch.cuda.current_stream()
        x = self.h.cuda(), self.W.cuda(), torch.from_numpy(self.words).cuda(), self.logits.cuda()
        eb.check(eb.echo_distill_fwd(self.desc, *x, K, self.T, loss, lse, b.bytes(eb.echo_distill_fwd_workspace_bytes(self.desc, K)), stream=st))
        r = {"loss": loss, "lse": lse}
        if not forward_only:
            if want_dh:
                r["dh"] = b.of(t, N, D)
            if want_dW:
                r["dW"] = b.of(t, V, D)
            eb.check(eb.echo_distill_bwd(self.desc, self.dloss.cuda(), lse, *x, K, self.T, r.get("dh"), r.get("dW"),
                                         b.bytes(eb.echo_distill_bwd_workspace_bytes(self.desc, K)), stream=st))
        torch.cuda.synchronize()
        b.check()
        return {k: v.double().cpu().numpy() for k, v in r.items()}

    def check(self, got):
        h, W = self.h.double().numpy(), self.W.double().numpy()
        N, V, D, K, T = self.N, self.V, self.D, self.K, self.T
        table = self.rows()
        rows = np.array(sorted(table), np.int64)
        loss, lse = sr.distill_forward(h, W, self.words, self.logits.numpy(), T)
        S = (6 if self.store == "f32" else 1) * -(-D // 16)
        h_ = h[rows]
        ez = (4 * S + 6) * U * (np.abs(h_) @ np.abs(W).T) / T
        z = h_ @ W.T / T
        sums = V / 64 + 80
        span = 2 + 2 * (z.max(1, initial=0) - z.min(1, initial=0)) if len(rows) else np.zeros(0)
        worst = ez.max(1, initial=0)
        e_lse = worst + (np.minimum(span, 220) + sums) * U + 3 * U * (np.abs(lse[rows]) + np.abs(z).max(1, initial=0) + 1)
        q, eq, e_loss = np.zeros((len(rows), V)), np.zeros((len(rows), V)), np.zeros(len(rows))
        for k, n in enumerate(rows):
            w, share, log_q = table[n]
            x = np.abs(log_q) + np.log(K)
            e = share * (2 * x + 2 * K + 8) * U + 2.0 ** -140
            np.add.at(q[k], w, share)
            np.add.at(eq[k], w, e)
            own = (share * np.abs(log_q)).sum()
            e_own = (e * (np.abs(log_q) + 1) + share * U * (6 * x + K)).sum()
            zw = np.abs(z[k, w])
            e_mean = (e * zw + share * ez[k, w] + (sums + 4) * U * share * zw).sum()
            e_loss[k] = T * T * (e_own + e_mean + e_lse[k] + 4 * U * (own + abs(lse[n]) + (share * zw).sum())) + 3 * U * abs(loss[n])
        for key, ref, e in (("lse", lse, e_lse), ("loss", loss, e_loss)):
            bound = np.zeros(N)
            bound[rows] = e
            assert (np.abs(got[key] - ref) <= bound).all(), (key, np.abs(got[key] - ref).max())
        if "dh" not in got and "dW" not in got:
            return
        dh, dW, dz = sr.distill_backward(self.dloss.double().numpy(), h, W, self.words, self.logits.numpy(), T)
        dz = dz[rows]
        g = T * np.abs(self.dloss.double().numpy()[rows, None])
        p = np.exp(z - lse[rows, None])
        e_dz = g * (p * (ez + e_lse[:, None] + (4 + 2 * np.abs(z - lse[rows, None])) * U) + eq + 3 * U) + 4 * U * np.abs(dz)
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
    # N, V, D, K, storage, gradients, T
    (1, 1, 1, 1, "f32", "f32", 1.0),
    (1, 2, 8, 3, "bf16", "f32", 2.0),
    (3, 5, 7, 128, "f32", "f32", 1.5),            # more entries than words
    (5, 129, 9, 4, "bf16", "bf16", 1.0),
    (16, 1000, 64, 10, "bf16", "f32", 4.0),       # rows of the kernel for up to 16
    (31, 127, 64, 5, "f32", "f32", 0.5),
    (33, 300, 63, 65, "bf16", "f32", 1.0),
    (64, 513, 64, 64, "f32", "f32", 3.0),
    (100, 700, 40, 17, "f32", "f32", 1.0),        # several groups of few rows
    (129, 257, 65, 32, "f32", "f32", 2.0),
    (127, 1000, 72, 100, "bf16", "bf16", 1.0),
    (300, 3001, 100, 20, "bf16", "f32", 1.5),
    (700, 1500, 260, 7, "f32", "f32", 1.0),
    (513, 500, 200, 128, "bf16", "bf16", 2.0),    # many entries of every row in every tile
    (600, 2000, 128, 1, "bf16", "f32", 1.0),
]


@pytest.mark.parametrize("N,V,D,K,store,out,T", CASES)
def test_against_the_oracle(N, V, D, K, store, out, T):
    p = Problem(N, V, D, K, store, out, T, seed=N + V, pad=0.0 if N == 1 else 0.3)
    if N == 1:
        p.words[0, 0], p.logits[0, 0] = V - 1, 0.5
    got = p.run()
    p.check(got)
    again = p.run()
    assert all(np.array_equal(got[k], again[k]) for k in got), "not the same from run to run"


@pytest.mark.parametrize("exponent", [-64, 64])
@pytest.mark.parametrize("N,V,D,K,store,out", [(3, 4, 16, 4, "f32", "f32"), (40, 130, 32, 9, "f32", "f32"), (40, 130, 32, 9, "bf16", "f32"),
                                               (200, 300, 32, 9, "f32", "f32"), (200, 300, 32, 9, "bf16", "bf16")])
def test_the_limits_of_the_temperature(N, V, D, K, store, out, exponent):
    """Its square is no fp32 number there.  At the upper limit a loss whose value is one is within the bound, other values are infinite."""
    p = Problem(N, V, D, K, store, out, 2.0 ** exponent, seed=N, pad=0.0)
    got = p.run()
    loss, _ = sr.distill_forward(p.h.double().numpy(), p.W.double().numpy(), p.words, p.logits.numpy(), p.T)
    huge = loss >= 2.0 ** 127
    assert (got["loss"][huge] >= 2.0 ** 126.9).all()
    got["loss"][huge] = loss[huge]
    p.check(got)


def test_larger_tiles():
    """Sizes that fill rounds of tiles of 256 x 256, in all three ways of keeping dz, against the smaller calls' results for the same rows."""
    for store, out in (("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")):
        p = Problem(4300, 4000, 64, 24, store, out, 1.5, seed=30)
        got = p.run()
        q = Problem(4300, 4000, 64, 24, store, out, 1.5, seed=30)
        keep = np.arange(4300) % 43 == 0
        q.words[~keep] = -1
        few = q.run()
        # each row's results depend on its own row and on W alone; the two calls differ by the sums' order and dz's scale at most
        for k, tol in (("loss", 2e-6), ("lse", 2e-6), ("dh", 2.0 ** -7 if out == "bf16" else 2e-6)):
            a, b = got[k][keep], few[k][keep]
            assert np.abs(a - b).max() <= tol * np.abs(a).max(), (store, out, k)
        dh, dW, _ = sr.distill_backward(p.dloss.double().numpy(), p.h.double().numpy(), p.W.double().numpy(), p.words, p.logits.numpy(), 1.5)
        for k, ref in (("dh", dh), ("dW", dW)):
            # bf16: half a step of the result and dz's own 2^-11; f32: sums of 4000 products' roundings, far below 1e-5 of the whole
            assert np.linalg.norm(got[k] - ref) <= (2.0 ** -8 if out == "bf16" else 1e-5) * np.linalg.norm(ref), (store, out, k)


@pytest.mark.parametrize("N,store", [(7, "f32"), (40, "bf16"), (300, "f32"), (300, "bf16")])
def test_rows_without_entries(N, store):
    torch, _, _ = _torch()
    p = Problem(N, 400, 48, 6, store, seed=40)
    p.words[:] = -1
    p.words[1::2] = 400
    got = p.run()
    assert all((x == 0).all() for x in got.values())
    p = Problem(N, 400, 48, 6, store, seed=41, pad=0.5)
    want = p.run()
    p.check(want)
    none = torch.from_numpy(np.array([n not in p.rows() for n in range(N)]))
    assert none.any()
    p.h[none], p.dloss[none], p.logits[none] = float("nan"), float("inf"), float("nan")
    got = p.run()
    assert all(np.array_equal(got[k], want[k]) for k in got)


def test_one_gradient_at_a_time():
    p = Problem(150, 600, 80, 9, "bf16", seed=42)
    both = p.run()
    for kw, key in ((dict(want_dW=False), "dh"), (dict(want_dh=False), "dW")):
        got = p.run(**kw)
        assert np.array_equal(got[key], both[key]) and len(got) == 3
    assert len(p.run(forward_only=True)) == 2


@pytest.mark.parametrize("N", [6, 60, 200])
@pytest.mark.parametrize("store", ["f32", "bf16"])
def test_one_word_is_the_label(N, store):
    """K = 1, T = 1 is the vocabulary loss without smoothing."""
    torch, eb, _ = _torch()
    p = Problem(N, 500, 64, 1, store, seed=43)
    got = p.run()
    st, dev = torch.cuda.current_stream(), lambda n: torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    labels = np.where(np.isin(np.arange(N), list(p.rows())), p.words[:, 0], -1).astype(np.int32)
    x = p.h.cuda(), p.W.cuda(), torch.from_numpy(labels).cuda(), 0.0
    loss, lse, dh, dW = (torch.empty(*s, device="cuda") for s in ((N,), (N,), (N, 64), (500, 64)))
    eb.check(eb.echo_vocab_loss_fwd(p.desc, *x, loss, lse, dev(eb.echo_vocab_loss_fwd_workspace_bytes(p.desc)), stream=st))
    eb.check(eb.echo_vocab_loss_bwd(p.desc, p.dloss.cuda(), lse, *x, dh, dW, dev(eb.echo_vocab_loss_bwd_workspace_bytes(p.desc)), stream=st))
    for k, ref in (("loss", loss), ("lse", lse), ("dh", dh), ("dW", dW)):
        ref = ref.double().cpu().numpy()
        assert np.abs(got[k] - ref).max() <= 2e-5 * np.abs(ref).max(), k


@pytest.mark.parametrize("N", [5, 50, 300])
def test_logits_without_end(N):
    p = Problem(N, 300, 32, 8, seed=44, pad=0.0)
    p.words[:, 0], p.logits[:, 0] = 5, 1.0
    want = p.run()
    p.logits[1, 0] = float("nan")
    p.logits[3, 0] = float("inf")
    got = p.run()
    for n in (1, 3):
        assert np.isnan(got["loss"][n]) and np.isnan(got["dh"][n]).all() and got["lse"][n] == want["lse"][n]
    rest = np.setdiff1d(np.arange(N), [1, 3])
    assert all(np.array_equal(got[k][rest], want[k][rest]) for k in ("loss", "lse", "dh"))


@pytest.mark.parametrize("N", [8, 40, 300])
def test_a_word_shut_out(N):
    """A word of logit minus infinity for every row: no share of it costs anything, and with one the loss is infinite."""
    torch, _, _ = _torch()
    p = Problem(N, 300, 32, 8, "bf16", seed=45, pad=0.0)
    p.words[p.words == 7] = 9
    p.words[:, 0], p.logits[:, 0] = 5, 1.0
    p.h[:, 0], p.W[7] = 1.0, 0.0
    p.W[7, 0] = -float("inf")
    got = p.run(forward_only=True)
    assert np.isfinite(got["loss"]).all() and np.isfinite(got["lse"]).all()
    q = Problem(N, 300, 32, 8, "bf16", seed=45, pad=0.0)
    q.words, q.logits, q.h, q.W = p.words.copy(), p.logits, p.h, p.W.clone()
    q.W[7] = 0
    q.W[7, 0] = -60.0                                       # as good as shut out: exp(-60) of a word of logit 0
    close = q.run(forward_only=True)
    assert np.abs(got["loss"] - close["loss"]).max() < 1e-4
    p.words[2, 0] = 7
    got = p.run(forward_only=True)
    assert got["loss"][2] == np.inf and np.isfinite(np.delete(got["loss"], 2)).all()


@pytest.mark.parametrize("N,V,store", [(20, 300, "f32"), (600, 900, "bf16")])
def test_captured_and_replayed(N, V, store):
    torch, eb, _ = _torch()
    p = Problem(N, V, 64, 12, store, T=2.0, seed=46)
    d, K, T = p.desc, p.K, p.T
    h, W, words, logits, dloss = p.h.cuda(), p.W.cuda(), torch.from_numpy(p.words).cuda(), p.logits.cuda(), p.dloss.cuda()
    out = dict(loss=torch.empty(N, device="cuda"), lse=torch.empty(N, device="cuda"), dh=torch.empty(N, 64, device="cuda"), dW=torch.empty(V, 64, device="cuda"))
    ws = torch.empty(max(eb.echo_distill_fwd_workspace_bytes(d, K), eb.echo_distill_bwd_workspace_bytes(d, K)), dtype=torch.uint8, device="cuda")

    def step():
        st = torch.cuda.current_stream()
        eb.check(eb.echo_distill_fwd(d, h, W, words, logits, K, T, out["loss"], out["lse"], ws, stream=st))
        eb.check(eb.echo_distill_bwd(d, dloss, out["lse"], h, W, words, logits, K, T, out["dh"], out["dW"], ws, stream=st))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    start = h.clone()
    for k in range(4):
        h.copy_(start * (k + 1) / 2)
        words.copy_(words.roll(1, 0))
        step()
        torch.cuda.synchronize()
        want = {key: x.clone() for key, x in out.items()}
        for x in out.values():
            x.fill_(float("nan"))
        ws.fill_(255 - k)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[key], want[key]) for key in out), k


def test_two_streams_at_once():
    torch, _, _ = _torch()
    p, q = Problem(300, 900, 64, 9, seed=47), Problem(30, 2000, 72, 30, "bf16", T=2.0, seed=48)
    want = p.run(), q.run()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for x, s, w in ((p, streams[0], want[0]), (q, streams[1], want[1])):
        got = x.run(stream=s)
        assert all(np.array_equal(got[k], w[k]) for k in w)
