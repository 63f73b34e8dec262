"""The gated linear recurrence and its gradients against the float64 oracle.

Tolerances, for every value, from the arithmetic; u = 2^-24.  A sigmoid s has an error of s (1 - s) (2 |x| + 2) u from its exponential (argument rounded twice, the
exponential 2 u) and of 3 u s from the sum and the reciprocal: below 4 u, as s (1 - s) |x| <= 0.23.  A tanh, 1 - 2 r with r the same at 2x, below 9 u.
  c   a step adds 4 u (|c| + |g|) from 1 - f, 9 u from g and two roundings of numbers up to |c| + |g|, whether it is taken by itself or as part of a map of
      several steps (a map's factor is off by 5 u for each of its gates):  E[t] = f E[t-1] + 16 u (ca[t-1] + 1), ca as c with |c0| and |g|
  r   the same backwards:  E[t] = f[t+1] E[t+1] + 16 u (ra[t] + |dh[t]|), ra as r with |dh| and |dc_last|
  dG  the products' factors' errors, as they stand below, and their roundings; what is stored is rounded by half a step of its type."""
import numpy as np
import pytest

from oracle import student_ref as sr

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"f32": U, "bf16": 2.0 ** -8}


def _torch():
    import torch
    assert torch.cuda.is_available(), "needs the GPU"
    from paper_1805_08899_amd import binding as eb
    return torch, eb, {"f32": torch.float32, "bf16": torch.bfloat16}


class Buffers:
    """Device buffers with a guard in front and behind, and their contents undefined (0xFF: NaN)."""
    def __init__(self, torch):
        self.torch, self.all = torch, []

    def bytes(self, n, guard=256):
        whole = self.torch.full((n + 2 * guard + 16,), 0xFF, dtype=self.torch.uint8, device="cuda")
        self.all.append((whole, guard, n))
        return whole[guard:guard + n]

    def of(self, dtype, *shape):
        return self.bytes(int(np.prod(shape)) * (2 if dtype == self.torch.bfloat16 else 4)).view(dtype).view(*shape)

    def check(self):
        for whole, guard, n in self.all:
            assert bool((whole[:guard] == 0xFF).all()) and bool((whole[guard + n:] == 0xFF).all()), "written outside its buffer"


class Problem:
    def __init__(self, B, T, H, store="f32", reverse=False, lengths=None, c0=True, dc_last=True, seed=0, keep=3.0, scale=1.0):
        torch, eb, types = _torch()
        self.B, self.T, self.H, self.store, self.reverse = B, T, H, store, reverse
        r = np.random.default_rng(seed)
        G = scale * r.standard_normal((B, T, 3 * H))
        G[:, :, :H] += keep * r.random(H)
        if lengths == "random":
            lengths = r.integers(0, T + 1, B)
            lengths[r.integers(0, B)] = T
            lengths[r.integers(0, B)] = 0
        self.n = None if lengths is None else np.asarray(lengths, np.int32)
        to = lambda x: torch.from_numpy(x.astype(np.float32))
        self.G, self.dh = to(G).to(types[store]), to(r.standard_normal((B, T, H))).to(types[store])
        if self.n is not None:                              # what stands behind a sequence's end is nobody's business
            behind = torch.from_numpy(np.arange(T) >= self.n[:, None])
            self.G[behind] = float("nan")
            self.dh[behind] = float("inf")
        self.c0 = to(r.standard_normal((B, H))) if c0 else None
        self.dc_last = to(r.standard_normal((B, H))) if dc_last else None
        self.desc = eb.make_scan_desc(B, T, H, store, reverse)

    def run(self, backward=True, stream=None, in_place=False, want_last=True):
        torch, eb, types = _torch()
        b, t = Buffers(torch), types[self.store]
        dev = lambda x: None if x is None else x.cuda()
        B, T, H = self.B, self.T, self.H
        G, dh, c0, dc = dev(self.G), dev(self.dh), dev(self.c0), dev(self.dc_last)
        n = None if self.n is None else torch.from_numpy(self.n).cuda()
        h, c_last = b.of(t, B, T, H), c0 if in_place else b.of(torch.float32, B, H) if want_last else None
        states = b.bytes(eb.echo_scan_states_bytes(self.desc)) if backward else None
        size = eb.echo_scan_fwd_workspace_bytes(self.desc)
        st = stream or torch.cuda.current_stream()
        eb.check(eb.echo_scan_fwd(self.desc, G, c0, n, h, c_last, states, b.bytes(size) if size else None, stream=st))
        out = {"h": h, "c_last": c_last}
        if backward:
            dG, dc0 = b.of(t, B, T, 3 * H), dc if in_place else b.of(torch.float32, B, H) if want_last else None
            size = eb.echo_scan_bwd_workspace_bytes(self.desc)
            eb.check(eb.echo_scan_bwd(self.desc, dh, dc, G, n, states, dG, dc0, b.bytes(size) if size else None, stream=st))
            out.update(dG=dG, dc0=dc0)
        torch.cuda.synchronize()
        b.check()
        return {k: x.double().cpu().numpy() for k, x in out.items() if x is not None}

    def check(self, got):
        f64 = lambda x: None if x is None else x.double().numpy()
        G, dh, c0, dc = f64(self.G), f64(self.dh), f64(self.c0), f64(self.dc_last)
        B, T, H = self.B, self.T, self.H
        c0 = np.zeros((B, H)) if c0 is None else c0
        dc = np.zeros((B, H)) if dc is None else dc
        bound = {"h": np.zeros((B, T, H)), "c_last": np.zeros((B, H)), "dG": np.zeros((B, T, 3 * H)), "dc0": np.zeros((B, H))}
        ref = {k: np.zeros_like(x) for k, x in bound.items()}
        half = HALF[self.store]
        for b, n in enumerate(sr.lengths(self.n, B, T)):
            order = list(range(n - 1, -1, -1) if self.reverse else range(n))
            s = lambda x: 1 / (1 + np.exp(-x))
            f, k, g, o = s(G[b, :, :H]), s(-G[b, :, :H]), np.tanh(G[b, :, H:2 * H]), s(G[b, :, 2 * H:])
            c, ca, E, before = c0[b], np.abs(c0[b]), np.zeros(H), {}
            for t in order:
                before[t] = (c, ca, E)
                E = f[t] * E + 16 * U * (ca + 1)
                c, ca = f[t] * c + k[t] * g[t], f[t] * ca + k[t] * np.abs(g[t])
                ref["h"][b, t] = o[t] * c
                bound["h"][b, t] = o[t] * E + 8 * U * ca + half * np.abs(o[t] * c)
                before[t] += (c, ca, E)
            ref["c_last"][b], bound["c_last"][b] = c, E
            if "dG" not in got:
                continue
            q, qa, E = dc[b], np.abs(dc[b]), np.zeros(H)
            for t in reversed(order):
                c_, ca_, Ec_, c, ca, Ec = before[t]
                d = np.abs(dh[b, t])
                r, ra = dh[b, t] * o[t] + q, d * o[t] + qa
                E = E + 16 * U * (ra + d)
                fk = f[t] * k[t]
                e_f = E * (ca_ + 1) * fk + ra * (Ec_ + 9 * U) * fk + 8 * U * ra * (ca_ + 1)
                e_g = E * k[t] * (1 - g[t] ** 2) + ra * U * (4 * (1 - g[t] ** 2) + 18 * k[t] + 8)
                e_o = d * (Ec + 12 * U * ca)
                want = np.concatenate([r * (c_ - g[t]) * fk, r * k[t] * (1 - g[t] ** 2), dh[b, t] * c * o[t] * (1 - o[t])])
                ref["dG"][b, t], bound["dG"][b, t] = want, np.concatenate([e_f, e_g, e_o]) + half * np.abs(want)
                q, qa, E = f[t] * r, f[t] * ra, f[t] * E + 8 * U * ra
            ref["dc0"][b], bound["dc0"][b] = q, E
        for key, x in got.items():
            off = np.abs(x - ref[key])
            assert (off <= 1.01 * bound[key]).all(), (key, off.max(), np.nanmax(off / np.maximum(bound[key], 1e-300)))


CASES = [
    # B, T, H, storage, reverse, lengths
    (1, 1, 1, "f32", False, None),
    (1, 1, 1, "bf16", True, None),
    (3, 1, 512, "f32", False, None),
    (5, 1, 70, "bf16", False, [1, 0, 1, 1, 0]),
    (2, 2, 3, "f32", True, None),
    (4, 4, 5, "bf16", False, "random"),
    (3, 5, 4, "f32", False, "random"),
    (2, 16, 66, "f32", True, "random"),
    (7, 17, 130, "bf16", True, "random"),
    (64, 50, 24, "f32", False, "random"),
    (3, 64, 65, "f32", False, "random"),
    (2, 65, 67, "bf16", True, "random"),
    (2, 127, 64, "f32", True, "random"),
    (2, 128, 31, "bf16", False, "random"),
    (3, 129, 129, "f32", False, "random"),
    (2, 257, 2, "f32", True, "random"),
    (5, 300, 62, "bf16", True, "random"),
    (1, 1025, 63, "f32", False, None),
    (2, 1500, 20, "f32", True, [1500, 1409]),
    (1, 4001, 16, "bf16", False, None),
    (2, 5000, 68, "f32", False, [4999, 130]),
]


@pytest.mark.parametrize("B,T,H,store,reverse,lengths", CASES)
def test_against_the_oracle(B, T, H, store, reverse, lengths):
    p = Problem(B, T, H, store, reverse, lengths, seed=B + T + H)
    got = p.run()
    p.check(got)
    again = p.run()
    assert all(np.array_equal(got[k], again[k]) for k in got), "not the same from run to run"


@pytest.mark.parametrize("store,reverse", [("f32", False), ("bf16", True)])
def test_lengths_at_the_ends_of_chunks(store, reverse):
    """Sequences that end with a chunk, one step behind it and in front of it, chunks without a step, and a sequence without any."""
    p = Problem(9, 520, 70, store, reverse, lengths=[128, 129, 127, 0, 256, 257, 520, 512, 1], seed=20)
    p.check(p.run())


@pytest.mark.parametrize("B,T,H,store", [(5, 129, 66, "f32"), (3, 255, 130, "bf16"), (9, 256, 3, "f32"), (40, 200, 64, "bf16"),      # two chunks
                                         (8, 260, 4094, "bf16"), (16, 385, 2047, "f32"), (2, 512, 16384, "f32"),                    # many chains of three or four
                                         (7, 260, 4094, "bf16")])                                                                  # a few less
@pytest.mark.parametrize("reverse", [False, True])
def test_chains_of_one_block_and_of_many(B, T, H, store, reverse):
    r = np.random.default_rng(B)
    lengths = r.integers(0, T + 1, B)
    lengths[:5] = [T, 128, 0, 129, 1][:B]
    p = Problem(B, T, H, store, reverse, lengths.tolist(), seed=21)
    got = p.run(in_place=True)
    p.check(got)
    again = p.run(in_place=True)
    assert all(np.array_equal(got[k], again[k]) for k in got)


def test_more_units_than_blocks():
    """222 chains of 3 chunks, which the blocks take in turns from queues of unequal length, a third of them empty; most sequences are short."""
    r = np.random.default_rng(21)
    p = Problem(37, 300, 330, "bf16", True, lengths=(300 * r.random(37) ** 2).astype(int).tolist(), seed=21)
    got = p.run()
    p.check(got)
    again = p.run()
    assert all(np.array_equal(got[k], again[k]) for k in got)


@pytest.mark.parametrize("T", [1, 7, 200])
def test_what_may_be_left_out(T):
    p = Problem(3, T, 37, lengths=None, c0=False, dc_last=False, seed=1)
    p.check(p.run())
    got = p.run(want_last=False)
    assert set(got) == {"h", "dG"}
    p.check(got)
    p.check(p.run(backward=False))


@pytest.mark.parametrize("B,T,H", [(4, 1, 65), (3, 9, 130), (2, 300, 66)])
@pytest.mark.parametrize("reverse", [False, True])
def test_states_in_place(B, T, H, reverse):
    """c_last over c0, dc0 over dc_last: also where the last channels' group begins in the neighbour's."""
    p = Problem(B, T, H, reverse=reverse, lengths="random", seed=2)
    p.check(p.run(in_place=True))


@pytest.mark.parametrize("B,T,H", [(40, 33, 130), (9, 64, 70), (300, 65, 66), (64, 128, 257)])
@pytest.mark.parametrize("reverse", [False, True])
def test_states_in_place_that_several_waves_read(B, T, H, reverse):
    """A chunk's states are read by each of its waves and written by one of them, which has to wait for the others' reads."""
    p = Problem(B, T, H, reverse=reverse, lengths="random", seed=B)
    p.check(p.run(in_place=True))


def test_steps_one_by_one_are_the_sequence():
    torch, eb, _ = _torch()
    p = Problem(4, 9, 70, seed=3)
    whole = p.run(backward=False)
    d, c, ws = eb.make_scan_desc(4, 1, 70), p.c0.cuda(), None
    for t in range(9):
        h = torch.full((4, 1, 70), float("nan"), device="cuda")
        eb.check(eb.echo_scan_fwd(d, p.G[:, t:t + 1].contiguous().cuda(), c, None, h, c, None, ws, stream=torch.cuda.current_stream()))
        assert np.abs(h[:, 0].double().cpu().numpy() - whole["h"][:, t]).max() < 1e-5
    assert np.abs(c.double().cpu().numpy() - whole["c_last"]).max() < 1e-5


@pytest.mark.parametrize("scale", [30.0, 1e4, 1e38])
def test_saturated_gates(scale):
    """Gates that are 0 or 1 to the last digit, and exponentials past the end of fp32's range."""
    for T in (3, 140):
        p = Problem(2, T, 8, scale=scale, seed=4)
        with np.errstate(over="ignore"):
            p.check(p.run())


def test_infinite_gates():
    torch, _, _ = _torch()
    p = Problem(1, 6, 8, seed=5)
    p.G[0, 1, :8] = float("inf")                            # keeps all
    p.G[0, 3, :8] = -float("inf")                           # forgets all
    p.G[0, 4, 8:16], p.G[0, 4, 16:] = float("inf"), -float("inf")
    with np.errstate(over="ignore"):
        p.check(p.run())


def test_a_NaN_stays_with_its_sequence_and_channel():
    p = Problem(3, 200, 9, seed=6)
    clean = p.run()
    p.G[1, 150, 4] = float("nan")
    got = p.run()
    for k in ("h", "c_last"):
        nan = np.isnan(got[k])
        assert nan[1, ..., 4].any()
        nan[1, ..., 4] = False
        assert not nan.any()
        keep = ~np.isnan(got[k])
        assert np.array_equal(got[k][keep], clean[k][keep])
    assert not np.isnan(got["dG"][[0, 2]]).any() and not np.isnan(got["h"][1, :150]).any()


@pytest.mark.parametrize("store", ["f32", "bf16"])
def test_longer_chains(store):
    """What the tests above show for chunks of one block, for those that are handed on: states left out, saturated gates, a NaN."""
    p = Problem(3, 600, 37, store, lengths=None, c0=False, dc_last=False, seed=11)
    p.check(p.run())
    p.check(p.run(want_last=False))
    for scale in (30.0, 1e4):
        p = Problem(2, 600, 8, store, scale=scale, seed=12)
        with np.errstate(over="ignore"):
            p.check(p.run())
    p = Problem(3, 700, 9, store, seed=13)
    clean = p.run()
    p.G[1, 150, 4] = float("nan")                           # a gate that forgets
    p.G[1, 450, 9 + 6] = float("nan")                       # a candidate
    got = p.run()
    for ch, t in ((4, 150), (6, 450)):
        assert np.isnan(got["h"][1, t:, ch]).all() and np.isnan(got["c_last"][1, ch]) and np.isnan(got["dc0"][1, ch]) == (ch == 4)
        assert np.array_equal(got["h"][1, :t, ch], clean["h"][1, :t, ch])
    rest = np.setdiff1d(np.arange(9), [4, 6])
    for k in ("h", "c_last", "dc0"):
        assert np.array_equal(got[k][..., rest], clean[k][..., rest]) and np.array_equal(got[k][[0, 2]], clean[k][[0, 2]])
    three = np.concatenate([rest, 9 + rest, 18 + rest])
    assert np.array_equal(got["dG"][..., three], clean["dG"][..., three])


def test_lengths_outside_their_range():
    p = Problem(3, 6, 5, lengths=[-3, 6, 4], seed=7)
    want = p.run()
    p.n = np.array([-2 ** 31, 2 ** 31 - 1, 4], np.int32)
    got = p.run()
    assert all(np.array_equal(got[k], want[k]) for k in got)


def test_on_another_stream_and_two_at_once():
    torch, _, _ = _torch()
    p, q = Problem(2, 700, 130, seed=8), Problem(3, 600, 64, "bf16", reverse=True, lengths="random", seed=9)
    want = p.run(), q.run()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for x, s, w in ((p, streams[0], want[0]), (q, streams[1], want[1])):
        got = x.run(stream=s)
        assert all(np.array_equal(got[k], w[k]) for k in w)


@pytest.mark.parametrize("T", [3, 60, 200, 1000])
def test_captured_and_replayed(T):
    torch, eb, types = _torch()
    p = Problem(2, T, 72, lengths="random", seed=10)
    d = p.desc
    G, dh, c0, dc, n = p.G.cuda(), p.dh.cuda(), p.c0.cuda(), p.dc_last.cuda(), torch.from_numpy(p.n).cuda()
    out = dict(h=torch.empty(2, T, 72, device="cuda"), c_last=torch.empty(2, 72, device="cuda"), dG=torch.empty(2, T, 216, device="cuda"),
               dc0=torch.empty(2, 72, device="cuda"))
    states = torch.empty(eb.echo_scan_states_bytes(d), dtype=torch.uint8, device="cuda")
    ws = torch.full((max(16, eb.echo_scan_fwd_workspace_bytes(d), eb.echo_scan_bwd_workspace_bytes(d)),), 1, dtype=torch.uint8, device="cuda")

    def step():
        st = torch.cuda.current_stream()
        eb.check(eb.echo_scan_fwd(d, G, c0, n, out["h"], out["c_last"], states, ws, stream=st))
        eb.check(eb.echo_scan_bwd(d, dh, dc, G, n, states, out["dG"], out["dc0"], ws, stream=st))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    inputs = torch.nan_to_num(torch.randn_like(G)), c0.clone()
    for k in range(4):
        G.copy_(inputs[0] * (k + 1) / 2)
        c0.copy_(inputs[1] * k)
        step()
        torch.cuda.synchronize()
        want = {key: x.clone() for key, x in out.items()}
        for x in out.values():
            x.fill_(float("nan"))
        ws.fill_(k)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[key], want[key]) for key in out), k


@pytest.mark.parametrize("B,T,H", [(3, 4096, 65536), (3, 256, 1 << 20), (6, 120, 1 << 20)])      # many blocks' chains, a block's, one chunk
def test_offsets_past_32_bits(B, T, H):
    """G of 2^31.2 numbers: the last sequence against the same one by itself."""
    torch, eb, _ = _torch()
    st = torch.cuda.current_stream()
    G = torch.empty(B, T, 3 * H, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(11)
    for b in range(B):
        G[b].normal_(generator=g)
    results = []
    for x in (G, G[B - 1:].contiguous()):
        d = eb.make_scan_desc(x.shape[0], T, H, "bf16")
        h = torch.empty(x.shape[0], T, H, dtype=torch.bfloat16, device="cuda")
        states = torch.empty(eb.echo_scan_states_bytes(d), dtype=torch.uint8, device="cuda")
        ws = torch.empty(max(16, eb.echo_scan_fwd_workspace_bytes(d), eb.echo_scan_bwd_workspace_bytes(d)), dtype=torch.uint8, device="cuda")
        c = torch.empty(x.shape[0], H, device="cuda")
        eb.check(eb.echo_scan_fwd(d, x, None, None, h, c, states, ws, stream=st))
        dG = torch.empty_like(x)
        eb.check(eb.echo_scan_bwd(d, h, None, x, None, states, dG, None, ws, stream=st))
        results.append((h[-1].clone(), c[-1].clone(), dG[-1].clone()))
        del dG, h
    for a, b in zip(*results):
        assert torch.equal(a, b)
    assert bool(torch.isfinite(results[0][1]).all())
