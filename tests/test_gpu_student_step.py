"""A student as a program runs it from the library's calls.  Training: words embedded, a layer of the gated recurrence in each direction, the distillation from
a teacher's top logits with the embedding's table as its words, every gradient back and clipped by their norm, against float64 autograd.  Use: the
student drafts words step by step, a model that reads whole sequences scores them in one pass, the drafts are verified.

Tolerance of the training step: 1e-4 of the largest value of each tensor.  A value passes some 6 operations per position and 9 positions, each with
errors below 1e-6 of its result's scale; a term left out, a wrong scale or a wrong row is off by far more than a hundredth."""
import numpy as np
import pytest

from oracle import student_ref as sr

pytestmark = pytest.mark.gpu

B, T, H, V, K, TEMP, LIMIT = 5, 9, 36, 80, 7, 2.0, 0.05


def _inputs():
    r = np.random.default_rng(31)
    n = lambda *s: (r.standard_normal(s) / np.sqrt(s[-1])).astype(np.float32)
    x = dict(E=n(V, H), Wf=n(3 * H, H) * 2, Wb=n(3 * H, H) * 2, c0=n(B, H) * 3)
    tokens, words = r.integers(0, V, (B, T)), r.integers(0, V, (B, T, K))
    words[..., 1][r.random((B, T)) < 0.3] = words[0, 0, 0]
    words[:, :, K - 1] = -1                                     # shorter lists
    lengths = np.array([9, 1, 4, 0, 7])
    past = np.arange(T) >= lengths[:, None]
    tokens[past], words[past] = -1, -1
    return x, tokens.astype(np.int32), words.astype(np.int32), (4 * r.standard_normal((B, T, K))).astype(np.float32), lengths.astype(np.int32)


def _autograd():
    import torch
    x, tokens, words, logits, lengths = _inputs()
    p = {k: torch.from_numpy(a).double().requires_grad_() for k, a in x.items()}
    word = torch.from_numpy(tokens.astype(np.int64))
    emb = p["E"][word.clamp(min=0)] * np.sqrt(H) * (word >= 0)[..., None]

    def layer(G, order, c):
        out = [torch.zeros(H).double()] * T
        for t in order:
            f, g, o = G[t].chunk(3)
            c = f.sigmoid() * c + (-f).sigmoid() * g.tanh()
            out[t] = o.sigmoid() * c
        return torch.stack(out)
    hs = torch.stack([layer(emb[b] @ p["Wf"].T, range(n), p["c0"][b]) + layer(emb[b] @ p["Wb"].T, range(n - 1, -1, -1), torch.zeros(H).double())
                      for b, n in enumerate(lengths)])
    total, rows = 0.0, 0
    log_p = torch.log_softmax(hs @ p["E"].T / TEMP, -1)
    for b in range(B):
        for t in range(lengths[b]):
            in_ = torch.from_numpy(words[b, t] >= 0)
            log_q = torch.log_softmax(torch.from_numpy(logits[b, t]).double()[in_] / TEMP, 0)
            total = total + TEMP ** 2 * (log_q.exp() * (log_q - log_p[b, t][torch.from_numpy(words[b, t].astype(np.int64))[in_]])).sum()
            rows += 1
    (total / rows).backward()
    norm = torch.sqrt(sum((q.grad ** 2).sum() for q in p.values()))
    assert norm > LIMIT, "nothing to clip"
    return float(total) / rows, float(norm), {k: (q.grad * (LIMIT / norm)).numpy() for k, q in p.items()}


def _library():
    import torch
    from paper_1805_08899_amd import binding as eb
    x, tokens, words, logits, lengths = _inputs()
    p = {k: torch.from_numpy(a).cuda() for k, a in x.items()}
    nan = lambda *s: torch.full(s, float("nan"), device="cuda")
    ws = lambda n: torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    st = torch.cuda.current_stream()
    dev = lambda a: torch.from_numpy(a).cuda()
    word, w, t, n = dev(tokens).reshape(-1), dev(words).reshape(-1, K), dev(logits).reshape(-1, K), dev(lengths)
    desc, emb = eb.make_vocab_desc(B * T, V, H), nan(B, T, H)
    eb.check(eb.echo_embed_fwd(desc, word, p["E"], float(np.sqrt(H)), emb, stream=st))
    layers = []
    for key, reverse, c0 in (("Wf", False, p["c0"]), ("Wb", True, None)):
        d = eb.make_scan_desc(B, T, H, reverse=reverse)
        G, h, states = emb @ p[key].T, nan(B, T, H), ws(eb.echo_scan_states_bytes(d))
        eb.check(eb.echo_scan_fwd(d, G, c0, n, h, None, states, ws(eb.echo_scan_fwd_workspace_bytes(d)), stream=st))
        layers.append((key, d, G, h, states, c0))
    out = (layers[0][3] + layers[1][3]).view(B * T, H)
    loss, lse = nan(B * T), nan(B * T)
    eb.check(eb.echo_distill_fwd(desc, out, p["E"], w, t, K, TEMP, loss, lse, ws(eb.echo_distill_fwd_workspace_bytes(desc, K)), stream=st))
    rows = int(lengths.sum())
    g, dout = {k: nan(*q.shape) for k, q in p.items()}, nan(B, T, H)
    eb.check(eb.echo_distill_bwd(desc, torch.full((B * T,), 1.0 / rows, device="cuda"), lse, out, p["E"], w, t, K, TEMP, dout, g["E"],
                                 ws(eb.echo_distill_bwd_workspace_bytes(desc, K)), stream=st))
    demb = torch.zeros(B, T, H, device="cuda")
    for key, d, G, h, states, c0 in layers:
        dG = nan(B, T, 3 * H)
        eb.check(eb.echo_scan_bwd(d, dout, None, G, n, states, dG, None if c0 is None else g["c0"], ws(eb.echo_scan_bwd_workspace_bytes(d)), stream=st))
        g[key] = dG.view(-1, 3 * H).T @ emb.view(-1, H)
        demb += dG @ p[key]
    eb.check(eb.echo_embed_bwd_accumulate(desc, word, demb, float(np.sqrt(H)), g["E"], ws(eb.echo_embed_bwd_workspace_bytes(desc)), stream=st))
    norm, names = nan(1), list(g)
    g = {k: g[k].contiguous() for k in names}
    table = eb.make_grads([g[k] for k in names])
    eb.check(eb.echo_grad_clip(table, len(names), LIMIT, norm, ws(eb.echo_grad_workspace_bytes(table, len(names))), stream=st))
    torch.cuda.synchronize()
    return float(loss.sum()) / rows, float(norm), {k: q.cpu().numpy() for k, q in g.items()}


def test_a_training_step_of_all_calls():
    loss, norm, grads = _library()
    want_loss, want_norm, want = _autograd()
    assert abs(loss - want_loss) <= 1e-4 * want_loss and abs(norm - want_norm) <= 1e-4 * want_norm
    for k, ref in want.items():
        assert np.abs(grads[k] - ref).max() <= 1e-4 * np.abs(ref).max(), k
    again = _library()
    assert again[0] == loss and again[1] == norm and all(np.array_equal(grads[k], again[2][k]) for k in grads)


def test_drafting_and_verification():
    """Five rounds: the student's steps draft, the model's pass over whole sequences scores, what is verified goes on from the state behind the last taken
    word.  The states after the rounds are those of the texts that came out, and each round's words the oracle's."""
    import torch
    from paper_1805_08899_amd import binding as eb
    n_draft, users = 4, 6
    r = np.random.default_rng(32)
    f32 = lambda *s: torch.from_numpy(r.standard_normal(s).astype(np.float32)).cuda()
    E, Ws, Wm = f32(V, H), f32(3 * H, H) / 6, f32(3 * H, H) / 6
    Wm = Ws + 0.3 * Wm                                           # a student that is close to its model
    st = torch.cuda.current_stream()
    one, several = eb.make_scan_desc(users, 1, H), eb.make_scan_desc(users, n_draft + 1, H)
    dd = eb.make_draft_desc(users, n_draft, V)
    ws = torch.empty(max(16, eb.echo_scan_fwd_workspace_bytes(several), eb.echo_draft_verify_workspace_bytes(dd)), dtype=torch.uint8, device="cuda")
    texts = [[int(x)] for x in r.integers(0, V, users)]
    c_student, c_model = torch.zeros(users, H, device="cuda"), torch.zeros(users, H, device="cuda")

    def run(desc, W, tokens, c, n=None):
        h, last = torch.empty(users, desc.T, H, device="cuda"), torch.empty(users, H, device="cuda")
        G = (E[tokens.long()] @ W.T).view(users, desc.T, 3 * H)
        eb.check(eb.echo_scan_fwd(desc, G, c, n, h, last, None, ws, stream=st))
        return torch.softmax(h @ E.T, -1), last
    for _ in range(5):
        before = torch.tensor([t[-1] for t in texts], dtype=torch.int32, device="cuda")
        word, c, drafts, q = before, c_student, [], []
        for _ in range(n_draft):
            probs, c = run(one, Ws, word.view(users, 1), c)
            q.append(probs[:, 0])
            word = (probs[:, 0].cumsum(-1) < torch.rand(users, 1, device="cuda")).sum(-1).clamp(max=V - 1).int()
            drafts.append(word)
        drafted, q = torch.stack(drafts, 1).contiguous(), torch.stack(q, 1).contiguous()
        fed = torch.cat([before[:, None], drafted], 1)
        p = run(several, Wm, fed, c_model)[0].contiguous()
        u, x = torch.rand(users, n_draft, device="cuda"), torch.rand(users, device="cuda")
        tokens, taken = torch.empty(users, n_draft + 1, dtype=torch.int32, device="cuda"), torch.empty(users, dtype=torch.int32, device="cuda")
        eb.check(eb.echo_draft_verify(dd, drafted, None, q, p, u, x, tokens, taken, ws, stream=st))
        want = sr.draft_verify(drafted.cpu().numpy(), None, *(a.double().cpu().numpy() for a in (q, p, u, x)))
        assert np.array_equal(tokens.cpu().numpy(), want[0]) and np.array_equal(taken.cpu().numpy(), want[1])
        # the states behind what was read and stands: the word in front and those taken
        n = (taken + 1).int()
        _, c_model = run(several, Wm, fed, c_model, n)
        _, c_student = run(several, Ws, fed, c_student, n)
        for b in range(users):
            texts[b] += tokens[b, :int(taken[b]) + 1].tolist()
    assert all(0 <= w < V for t in texts for w in t) and max(map(len, texts)) > 6
    for W, c in ((Ws, c_student), (Wm, c_model)):
        for b in range(users):
            G = (E[torch.tensor(texts[b][:-1], device="cuda")] @ W.T)[None].double().cpu().numpy()
            ref = sr.scan_forward(G, None, None)[1][0]
            assert np.abs(c[b].double().cpu().numpy() - ref).max() < 1e-4
