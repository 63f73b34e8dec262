"""One training step of a decoder from the library's calls, as a program runs them, against float64 autograd: words embedded, LSTM cells, attention
over the source, the loss over the vocabulary with the embedding's table as its words, every gradient back (the table's from
both ends), and all of them clipped by their norm.

Tolerance: 1e-4 of the largest value of each tensor.  A value passes some 6 operations per step and 5 steps one after the other, each
with errors below 1e-6 of its result's scale (products of at most 40 terms, cells, a softmax over 7), each adding to the
errors of what it takes with a factor of about one; a term left out, a wrong scale or a wrong row is off by far more than a hundredth."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

B, T, S, H, V, EPS = 6, 5, 7, 40, 90, 0.1
LIMIT = 0.5


def _inputs():
    r = np.random.default_rng(21)
    n = lambda *s: (r.standard_normal(s) / np.sqrt(s[-1])).astype(np.float32)
    x = dict(E=n(V, H), Wx=n(4 * H, H), Wh=n(4 * H, H), Wq=n(H, H), Kp=n(B, S, H) * 6, Vs=n(B, S, H) * 6, v=n(H) * 6)
    tokens = r.integers(0, V, (B, T))
    tokens[:, 1] = tokens[0, 0]                                  # one word in every sentence
    labels = r.integers(0, V, (B, T))
    lengths = np.array([5, 1, 3, 5, 2, 4])
    past = np.arange(T) >= lengths[:, None]
    tokens[past], labels[past] = -1, -1
    return x, tokens.astype(np.int32), labels.astype(np.int32), np.array([7, 1, 4, 7, 3, 6], np.int32)


def _autograd():
    import torch
    x, tokens, labels, key_len = _inputs()
    p = {k: torch.from_numpy(a).double().requires_grad_() for k, a in x.items()}
    word = torch.from_numpy(tokens.astype(np.int64))
    emb = p["E"][word.clamp(min=0)] * np.sqrt(H) * (word >= 0)[..., None]
    h, c, hs = torch.zeros(B, H).double(), torch.zeros(B, H).double(), []
    for t in range(T):
        i, f, g, o = (emb[:, t] @ p["Wx"].T + h @ p["Wh"].T).chunk(4, 1)
        c = f.sigmoid() * c + i.sigmoid() * g.tanh()
        h = o.sigmoid() * c.tanh()
        hs.append(h)
    hs = torch.stack(hs, 1)
    s = ((hs @ p["Wq"].T)[:, :, None] + p["Kp"][:, None]).tanh() @ p["v"]
    s = s.masked_fill(torch.arange(S) >= torch.from_numpy(key_len)[:, None, None], -np.inf)
    out = hs + s.softmax(-1) @ p["Vs"]
    y = torch.from_numpy(labels.astype(np.int64))
    loss = torch.nn.functional.cross_entropy((out @ p["E"].T).reshape(B * T, V), y.reshape(-1), ignore_index=-1, label_smoothing=EPS)
    loss.backward()
    norm = torch.sqrt(sum((q.grad ** 2).sum() for q in p.values()))
    assert norm > LIMIT, "nothing to clip"
    return float(loss.detach()), float(norm), {k: (q.grad * (LIMIT / norm)).numpy() for k, q in p.items()}


def _library():
    import torch
    from paper_1805_08899_amd import binding as eb
    x, tokens, labels, key_len = _inputs()
    p = {k: torch.from_numpy(a).cuda() for k, a in x.items()}
    nan = lambda *s: torch.full(s, float("nan"), device="cuda")
    zeros = lambda *s: torch.zeros(*s, device="cuda")
    st = torch.cuda.current_stream()
    ws = lambda n: torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    word = torch.from_numpy(tokens.T.copy()).cuda().reshape(-1)                # step by step
    y, length = torch.from_numpy(labels).cuda().reshape(-1), torch.from_numpy(key_len).cuda()
    emb = nan(T, B, H)
    desc = eb.make_vocab_desc(T * B, V, H)
    eb.check(eb.echo_embed_fwd(desc, word, p["E"], float(np.sqrt(H)), emb, stream=st))
    hs, cs, sums = zeros(T + 1, B, H), zeros(T + 1, B, H), nan(T, B, 4 * H)
    for t in range(T):
        eb.check(eb.echo_lstm_cell_fwd(B, H, emb[t] @ p["Wx"].T, hs[t] @ p["Wh"].T, cs[t], hs[t + 1], cs[t + 1], sums[t], stream=st))
    states = hs[1:].transpose(0, 1).contiguous()                               # [B, T, H]
    Qp = states @ p["Wq"].T
    ad = eb.make_desc(B, T, S, H, H)
    context, P = nan(B, T, H), nan(B, T, S)
    eb.check(eb.echo_attn_fwd(ad, Qp, p["Kp"], p["Vs"], p["v"], length, context, P, ws(eb.echo_attn_fwd_workspace_bytes(ad)), stream=st))
    out = (states + context).reshape(B * T, H)
    loss, lse = nan(B * T), nan(B * T)
    eb.check(eb.echo_vocab_loss_fwd(desc, out, p["E"], y, EPS, loss, lse, ws(eb.echo_vocab_loss_fwd_workspace_bytes(desc)), stream=st))
    n = int((labels >= 0).sum())
    # back
    dout, g = nan(B * T, H), {k: nan(*q.shape) for k, q in p.items()}
    eb.check(eb.echo_vocab_loss_bwd(desc, torch.full((B * T,), 1.0 / n, device="cuda"), lse, out, p["E"], y, EPS, dout, g["E"],
                                    ws(eb.echo_vocab_loss_bwd_workspace_bytes(desc)), stream=st))
    dQp = nan(B, T, H)
    dout = dout.view(B, T, H)
    eb.check(eb.echo_attn_bwd(ad, dout, P, Qp, p["Kp"], p["Vs"], p["v"], length, dQp, g["Kp"], g["Vs"], g["v"],
                              ws(eb.echo_attn_bwd_workspace_bytes(ad)), stream=st))
    dstates = dout + dQp @ p["Wq"]
    g["Wq"] = dQp.reshape(-1, H).T @ states.reshape(-1, H)
    demb, da = nan(T, B, H), nan(T, B, 4 * H)
    dh, dc = zeros(B, H), None
    for t in reversed(range(T)):
        dc_prev = nan(B, H)
        eb.check(eb.echo_lstm_cell_bwd(B, H, (dstates[:, t] + dh).contiguous(), dc, sums[t], cs[t], da[t], dc_prev, stream=st))
        dh, dc = da[t] @ p["Wh"], dc_prev
        demb[t] = da[t] @ p["Wx"]
    g["Wx"] = da.reshape(-1, 4 * H).T @ emb.reshape(-1, H)
    g["Wh"] = da.reshape(-1, 4 * H).T @ hs[:T].reshape(-1, H)
    eb.check(eb.echo_embed_bwd_accumulate(desc, word, demb, float(np.sqrt(H)), g["E"], ws(eb.echo_embed_bwd_workspace_bytes(desc)), stream=st))
    names = list(g)
    norm = nan(1)
    g = {k: g[k].contiguous() for k in names}
    table = eb.make_grads([g[k] for k in names], [g[k] for k in names])
    eb.check(eb.echo_grad_clip(table, len(names), LIMIT, norm, ws(eb.echo_grad_workspace_bytes(table, len(names))), stream=st))
    torch.cuda.synchronize()
    return float(loss.sum()) / n, float(norm), {k: q.cpu().numpy() for k, q in g.items()}


def test_a_decoder_step_of_all_calls():
    loss, norm, grads = _library()
    want_loss, want_norm, want = _autograd()
    assert abs(loss - want_loss) <= 1e-4 * want_loss and abs(norm - want_norm) <= 1e-4 * want_norm
    for k, ref in want.items():
        assert np.abs(grads[k] - ref).max() <= 1e-4 * np.abs(ref).max(), k
    again = _library()
    assert again[0] == loss and again[1] == norm and all(np.array_equal(grads[k], again[2][k]) for k in grads)
