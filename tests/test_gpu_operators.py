"""The joiner's operators used together, as training and as decoding use them, on streams, in
captured graphs and twice at once."""
import math

import numpy as np
import pytest

from gpu_util import say

pytestmark = pytest.mark.gpu


def _model(D=40, C=48, V=60, seed=0, dtype="float32"):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")
    dt = getattr(torch, dtype)
    return {"we": (r(C, D) * D ** -0.5).to(dt), "be": (r(C) * 0.1).to(dt),
            "wo": (r(V, C) * C ** -0.5).to(dt), "bo": (r(V) * 0.1).to(dt)}


def _train_step(kind, p, enc, dec, y, lens, weights):
    """Joiner over every cell, loss and gradients: enc [B, T, D], dec [B, U+1, C] (the
    decoder's output), y [B, U].  The projection of the frames, with the decoder's rows as
    its residual, runs over cells, so that the pre-activation is the joiner's."""
    import torch
    from paper_2211_00484_amd import tbs
    B, T, D = enc.shape
    U1, C = dec.shape[1], dec.shape[2]
    V = p["wo"].shape[0]
    cells = enc[:, :, None, :].expand(B, T, U1, D).contiguous()
    res = dec[:, None].expand(B, T, U1, C).contiguous()
    h, pre = tbs.linear(cells, p["we"], p["be"], residual=res, activation="tanh", want_pre=True)
    z = tbs.linear(h, p["wo"], p["bo"])
    logp = tbs.adjust_logits(z, normalize=True).float()
    at = y[:, None, :, None].expand(B, T, U1 - 1, 1)
    blank = logp[..., 0].contiguous()
    label = torch.gather(logp[:, :, :-1], 3, at)[..., 0].contiguous()
    total, gb, gl, status = tbs.transducer_gradient(kind, blank, label, lens, weights=weights)
    # through the log-softmax: d logp is sparse
    dl = torch.zeros_like(logp)
    dl[..., 0] = gb
    dl[:, :, :-1].scatter_add_(3, at, gl[..., None])
    dz = (dl - torch.exp(logp) * dl.sum(-1, keepdim=True)).to(z.dtype)
    go = tbs.linear_backward(dz, h, p["wo"])
    gi = tbs.linear_backward(go.x, cells, p["we"], pre=pre, activation="tanh", want_pre=True)
    return {"total": total, "wo": go.weight, "bo": go.bias, "we": gi.weight, "be": gi.bias,
            "enc": gi.x.float().sum(2), "dec": gi.pre.float().sum(1)}


def _reference_step(kind, p, enc, dec, y, frames, labels, weights):
    """The same in 64 bits with automatic differentiation, on the CPU."""
    import torch
    q = {k: v.double().cpu().requires_grad_(True) for k, v in p.items()}
    e, d = (t.double().cpu().requires_grad_(True) for t in (enc, dec))
    h = torch.tanh((e @ q["we"].t())[:, :, None] + q["be"] + d[:, None])
    logp = torch.log_softmax(h @ q["wo"].t() + q["bo"], -1)
    loss, totals = 0.0, []
    yc = y.cpu()
    for b in range(e.shape[0]):
        T, U = int(frames[b]), int(labels[b])
        bl = logp[b, :T, :U + 1, 0]
        lb = torch.gather(logp[b, :T, :U], 2, yc[b, :U][None, :, None].expand(T, U, 1))[..., 0]
        a = torch.full((U + 1,), -1e30, dtype=torch.float64)
        a = torch.cat([torch.zeros(1, dtype=torch.float64), a[1:]])
        wall = torch.full((1,), -1e30, dtype=torch.float64)
        if kind == "standard":
            for t in range(T):
                come = a if t == 0 else a + bl[t - 1]
                row = [come[0]]
                for u in range(1, U + 1):
                    v = row[-1] + lb[t, u - 1]
                    row.append(v if t == 0 else torch.logaddexp(come[u], v))
                a = torch.stack(row)
            tot = a[U] + bl[T - 1, U]
        else:
            for t in range(T):
                up = torch.cat([wall, a[:U] + lb[t]])
                if kind == "constrained":
                    up = up + bl[t]
                a = torch.logaddexp(a + bl[t], up)
            tot = a[U]
        totals.append(tot.detach())
        loss = loss + float(weights[b]) * tot
    loss.backward()
    out = {k: v.grad for k, v in q.items()}
    out.update(total=torch.stack(totals), enc=e.grad, dec=d.grad)
    return out


@pytest.mark.parametrize("kind", ["standard", "modified", "constrained"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_training_step(kind, dtype):
    """Gradients of a whole step.  fp32: every stage is within a few 1e-6 of its values, of
    which the totals' recursion sums T + U; bf16: three tensors are rounded to 2^-9 (rms) on
    the way there and three back, and the log-probabilities' error (2^-9 of about 4) moves the
    occupancies by as much."""
    import torch
    B, T, D, U, C = 3, 14, 40, 6, 48
    p = _model(D, C, 60, 1, dtype)
    g = torch.Generator(device="cuda").manual_seed(5)
    dt = getattr(torch, dtype)
    enc = torch.randn((B, T, D), generator=g, device="cuda").to(dt)
    dec = torch.relu(torch.randn((B, U + 1, C), generator=g, device="cuda")).to(dt)
    y = torch.randint(1, 60, (B, U), generator=g, device="cuda")
    frames, labels = [14, 9, 12], [6, 4, 0]
    lens = torch.tensor(list(zip(frames, labels)), dtype=torch.int32, device="cuda")
    weights = torch.tensor([-0.5, -1.0, -0.25], dtype=torch.float64, device="cuda")
    got = _train_step(kind, p, enc, dec, y, lens, weights)
    want = _reference_step(kind, p, enc, dec, y, frames, labels, weights.cpu())
    rel = 2e-5 if dtype == "float32" else 0.1
    for k, w in want.items():
        v = got[k].double().cpu()
        assert torch.isfinite(v).all()
        err = (v - w).norm().item() / w.norm().item()
        say(f"  {kind} {dtype} {k}: {err:.2e}")
        assert err <= rel, k


def _answer_step(p, x, hist, hlen, pen, graph, states):
    import torch
    from paper_2211_00484_amd import tbs
    h = tbs.linear(x, p["we"], p["be"], activation="tanh")
    z = tbs.linear(h, p["wo"], p["bo"])
    return tbs.adjust_logits(z, history=hist, history_lengths=hlen, row_penalties=pen, graph=graph,
                             states=states, normalize=True)


def test_answer_step():
    """Projection, logits, adjustments and the label taken, one frame after the other: the labels
    follow the graph and the history grows."""
    import torch
    from paper_2211_00484_amd import tbs
    R, D, C, V, T = 6, 40, 48, 60, 25
    p = _model(D, C, V, 2)
    rng = np.random.default_rng(0)
    S = 30
    deg = rng.integers(1, 5, S)
    rp = np.concatenate([[0], np.cumsum(deg)]).astype(np.int32)
    dest = rng.integers(0, S, rp[-1]).astype(np.int32)
    lab = rng.integers(1, V, rp[-1]).astype(np.int32)
    graph = tbs.Graph.from_csr(S, 0, V, rp, dest, lab, np.zeros(rp[-1], np.float32))
    hist = torch.full((R, T), -1, dtype=torch.int32, device="cuda")
    n = torch.zeros(R, dtype=torch.int32, device="cuda")
    states = torch.zeros(R, dtype=torch.int32, device="cuda")
    pen = torch.tensor([[1.2, 0.3, 0.1]], device="cuda").repeat(R, 1)
    pd = {k: v.double().cpu() for k, v in p.items()}
    for t in range(T):
        x = torch.randn((R, D), generator=torch.Generator(device="cuda").manual_seed(t), device="cuda")
        logp = _answer_step(p, x, hist, n, pen, graph, states)
        z = torch.tanh(x.double().cpu() @ pd["we"].t() + pd["be"]) @ pd["wo"].t() + pd["bo"]
        for r in range(R):
            s = int(states[r])
            ok = sorted({0} | set(lab[rp[s]:rp[s + 1]].tolist()))
            cnt = np.bincount(hist[r, :int(n[r])].cpu().numpy(), minlength=V)
            v = z[r].clone()
            for c in np.nonzero(cnt)[0]:
                v[c] = (v[c] / np.float32(1.2) if v[c] > 0 else v[c] * np.float32(1.2)) \
                    - np.float32(0.3) - np.float32(0.1) * cnt[c]
            want = torch.full((V,), -math.inf, dtype=torch.float64)
            want[ok] = torch.log_softmax(v[ok], 0)
            g = logp[r].double().cpu()
            assert torch.equal(torch.isfinite(g), torch.isfinite(want))
            assert (g - want)[ok].abs().max() <= 2e-5
            c = int(logp[r].argmax())
            assert c in ok
            if c:
                arc = rp[s] + int(np.nonzero(lab[rp[s]:rp[s + 1]] == c)[0][0])
                states[r] = int(dest[arc])
                hist[r, int(n[r])] = c
                n[r] += 1


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_captured_and_replayed(dtype):
    """A training and an answering step in one graph, replayed with new inputs and the eager
    program's own work between the replays."""
    import torch
    B, T, D, U, C, V = 4, 30, 40, 9, 48, 60
    p = _model(D, C, V, 3, dtype)
    dt = getattr(torch, dtype)
    enc = torch.zeros((B, T, D), dtype=dt, device="cuda")
    dec = torch.zeros((B, U + 1, C), dtype=dt, device="cuda")
    y = torch.ones((B, U), dtype=torch.int64, device="cuda")
    lens = torch.tensor([[T, U]] * B, dtype=torch.int32, device="cuda")
    w = torch.full((B,), -0.25, dtype=torch.float64, device="cuda")
    hist = torch.zeros((B * T, 8), dtype=torch.int32, device="cuda")
    from paper_2211_00484_amd import tbs

    def step():
        out = _train_step("modified", p, enc, dec, y, lens, w)
        out["logp"] = tbs.adjust_logits(tbs.linear(tbs.linear(enc.view(-1, D), p["we"], p["be"], activation="tanh"),
                                                   p["wo"], p["bo"]),
                                        history=hist, repetition=1.5, presence=0.5, normalize=True)
        return out

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        for _ in range(2):
            step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for k in range(4):
        g = torch.Generator(device="cuda").manual_seed(k)
        enc.copy_(torch.randn((B, T, D), generator=g, device="cuda"))
        dec.copy_(torch.randn((B, U + 1, C), generator=g, device="cuda"))
        y.copy_(torch.randint(1, V, (B, U), generator=g, device="cuda"))
        hist.copy_(torch.randint(-1, V, hist.shape, generator=g, device="cuda"))
        lens.copy_(torch.tensor([[T - k, U], [T, U - k], [T - 2 * k, 3], [T, 0]], dtype=torch.int32))
        graph.replay()
        got = {n: t.clone() for n, t in captured.items()}
        eager = step()
        torch.cuda.synchronize()
        for n in eager:
            assert torch.equal(got[n], eager[n]), (k, n)


def test_two_streams_at_once():
    """Two steps in flight on two streams, each with its own workspaces, many times."""
    import torch
    from paper_2211_00484_amd import tbs
    g = torch.Generator(device="cuda").manual_seed(1)
    sets = []
    for i in range(2):
        x = torch.randn((6000, 300), generator=g, device="cuda")
        w = torch.randn((100, 300), generator=g, device="cuda")
        dy = torch.randn((6000, 100), generator=g, device="cuda")
        bl = -torch.rand((8, 60, 21), generator=g, device="cuda")
        lb = -torch.rand((8, 60, 20), generator=g, device="cuda")
        lens = torch.tensor([[60, 20 - i]] * 8, dtype=torch.int32, device="cuda")
        sets.append((x, w, dy, bl, lb, lens))

    def step(s, stream=None):
        x, w, dy, bl, lb, lens = s
        gr = tbs.linear_backward(dy, x, w, pre=dy, activation="silu", stream=stream)
        return [tbs.linear(x, w, activation="gelu", stream=stream), gr.x, gr.weight, gr.bias,
                tbs.adjust_logits(dy, normalize=True, stream=stream),
                *tbs.transducer_gradient("standard", bl, lb, lens, stream=stream)]

    want = [step(s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for _ in range(10):
        for s, st in zip(sets, streams):
            got.append(step(s, st))
    torch.cuda.synchronize()
    for i, out in enumerate(got):
        for a, b in zip(out, want[i % 2]):
            assert torch.equal(a, b)
