"""Performance cases of the operators around the joiner: linear layers with a fused epilogue
and their gradients, adjusted logits, and the gradient of the transducer losses.

listed()  the named cases; draw(rng) gives more of the same ranges.
prepare(case, seed)  the inputs on the GPU; run(state) one pass: through
``paper_2211_00484_amd.tbs`` where ``own`` is true, else in elementary torch operations.
work(case)  bytes and operations a pass cannot do without.
exact(case, seed)  the same outputs in 64 bits.
"""
import math

import numpy as np
import torch

own = False
DEV = "cuda"

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZES = {"fp32": 4, "bf16": 2, "fp16": 2}


# ---------------------------------------------------------------------------
# the cases

def _linear(M, K, N, dtype, act, res, pre=False, **more):
    return dict(kind="linear", M=M, K=K, N=N, dtype=dtype, act=act, res=res, pre=pre, **more)


def _grad(M, K, N, dtype, act, **more):
    return dict(kind="linear_grad", M=M, K=K, N=N, dtype=dtype, act=act, **more)


def _adjust(R, V, dtype, L, graph, bits, normalize, **more):
    return dict(kind="adjust", R=R, V=V, dtype=dtype, L=L, graph=graph, bits=bits,
                normalize=normalize, **more)


def _loss(form, B, T, lo, U, ulo, **more):
    return dict(kind="loss", form=form, B=B, T=T, lo=lo, U=U, ulo=ulo, **more)


def listed():
    return [
        # one frame of four live streams through the output layer: launch latency
        _linear(4, 512, 500, "bf16", "none", "none", name="output_step"),
        # the encoder projection of a joiner, batch of 32 utterances of 10 s, in training
        # (the pre-activation is kept): tanh(enc We' + be + dec)
        _linear(8000, 384, 512, "fp32", "tanh", "before", pre=True, name="project_batch"),
        # logits of 6,000 joiner rows over 5,000 word pieces
        _linear(6000, 512, 5000, "bf16", "none", "none", name="output_vocab"),
        # the second half of a feed-forward block over a full offline batch, added to its input
        _linear(64000, 2048, 512, "fp16", "none", "after", name="feed_forward"),
        # training: the output layer's gradients over five labels around the alignment per frame
        _grad(40000, 512, 500, "bf16", "none", name="output_grad"),
        # training: the projection's gradients
        _grad(8000, 384, 512, "fp32", "tanh", name="project_grad"),
        # live decoding: 32 streams of 4 contexts, all of history, bias and a decoding graph
        _adjust(128, 500, "fp32", 80, 5000, False, True, name="adjust_step"),
        # a large vocabulary with a large decoding graph
        _adjust(2048, 5000, "fp32", 120, 200_000, False, True, name="adjust_large"),
        # the largest vocabulary, bit masks, long histories, 16-bit logits left unnormalised
        _adjust(512, 46340, "bf16", 2000, 0, True, False, name="adjust_vocab"),
        # loss gradient of one long utterance: latency
        _loss("constrained", 1, 1000, 1000, 150, 150, name="loss_long"),
        # loss gradient of a training batch of 10 s utterances
        _loss("modified", 32, 250, 125, 80, 40, name="loss_batch"),
        # the same of a large batch, with the standard recursion
        _loss("standard", 1024, 250, 125, 80, 40, name="loss_large"),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(["linear", "linear_grad", "adjust", "loss"])
        dtype = rng.choice(["fp32", "bf16", "fp16"])
        if kind in ("linear", "linear_grad"):
            M = _logint(rng, 1, 64000)
            K = rng.choice([rng.randint(32, 2048), 256, 512, 640, _logint(rng, 32, 2048)])
            N = rng.choice([_logint(rng, 16, 5000), 500, 512])
            act = rng.choice(["none", "relu", "tanh", "silu", "gelu"])
            if kind == "linear":
                c = _linear(M, K, N, dtype, act, rng.choice(["none", "before", "after"]),
                            rng.random() < 0.3)
                cost = 2.0 * M * K * N
            else:
                c = _grad(M, K, N, dtype, act)
                cost = 4.0 * M * K * N
            if cost <= (1.0e11 if dtype != "fp32" else 2.0e10):
                return c
        elif kind == "adjust":
            c = _adjust(_logint(rng, 1, 4096), _logint(rng, 16, 46340), dtype,
                        rng.choice([0, _logint(rng, 1, 2000)]),
                        rng.choice([0, _logint(rng, 10, 200_000)]), rng.random() < 0.5,
                        rng.random() < 0.5)
            if c["R"] * c["V"] <= 20_000_000:
                return c
        else:
            T, U = _logint(rng, 1, 1000), _logint(rng, 1, 200)
            c = _loss(rng.choice(["standard", "modified", "constrained"]), _logint(rng, 1, 1024),
                      T, max(1, T // 2), U, U // 2)
            if c["B"] * T * U <= 20_000_000:
                return c


# ---------------------------------------------------------------------------
# inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _randn(g, *shape, scale=1.0):
    return torch.randn(shape, generator=g, device=DEV) * scale


def _graph_csr(case, seed):
    """A decoding graph of ``graph`` states, five arcs a state on average, a few states (the
    word-start states of a lexicon) with hundreds."""
    rng = np.random.default_rng(seed)
    S, V = case["graph"], case["V"]
    deg = np.minimum((rng.pareto(1.5, size=S) * 3 + 1).astype(np.int64), min(V - 1, 1500))
    rp = np.zeros(S + 1, np.int64)
    np.cumsum(deg, out=rp[1:])
    A = int(rp[-1])
    return (rp.astype(np.int32), rng.integers(0, S, A, dtype=np.int32),
            rng.integers(1, V, A, dtype=np.int32),
            np.log(rng.uniform(0.01, 1.0, A)).astype(np.float32))


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}
    if case["kind"] in ("linear", "linear_grad"):
        M, K, N, dt = case["M"], case["K"], case["N"], DTYPES[case["dtype"]]
        s["x"] = _randn(g, M, K).to(dt)
        s["w"] = _randn(g, N, K, scale=K ** -0.5).to(dt)
        s["b"] = _randn(g, N, scale=0.1).to(dt)
        if case["kind"] == "linear":
            s["res"] = _randn(g, M, N).to(dt) if case["res"] != "none" else None
        else:
            s["dy"] = _randn(g, M, N, scale=1e-2).to(dt)
            s["pre"] = None if case["act"] == "none" else _randn(g, M, N).to(dt)
    elif case["kind"] == "adjust":
        R, V, L = case["R"], case["V"], case["L"]
        z = _randn(g, R, V, scale=2.0)
        z[:, 0] += 4.0  # blank leads on most frames
        s["logits"] = z.to(DTYPES[case["dtype"]])
        s["bias"] = torch.where(torch.rand(V, generator=g, device=DEV) < 0.05, 1.5, 0.0)
        s["history"] = s["hlen"] = s["pen"] = None
        if L:
            # frequent labels first, as word pieces are
            u = torch.rand((R, L), generator=g, device=DEV, dtype=torch.float64)
            s["hlen"] = torch.randint(0, L + 1, (R,), generator=g, device=DEV, dtype=torch.int32)
            tok = 1 + ((V - 1) * u * u).to(torch.int32).clamp_(max=V - 2)
            pad = torch.arange(L, device=DEV)[None, :] >= s["hlen"][:, None]
            s["history"] = tok.masked_fill_(pad, -1)
            s["pen"] = torch.stack([1.0 + 0.3 * torch.rand(R, generator=g, device=DEV),
                                    0.5 * torch.rand(R, generator=g, device=DEV),
                                    0.2 * torch.rand(R, generator=g, device=DEV)], 1).contiguous()
        s["allowed"] = None
        if case["bits"]:
            s["allowed"] = torch.randint(-2 ** 31, 2 ** 31, (R, (V + 31) // 32), generator=g,
                                         device=DEV, dtype=torch.int64).to(torch.int32)
        s["graph"] = s["states"] = None
        if case["graph"]:
            csr = _graph_csr(case, seed)
            s["states"] = torch.randint(-1, case["graph"], (R,), generator=g, device=DEV,
                                        dtype=torch.int32)
            if own:
                from paper_2211_00484_amd import tbs
                s["graph"] = tbs.Graph.from_csr(case["graph"], 0, V, *csr)
            else:
                s["graph"] = (torch.from_numpy(csr[0]).to(DEV), torch.from_numpy(csr[2]).to(DEV),
                              int(np.max(np.diff(csr[0]))))
    else:
        B, T, U = case["B"], case["T"], case["U"]
        fr = torch.randint(case["lo"], T + 1, (B,), generator=g, device=DEV)
        lab = torch.randint(case["ulo"], U + 1, (B,), generator=g, device=DEV)
        fr[0], lab[0] = T, U
        if case["form"] != "standard":
            lab = torch.minimum(lab, fr)  # a label moves to the next frame
        s["lengths"] = torch.stack([fr, lab], 1).to(torch.int32).contiguous()
        # label u + 1 is likely around its frame, less so away from it; blank takes the rest
        t = torch.arange(T, device=DEV)[None, :, None]
        u = torch.arange(U + 1, device=DEV)[None, None, :]
        at = (u + 0.5) * fr[:, None, None] / (lab[:, None, None] + 1.0)
        score = 3.0 - 0.3 * (t - at).abs() + _randn(g, B, T, U + 1)
        s["blank"] = torch.nn.functional.logsigmoid(-score).contiguous()
        s["label"] = (torch.nn.functional.logsigmoid(score[:, :, :U])
                      - 0.2 * torch.rand((B, T, U), generator=g, device=DEV)).contiguous()
        s["weights"] = torch.full((B,), -1.0 / B, dtype=torch.float64, device=DEV)
    return s


# ---------------------------------------------------------------------------
# one pass

def run(s):
    c = s["case"]
    if own:
        return _RUN_OWN[c["kind"]](c, s)
    return _RUN_PLAIN[c["kind"]](c, s)


def _own_linear(c, s):
    from paper_2211_00484_amd import tbs
    r = tbs.linear(s["x"], s["w"], s["b"], residual=s["res"], activation=c["act"],
                   residual_after=c["res"] == "after", want_pre=c["pre"])
    return {"out": r[0], "pre": r[1]} if c["pre"] else {"out": r}


def _own_grad(c, s):
    from paper_2211_00484_amd import tbs
    act = c["act"] != "none"
    r = tbs.linear_backward(s["dy"], s["x"], s["w"], pre=s["pre"], activation=c["act"],
                            want_pre=act)
    out = {"x": r.x, "weight": r.weight, "bias": r.bias}
    if act:
        out["pre"] = r.pre
    return out


def _own_adjust(c, s):
    from paper_2211_00484_amd import tbs
    return tbs.adjust_logits(s["logits"], history=s["history"], history_lengths=s["hlen"],
                             row_penalties=s["pen"], bias=s["bias"], allowed=s["allowed"],
                             graph=s["graph"], states=s["states"], normalize=c["normalize"])


def _own_loss(c, s):
    from paper_2211_00484_amd import tbs
    total, gb, gl, status = tbs.transducer_gradient(c["form"], s["blank"], s["label"],
                                                    s["lengths"], weights=s["weights"])
    return {"total": total, "blank": gb, "label": gl, "status": status}


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "tanh":
        return torch.tanh(z)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "tanh":
        return 1 - torch.tanh(z) ** 2
    if act == "silu":
        sg = 1 / (1 + torch.exp(-z))
        return sg * (1 + z * (1 - sg))
    return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (
        1 / math.sqrt(2 * math.pi))


def _plain_linear(c, s):
    dt = DTYPES[c["dtype"]]
    z = s["x"].float() @ s["w"].float().t() + s["b"].float()
    if c["res"] == "before":
        z = z + s["res"].float()
    y = _act(z, c["act"])
    if c["res"] == "after":
        y = y + s["res"].float()
    out = {"out": y.to(dt)}
    if c["pre"]:
        out["pre"] = z.to(dt)
    return out


def _plain_grad(c, s):
    dt = DTYPES[c["dtype"]]
    dz = s["dy"].float()
    if c["act"] != "none":
        dz = dz * _act_slope(s["pre"].float(), c["act"])
    out = {"x": (dz @ s["w"].float()).to(dt), "weight": (dz.t() @ s["x"].float()).to(dt),
           "bias": dz.sum(0).to(dt)}
    if c["act"] != "none":
        out["pre"] = dz.to(dt)
    return out


def _plain_adjust(c, s):
    z = s["logits"].float()
    R, V = z.shape
    if s["history"] is not None:
        h = s["history"].long()
        ok = (torch.arange(h.shape[1], device=DEV)[None, :] < s["hlen"][:, None]) & (h >= 0) & (h < V)
        cnt = torch.zeros((R, V + 1), device=DEV)
        cnt.scatter_add_(1, torch.where(ok, h, V), ok.float())
        cnt = cnt[:, :V]
        rep, pres, freq = (s["pen"][:, i:i + 1] for i in range(3))
        seen = torch.where(z > 0, z / rep, z * rep) - pres - freq * cnt
        z = torch.where(cnt > 0, seen, z)
    z = z + s["bias"]
    if s["allowed"] is not None:
        col = torch.arange(V, device=DEV)
        bit = (s["allowed"][:, col // 32] >> (col % 32)) & 1
        z = torch.where(bit != 0, z, -math.inf)
    if s["graph"] is not None:
        rp, label, maxdeg = s["graph"]
        st = s["states"].long()
        lo, hi = rp[st.clamp(min=0)].long(), rp[st.clamp(min=0) + 1].long()
        at = lo[:, None] + torch.arange(maxdeg, device=DEV)[None, :]
        lab = torch.where(at < hi[:, None], label[at.clamp(max=label.numel() - 1)].long(), 0)
        can = torch.zeros((R, V), dtype=torch.bool, device=DEV)
        can.scatter_(1, lab, True)
        can[:, 0] = True  # blank keeps the state
        z = torch.where(can | (st < 0)[:, None], z, -math.inf)
    if c["normalize"]:
        m = z.amax(1, keepdim=True)
        m = torch.where(m == -math.inf, 0.0, m)
        z = z - (m + torch.log(torch.exp(z - m).sum(1, keepdim=True)))
        z = torch.where(torch.isnan(z), -math.inf, z)  # a row whose masks leave nothing
    return z.to(DTYPES[c["dtype"]])


def _shift(x, fill=-math.inf):
    """x one place to the right along the last axis."""
    return torch.cat([torch.full_like(x[..., :1], fill), x[..., :-1]], -1)


def _plain_loss(c, s):
    """alpha and beta in 64 bits (the occupancies are exponentials of differences of long
    sums); eq. (1) along the diagonals t + u."""
    B, T, U = c["B"], c["T"], c["U"]
    blank, label = s["blank"].double(), s["label"].double()
    Tb, Ub = s["lengths"][:, 0].long(), s["lengths"][:, 1].long()
    inf = math.inf
    lab1 = torch.cat([label, torch.full((B, T, 1), -inf, dtype=torch.float64, device=DEV)], 2)
    t = torch.arange(T, device=DEV)[None, :, None]
    u = torch.arange(U + 1, device=DEV)[None, None, :]
    last = torch.arange(U + 1, device=DEV)[None, :] == Ub[:, None]
    inside = (t < Tb[:, None, None]) & (u <= Ub[:, None, None])
    blank = torch.where(inside, blank, -inf)
    lab1 = torch.where(inside & (u < Ub[:, None, None]), lab1, -inf)
    if c["form"] == "standard":
        # cell (t, u) on row s = t + u of a skewed grid, frames along it
        S = T + U
        ss = torch.arange(S, device=DEV)[:, None]
        tt = torch.arange(T, device=DEV)[None, :]
        uu = ss - tt
        at = torch.where((uu >= 0) & (uu <= U), tt * (U + 1) + uu, T * (U + 1))
        end = torch.full((B, 1), -inf, dtype=torch.float64, device=DEV)
        skew = lambda x: torch.cat([x.reshape(B, -1), end], 1)[:, at]
        bl, lb = skew(blank), skew(lab1)
        a = torch.empty((B, S, T), dtype=torch.float64, device=DEV)
        a[:, 0] = -inf
        a[:, 0, 0] = 0.0
        for i in range(1, S):
            a[:, i] = torch.logaddexp(_shift(a[:, i - 1] + bl[:, i - 1]), a[:, i - 1] + lb[:, i - 1])
        fin = (tt == (Tb - 1)[:, None, None]) & ((uu[None] == Ub[:, None, None]))
        b = torch.full((B, S + 1, T + 1), -inf, dtype=torch.float64, device=DEV)
        for i in range(S - 1, -1, -1):
            v = torch.logaddexp(bl[:, i] + b[:, i + 1, 1:], lb[:, i] + b[:, i + 1, :T])
            b[:, i, :T] = torch.where(fin[:, i], bl[:, i], v)
        total = b[:, 0, 0]
        z = total[:, None, None]
        nextb = torch.where(fin, 0.0, b[:, 1:, 1:])
        gb, gl = torch.exp(a + bl + nextb - z), torch.exp(a + lb + b[:, 1:, :T] - z)
        t2 = torch.arange(T, device=DEV)[:, None]
        back = t2 + torch.arange(U + 1, device=DEV)[None, :]
        gb, gl = gb[:, back, t2], gl[:, back, t2]
    else:
        con = c["form"] == "constrained"
        a = torch.empty((B, T + 1, U + 1), dtype=torch.float64, device=DEV)
        a[:, 0] = -inf
        a[:, 0, 0] = 0.0
        nb = torch.cat([blank[:, :, 1:], torch.full_like(blank[:, :, :1], -inf)], 2)
        arc = lab1 + nb if con else lab1  # weight of the arc that emits label u + 1
        for i in range(T):
            a[:, i + 1] = torch.logaddexp(a[:, i] + blank[:, i], _shift(a[:, i] + arc[:, i]))
        b = torch.full((B, T + 1, U + 2), -inf, dtype=torch.float64, device=DEV)
        for i in range(T, -1, -1):
            if i < T:
                b[:, i, :U + 1] = torch.logaddexp(blank[:, i] + b[:, i + 1, :U + 1],
                                                  arc[:, i] + b[:, i + 1, 1:])
            b[:, i, :U + 1] = torch.where(last & (Tb == i)[:, None], 0.0, b[:, i, :U + 1])
        total = b[:, 0, 0]
        z = total[:, None, None]
        gb = torch.exp(a[:, :T] + blank + b[:, 1:, :U + 1] - z)
        gl = torch.exp(a[:, :T] + arc + b[:, 1:, 1:] - z)
        if con:
            gb = gb + _shift(gl, 0.0)
    w = s["weights"][:, None, None]
    reach = (total > -inf)[:, None, None]
    return {"total": total, "blank": torch.where(reach, w * gb, 0.0).float(),
            "label": torch.where(reach, w * gl, 0.0)[:, :, :U].float().contiguous(),
            "status": torch.zeros(B, dtype=torch.int32, device=DEV)}


_RUN_OWN = {"linear": _own_linear, "linear_grad": _own_grad, "adjust": _own_adjust,
            "loss": _own_loss}
_RUN_PLAIN = {"linear": _plain_linear, "linear_grad": _plain_grad, "adjust": _plain_adjust,
              "loss": _plain_loss}


# ---------------------------------------------------------------------------
# unavoidable work

def work(case):
    c = case
    if c["kind"] == "linear":
        M, K, N = c["M"], c["K"], c["N"]
        outs = 1 + (c["res"] != "none") + bool(c["pre"])
        return {"bytes": SIZES[c["dtype"]] * (M * K + N * K + N + outs * M * N),
                "flops": 2 * M * N * K}
    if c["kind"] == "linear_grad":
        M, K, N = c["M"], c["K"], c["N"]
        mats = 3 if c["act"] != "none" else 1  # dy; the pre-activation and its gradient
        return {"bytes": SIZES[c["dtype"]] * (2 * M * K + 2 * N * K + N + mats * M * N),
                "flops": 4 * M * N * K}
    if c["kind"] == "adjust":
        R, V = c["R"], c["V"]
        more = 4 * V + (R * (c["L"] * 2 + 16) if c["L"] else 0)
        more += R * ((V + 31) // 32) * 4 if c["bits"] else 0
        more += R * (12 + 5 * 4) if c["graph"] else 0
        return {"bytes": 2 * SIZES[c["dtype"]] * R * V + more,
                "flops": (8 if c["normalize"] else 4) * R * V}
    frames, labels = 0.5 * (c["lo"] + c["T"]), 0.5 * (c["ulo"] + c["U"])
    inside = c["B"] * frames * (2 * labels + 1)  # cells that are read
    whole = c["B"] * c["T"] * (2 * c["U"] + 1)   # and written
    return {"bytes": int(4 * inside + 4 * whole), "flops": int(10 * inside)}


# ---------------------------------------------------------------------------
# the same outputs in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    c = case
    if c["kind"] == "linear":
        z = torch.addmm(s["b"].double(), s["x"].double(), s["w"].double().t().contiguous())
        if c["res"] == "before":
            z += s["res"].double()
        f = {"none": lambda v: v, "relu": torch.relu, "tanh": torch.tanh,
             "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}[c["act"]]
        y = f(z)
        if c["res"] == "after":
            y = y + s["res"].double()
        return {"out": y, "pre": z} if c["pre"] else {"out": y}
    if c["kind"] == "linear_grad":
        dy = s["dy"].double()
        if c["act"] == "none":
            dz = dy
        else:
            p = s["pre"].double().requires_grad_(True)
            f = {"relu": torch.relu, "tanh": torch.tanh, "silu": torch.nn.functional.silu,
                 "gelu": torch.nn.functional.gelu}[c["act"]]
            dz, = torch.autograd.grad(f(p), p, dy)
        out = {"x": dz @ s["w"].double(), "weight": dz.t().contiguous() @ s["x"].double(),
               "bias": dz.sum(0)}
        if c["act"] != "none":
            out["pre"] = dz
        return out
    if c["kind"] == "adjust":
        return _exact_adjust(c, s, seed)
    return _exact_loss(c, s)


def _exact_adjust(c, s, seed):
    R, V = c["R"], c["V"]
    z = s["logits"].double().cpu().numpy()
    if s["history"] is not None:
        hist, hlen = s["history"].cpu().numpy(), s["hlen"].cpu().numpy()
        pen = s["pen"].double().cpu().numpy()
        for r in range(R):
            lab, cnt = np.unique(hist[r, :hlen[r]], return_counts=True)
            v = z[r, lab]
            v = np.where(v > 0, v / pen[r, 0], v * pen[r, 0])
            z[r, lab] = v - pen[r, 1] - pen[r, 2] * cnt
    z += s["bias"].double().cpu().numpy()[None, :]
    if s["allowed"] is not None:
        words = np.ascontiguousarray(s["allowed"].cpu().numpy()).view(np.uint8)
        bits = np.unpackbits(words, axis=1, bitorder="little")[:, :V]
        z[bits == 0] = -np.inf
    if c["graph"]:
        rp, _, label, _ = _graph_csr(c, seed)
        states = s["states"].cpu().numpy()
        for r in range(R):
            if states[r] >= 0:
                keep = np.zeros(V, bool)
                keep[0] = True
                keep[label[rp[states[r]]:rp[states[r] + 1]]] = True
                z[r, ~keep] = -np.inf
    z = torch.from_numpy(z).to(DEV)
    if c["normalize"]:
        lse = torch.logsumexp(z, 1, keepdim=True)
        z = torch.where(lse == -math.inf, z, z - lse)
    return z


def _exact_loss(c, s):
    """The log-likelihood by its recursion, row by row, and its derivative by automatic
    differentiation; -1e30 stands for an impossible cell, so that no term is NaN."""
    B, T, U = c["B"], c["T"], c["U"]
    low = -1e30
    blank = s["blank"].double().requires_grad_(True)
    label = s["label"].double().requires_grad_(True)
    Tb, Ub = s["lengths"][:, 0].long(), s["lengths"][:, 1].long()
    rows = torch.arange(B, device=DEV)
    wall = torch.full((B, 1), low, dtype=torch.float64, device=DEV)
    a = torch.full((B, U + 1), low, dtype=torch.float64, device=DEV)
    a[:, 0] = 0.0
    keep = []
    if c["form"] == "standard":
        zero = torch.zeros((B, 1), dtype=torch.float64, device=DEV)
        for t in range(T):
            run_ = torch.cat([zero, torch.cumsum(label[:, t], 1)], 1)
            come = a if t == 0 else a + blank[:, t - 1]
            a = run_ + torch.logcumsumexp(come - run_, 1)
            keep.append(a)
        total = torch.stack(keep, 1)[rows, Tb - 1, Ub] + blank[rows, Tb - 1, Ub]
    else:
        for t in range(T):
            up = torch.cat([wall, a[:, :U] + label[:, t]], 1)
            if c["form"] == "constrained":
                up = up + blank[:, t]
            a = torch.logaddexp(a + blank[:, t], up)
            keep.append(a)
        total = torch.stack(keep, 1)[rows, Tb - 1, Ub]
    gb, gl = torch.autograd.grad(total, [blank, label], s["weights"])
    total = total.detach()
    none = total < 0.5 * low
    gb[none], gl[none], total[none] = 0.0, 0.0, -math.inf
    return {"total": total, "blank": gb, "label": gl, "status": None}
