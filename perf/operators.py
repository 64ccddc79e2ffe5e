"""What is measured of the output layers and the beam search: each operator in its plain
form (elementary torch operations, in 32 bits), the calls a user makes of the library, and
the definition in 64 bits.

Sizes come from the repository's own workloads (the outputs of parser-scale StackLSTMs with
H = 200, 64 sentences and up to 185 transitions; of a decoder-like one with H = 1024; the
parser's 600 -> 200 state layer; the toy fp32 ones), with generic sizes for what the
repository has no workload of: label sets of 83 transitions, a vocabulary of 32003 words,
beams of up to 16.
"""
from __future__ import annotations

import math

import torch

own = False  # False: the plain forms; True: the library's calls

ACTS = ("none", "relu", "tanh", "gelu", "silu")


# ------------------------------------------------------------------------------- cases
def _norm(name, dtype, R, N, call):
    return dict(name=name, kind="norm", dtype=dtype, R=R, N=N, call=call)


def _linear(name, dtype, R, K, N, call, act="none", res=False, pre=False):
    return dict(name=name, kind="linear", dtype=dtype, R=R, K=K, N=N, call=call, act=act, res=res, pre=pre)


def _distill(name, dtype, R, V, k, tau, alpha):
    return dict(name=name, kind="distill", dtype=dtype, R=R, V=V, k=k, tau=tau, alpha=alpha)


def _beam(name, dtype, B, K, V, S, H):
    return dict(name=name, kind="beam", dtype=dtype, B=B, K=K, V=V, S=S, H=H)


def listed():
    return [
        # five hypotheses of one sentence, one step of decoding: the tops normalised; latency alone
        _norm("norm_step5", "fp32", 5, 100, "forward"),
        # a training step of a parser: every output of 64 sentences, forward and backward
        _norm("norm_train64", "bf16", 185 * 64, 200, "train"),
        # the same of a wide decoder-like model, 256 instances of 256 steps
        _norm("norm_train256", "bf16", 256 * 256, 1024, "train"),
        # one step of a beam of 8 over the words: bound by the weights
        _linear("words_step8", "bf16", 8, 1024, 32003, "forward"),
        # a hidden layer with its residual over the same outputs as norm_train256, its backward's
        # input kept
        _linear("hidden_train256", "bf16", 256 * 256, 1024, 1024, "forward", "gelu", True, True),
        # the backward of the word layer for a batch of 4096 tops
        _linear("words_back4096", "bf16", 4096, 1024, 32003, "backward"),
        # a full-precision parser state layer: the backward over 64 sentences
        _linear("state_back_fp32", "fp32", 185 * 64, 600, 200, "backward", "relu"),
        # labelled transitions of a full-precision parser learnt from a teacher's eight best
        _distill("labels_train64", "fp32", 185 * 64, 83, 8, 2.0, 0.75),
        # words learnt from a teacher's 32 best, 4096 tops
        _distill("words_train4096", "bf16", 4096, 32003, 32, 1.5, 0.5),
        # the normalisers of 512 hypotheses' words before a step of the search
        dict(name="normaliser512", kind="lse", dtype="bf16", B=64, K=8, V=32003),
        # one sentence decoded online with a beam of 8 labelled transition sequences
        _beam("beam_sentence", "fp32", 1, 8, 83, 121, 200),
        # 64 sentences, 8 hypotheses each, over the words, deep stacks
        _beam("beam_words64", "bf16", 64, 8, 32003, 186, 200),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ranges; sizes are spread over their logarithm, and half of
    the widths are multiples of 8."""
    kind = rng.choice(("norm", "linear", "linear", "distill", "beam", "lse"))
    dtype = rng.choice(("bf16", "bf16", "fp32"))
    even = lambda n: max(8, n // 8 * 8) if rng.random() < 0.5 else n
    if kind == "norm":
        N = even(_log(rng, 8, 2048))
        c = _norm(None, dtype, _log(rng, 1, min(65536, (1 << 25) // N)), N, rng.choice(("forward", "train")))
    elif kind == "linear":
        K, N = even(_log(rng, 16, 2048)), even(_log(rng, 16, 32003))
        most = (1 << 35) // (K * N) if dtype == "bf16" else (1 << 33) // (K * N)
        call = rng.choice(("forward", "backward"))
        c = _linear(None, dtype, _log(rng, 1, max(1, min(65536, most, (1 << 28) // N))), K, N, call, rng.choice(ACTS),
                    rng.random() < 0.5, call == "forward" and rng.random() < 0.5)
    elif kind == "distill":
        V = even(_log(rng, 8, 32003))
        c = _distill(None, dtype, _log(rng, 1, min(32768, (1 << 26) // V)), V, _log(rng, 1, min(64, V)),
                     rng.choice((1.0, 1.5, 2.0, 4.0)), rng.choice((0.5, 0.75, 1.0)))
    elif kind == "lse":
        V = even(_log(rng, 8, 32003))
        K = _log(rng, 1, 16)
        c = dict(kind="lse", dtype=dtype, B=_log(rng, 1, max(1, min(1024, (1 << 25) // (V * K)))), K=K, V=V)
    else:
        K, V, H, S = _log(rng, 1, 16), even(_log(rng, 8, 32003)), 8 * _log(rng, 4, 128), rng.randint(2, 186)
        most = min((1 << 23) // (K * V), (1 << 24) // (K * S * H))
        c = _beam(None, dtype, _log(rng, 1, max(1, min(256, most))), K, V, S, H)
    c.pop("name", None)
    return c


# ------------------------------------------------------------------------------ inputs
def _dt(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * seed + 17)
    randn = lambda *s: torch.randn(*s, device="cuda", generator=g)
    rand = lambda *s: torch.rand(*s, device="cuda", generator=g)
    ints = lambda hi, *s: torch.randint(0, hi, s, device="cuda", generator=g)
    dt, s = _dt(case), {}
    if case["kind"] == "norm":
        R, N = case["R"], case["N"]
        # StackLSTM outputs: o tanh(c), within (-1, 1), rows of different scale
        s["x"] = (torch.tanh(randn(R, N)) * (0.2 + 0.8 * rand(R, 1))).to(dt)
        s["gamma"], s["beta"], s["eps"] = 1 + 0.1 * randn(N), 0.1 * randn(N), 1e-5
        if case["call"] == "train":
            s["dy"] = randn(R, N) / R
    elif case["kind"] == "linear":
        R, K, N = case["R"], case["K"], case["N"]
        s["x"], s["W"], s["bias"] = randn(R, K).to(dt), (randn(N, K) / math.sqrt(K)).to(dt), 0.1 * randn(N)
        s["residual"] = randn(R, N).to(dt) if case["res"] and case["call"] == "forward" else None
        if case["call"] == "backward":
            s["dy"] = randn(R, N) / R
            s["pre"] = randn(R, N).to(dt) if case["act"] != "none" else None
            s["add"] = randn(R, K) / R if case["res"] else None
    elif case["kind"] == "distill":
        R, V, k = case["R"], case["V"], case["k"]
        z = 2 * randn(R, V)
        # the teacher agrees with the student in part; its best are anywhere in the vocabulary
        t = z.gather(1, ints(V, R, k))
        s["t_idx"] = torch.argsort(rand(R, V), 1)[:, :k].to(torch.int32).contiguous() if V <= 1024 else ints(V, R, k).to(torch.int32)
        s["t_logit"] = (0.5 * t + 2 * randn(R, k)).contiguous()
        s["gold"] = ints(V, R).to(torch.int32)
        if V <= 1024:  # transitions that a state does not allow
            bad = rand(R, V) < 0.1
            bad.scatter_(1, s["gold"].long()[:, None], False).scatter_(1, s["t_idx"].long(), False)
            z = z.masked_fill(bad, -math.inf)
        s["t_idx"][rand(R, k) < 0.05] = -1  # teachers that gave fewer than k
        pad = rand(R) < 0.1  # padding after the end of a sentence
        s["t_idx"][pad] = -1
        s["gold"][pad] = -1
        s["logits"], s["scale"] = z.to(dt), 1.0 / R
    else:
        B, K, V = case["B"], case["K"], case["V"]
        z = 2 * randn(B, K, V)
        z = z.masked_fill(rand(B, K, V) < 0.05, -math.inf)
        s["logits"] = z.to(dt)
        if case["kind"] == "beam":
            S, H = case["S"], case["H"]
            s["lse"] = torch.logsumexp(s["logits"].float(), 2)
            s["score"] = -20 * rand(B, K)
            s["score"][rand(B, K) < 0.05] = -math.inf  # beams that the first steps have not filled
            s["done"] = (rand(B, K) < 0.1).to(torch.uint8)
            s["p"] = ints(S, B * K).to(torch.int32)
            s["h"], s["c"] = torch.tanh(randn(S, B * K, H)).to(dt), randn(S, B * K, H)
            s["h_new"], s["c_new"] = torch.zeros_like(s["h"]), torch.zeros_like(s["c"])
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if not own:
        return s
    from paper_1904_03409_gb300 import binding as bd

    dt, kind = _dt(case), case["kind"]
    dev = s["x" if "x" in s else "logits"].device
    e = lambda *n, d=torch.float32: torch.empty(*n, dtype=d, device=dev)
    ldt = bd.SL_BF16 if case["dtype"] == "bf16" else bd.SL_FP32
    if kind == "norm":
        R, N = case["R"], case["N"]
        s["op"] = bd.stacklstm_norm_create(R, N, ldt, dev.index)
        s["y"], s["mean"], s["rstd"] = e(R, N, d=dt), e(R), e(R)
        if case["call"] == "train":
            s["dx"], s["dgamma"], s["dbeta"] = e(R, N), e(N), e(N)
    elif kind == "linear":
        R, K, N = case["R"], case["K"], case["N"]
        s["op"] = bd.stacklstm_linear_create(R, K, N, ldt, ACTS.index(case["act"]), dev.index)
        if case["call"] == "forward":
            s["y"], s["pre"] = e(R, N, d=dt), e(R, N, d=dt) if case["pre"] else None
        else:
            s["dx"], s["dW"], s["dbias"] = e(R, K), e(N, K), e(N)
    elif kind == "distill":
        s["op"] = bd.stacklstm_distill_create(case["R"], case["V"], case["k"], ldt, dev.index)
        s["loss"], s["dlogits"] = e(case["R"]), e(case["R"], case["V"])
    else:
        B, K = case["B"], case["K"]
        S, H = case.get("S", 1), case.get("H", 8)
        s["op"] = bd.stacklstm_beam_create(B, K, case["V"], S, H, ldt, dev.index)
        if kind == "lse":
            s["lse_new"] = e(B, K)
        else:
            s["score_new"], s["parent"], s["token"] = e(B, K), e(B, K, d=torch.int32), e(B, K, d=torch.int32)
            s["p_new"], s["top_h"], s["top_c"] = e(B * K, d=torch.int32), e(B * K, H, d=dt), e(B * K, H)
    return s


# --------------------------------------------------------------- the library's calls
def _run_own(s):
    from paper_1904_03409_gb300 import binding as bd

    case, op = s["case"], s["op"]
    kind = case["kind"]
    if kind == "norm":
        bd.stacklstm_norm_forward(op, s["x"], s["gamma"], s["beta"], s["eps"], s["y"], s["mean"], s["rstd"])
        if case["call"] == "forward":
            return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
        bd.stacklstm_norm_backward(op, s["dy"], s["x"], s["gamma"], s["mean"], s["rstd"], s["dx"], s["dgamma"], s["dbeta"])
        return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"], "dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    if kind == "linear":
        if case["call"] == "forward":
            bd.stacklstm_linear_forward(op, s["x"], s["W"], s["bias"], s["residual"], s["y"], s["pre"])
            return {"y": s["y"], "pre": s["pre"]}
        bd.stacklstm_linear_backward(op, s["dy"], s["x"], s["W"], s["pre"], s["add"], s["dx"], s["dW"], s["dbias"])
        return {"dx": s["dx"], "dW": s["dW"], "dbias": s["dbias"]}
    if kind == "distill":
        bd.stacklstm_distill_run(op, s["logits"], s["t_idx"], s["t_logit"], s["gold"], case["tau"], case["alpha"], s["scale"],
                                 s["loss"], s["dlogits"])
        return {"loss": s["loss"], "dlogits": s["dlogits"]}
    if kind == "lse":
        bd.stacklstm_beam_lse(op, s["logits"], s["lse_new"])
        return {"lse": s["lse_new"]}
    bd.stacklstm_beam_select(op, s["logits"], s["lse"], s["score"], s["done"], s["score_new"], s["parent"], s["token"])
    bd.stacklstm_beam_reorder(op, s["parent"], s["p"], s["h"], s["c"], s["p_new"], s["h_new"], s["c_new"], s["top_h"], s["top_c"])
    return {k: s[k] for k in ("score_new", "parent", "token", "p_new", "h_new", "c_new", "top_h", "top_c")}


# ------------------------------------------------------------------ the plain forms
def _act(z, act):
    if act == "relu":
        return z.clamp_min(0)
    if act == "tanh":
        return torch.tanh(z)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).float()
    if act == "tanh":
        return 1 - torch.tanh(z) ** 2
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    sg = torch.sigmoid(z)
    return sg * (1 + z * (1 - sg))


def _log_softmax(z):
    m = z.amax(1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    return z - m - torch.log(torch.exp(z - m).sum(1, keepdim=True))


def _plain_norm(s, case):
    x, R, N = s["x"].float(), case["R"], case["N"]
    mean = x.mean(1)
    xc = x - mean[:, None]
    rstd = 1 / torch.sqrt((xc * xc).mean(1) + s["eps"])
    xh = xc * rstd[:, None]
    out = {"y": (xh * s["gamma"] + s["beta"]).to(_dt(case)), "mean": mean, "rstd": rstd}
    if case["call"] == "train":
        a = s["dy"] * s["gamma"]
        out["dx"] = rstd[:, None] * (a - a.mean(1, keepdim=True) - xh * (a * xh).mean(1, keepdim=True))
        out["dgamma"], out["dbeta"] = (s["dy"] * xh).sum(0), s["dy"].sum(0)
    return out


def _plain_linear(s, case):
    x, W = s["x"].float(), s["W"].float()
    if case["call"] == "forward":
        z = x @ W.T + s["bias"]
        y = _act(z, case["act"])
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return {"y": y.to(_dt(case)), "pre": z.to(_dt(case)) if case["pre"] else None}
    dz = s["dy"]
    if s["pre"] is not None:
        dz = dz * _act_grad(s["pre"].float(), case["act"])
    dx = dz @ W
    if s["add"] is not None:
        dx = dx + s["add"]
    return {"dx": dx, "dW": dz.T @ x, "dbias": dz.sum(0)}


def _plain_distill(s, case):
    z, tau, alpha, scale = s["logits"].float(), case["tau"], case["alpha"], s["scale"]
    here = s["t_idx"] >= 0
    idx = torch.where(here, s["t_idx"], torch.zeros_like(s["t_idx"])).long()
    some = here.any(1)
    t = torch.where(here, s["t_logit"] / tau, torch.full_like(s["t_logit"], -math.inf))
    lq = _log_softmax(torch.where(some[:, None], t, torch.zeros_like(t)))
    q = torch.where(here, torch.exp(lq), torch.zeros_like(lq))
    lp = _log_softmax(z / tau)
    kl = torch.where(q > 0, q * (lq - lp.gather(1, idx)), torch.zeros_like(q)).sum(1) * (alpha * tau * tau)
    lP = _log_softmax(z)
    has = s["gold"] >= 0
    gold = torch.where(has, s["gold"], torch.zeros_like(s["gold"])).long()
    ce = torch.where(has, -lP.gather(1, gold[:, None])[:, 0], torch.zeros_like(kl)) * (1 - alpha)
    d = (alpha * tau * some)[:, None] * torch.exp(lp) + ((1 - alpha) * has)[:, None] * torch.exp(lP)
    d.scatter_add_(1, idx, -alpha * tau * q)
    d.scatter_add_(1, gold[:, None], -(1 - alpha) * has[:, None].float())
    return {"loss": scale * (kl + ce), "dlogits": scale * d}


def _plain_lse(s, case):
    z = s["logits"].float()
    m = z.amax(2)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    return {"lse": m + torch.log(torch.exp(z - m[..., None]).sum(2))}


def _plain_beam(s, case):
    B, K, V, S = case["B"], case["K"], case["V"], case["S"]
    low = torch.iinfo(torch.int64).min
    cand = s["score"][..., None] + (s["logits"].float() - s["lse"][..., None])
    done = s["done"] != 0
    cand = torch.where(done[..., None], torch.full_like(cand, -math.inf), cand)
    cand[..., 0] = torch.where(done, s["score"], cand[..., 0])
    cand = cand.view(B, K * V) + 0.0
    # one integer a candidate: the score's order above, the lowest place first below
    bits = cand.view(torch.int32)
    order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long()
    place = torch.arange(K * V, device=cand.device)
    key = torch.where(cand > -math.inf, (order << 32) | (0xFFFFFFFF - place), torch.full_like(order, low))
    best = key.topk(K, 1, largest=True, sorted=True).values
    none = best == low
    place = torch.where(none, torch.zeros_like(best), 0xFFFFFFFF - (best & 0xFFFFFFFF))
    minus = torch.full_like(place, -1)
    parent = torch.where(none, minus, place // V)
    was_done = done.gather(1, parent.clamp_min(0))
    token = torch.where(none | was_done, minus, place % V)
    score = torch.where(none, torch.full_like(s["score"], -math.inf), cand.gather(1, place))
    beam = torch.arange(K, device=cand.device)[None]
    src = (torch.arange(B, device=cand.device)[:, None] * K + torch.where(none, beam, parent)).view(-1)
    p = s["p"][src]
    live = (torch.arange(S, device=cand.device)[:, None] <= p[None])[..., None]
    h, c = s["h"][:, src], s["c"][:, src]
    rows = torch.arange(B * K, device=cand.device)
    return {"score_new": score, "parent": parent.to(torch.int32), "token": token.to(torch.int32), "p_new": p,
            "h_new": torch.where(live, h, s["h_new"]), "c_new": torch.where(live, c, s["c_new"]),
            "top_h": h[p.long(), rows], "top_c": c[p.long(), rows]}


_PLAIN = {"norm": _plain_norm, "linear": _plain_linear, "distill": _plain_distill, "lse": _plain_lse, "beam": _plain_beam}


def run(state):
    return _run_own(state) if own else _PLAIN[state["case"]["kind"]](state, state["case"])


# ------------------------------------------------------------------------------- work
def work(case):
    e, kind = (2 if case["dtype"] == "bf16" else 4), case["kind"]
    if kind == "norm":
        R, N = case["R"], case["N"]
        b, f = 2 * R * N * e + 8 * N + 8 * R, 8 * R * N
        if case["call"] == "train":
            b, f = b + 8 * R * N + 8 * N, f + 14 * R * N
        return {"bytes": b, "flops": f}
    if kind == "linear":
        R, K, N = case["R"], case["K"], case["N"]
        if case["call"] == "forward":
            return {"bytes": e * (R * K + N * K + R * N * (1 + case["res"] + case["pre"])) + 4 * N, "flops": 2 * R * K * N}
        back = 4 * R * N + e * (R * K + N * K + (R * N if case["act"] != "none" else 0))
        return {"bytes": back + 4 * (R * K * (1 + case["res"]) + N * K + N), "flops": 4 * R * K * N}
    if kind == "distill":
        R, V, k = case["R"], case["V"], case["k"]
        return {"bytes": R * V * (e + 4) + 8 * R * k + 8 * R, "flops": 10 * R * V}
    n = case["B"] * case["K"]
    if kind == "lse":
        return {"bytes": n * case["V"] * e + 4 * n, "flops": 4 * n * case["V"]}
    live = n * (case["S"] + 1) / 2
    return {"bytes": n * case["V"] * e + 2 * live * case["H"] * (e + 4) + n * (case["H"] * (e + 4) + 29), "flops": 3 * n * case["V"]}


# -------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    s, kind = _inputs(case, seed), case["kind"]
    f = lambda k: s[k].double()
    if kind == "norm":
        x, g, N = f("x"), f("gamma"), case["N"]
        mean = x.sum(1) / N
        var = (x * x).sum(1) / N - mean * mean
        rstd = (var + s["eps"]) ** -0.5
        xh = (x - mean.unsqueeze(1)) * rstd.unsqueeze(1)
        out = {"y": xh * g + f("beta"), "mean": mean, "rstd": rstd}
        if case["call"] == "train":
            dy = f("dy")
            # dL/dx = rstd (I - 1 1^T / N - xh xh^T / N) (dy g), row by row
            a = dy * g
            out["dx"] = rstd.unsqueeze(1) * (a - (a.sum(1, True) + xh * torch.einsum("rn,rn->r", a, xh).unsqueeze(1)) / N)
            out["dgamma"], out["dbeta"] = torch.einsum("rn,rn->n", dy, xh), torch.einsum("rn->n", dy)
        return out
    if kind == "linear":
        x, W, act = f("x"), f("W"), case["act"]
        if case["call"] == "forward":
            z = torch.einsum("rk,nk->rn", x, W) + f("bias")
            y = {"none": lambda: z, "relu": lambda: torch.where(z > 0, z, 0 * z), "tanh": lambda: z.tanh(),
                 "gelu": lambda: z * torch.special.ndtr(z), "silu": lambda: z / (1 + (-z).exp())}[act]()
            return {"y": y + f("residual") if s["residual"] is not None else y, "pre": z if case["pre"] else None}
        d = f("dy")
        if act != "none":
            z = f("pre")
            phi = lambda: torch.special.ndtr(z) + z * (-z * z / 2).exp() / math.sqrt(2 * math.pi)
            sig = lambda: 1 / (1 + (-z).exp())
            d = d * {"relu": lambda: torch.where(z > 0, 1.0, 0.0), "tanh": lambda: z.cosh() ** -2, "gelu": phi,
                     "silu": lambda: sig() + z * sig() * sig() * (-z).exp()}[act]()
        dx = torch.einsum("rn,nk->rk", d, W)
        return {"dx": dx + f("add") if s["add"] is not None else dx, "dW": torch.einsum("rn,rk->nk", d, x), "dbias": d.sum(0)}
    if kind == "distill":
        R, V, tau, alpha = case["R"], case["V"], case["tau"], case["alpha"]
        z, idx, gold = f("logits"), s["t_idx"].long(), s["gold"].long()
        w = torch.where(idx < 0, 0.0, torch.exp(f("t_logit") / tau))
        total = w.sum(1, True)
        q = torch.where(total > 0, w / total, 0.0)
        target = torch.zeros(R, V + 1, dtype=torch.float64, device=z.device)  # place V: what is not there
        target.scatter_add_(1, torch.where(idx < 0, V, idx), q)
        taught, known = (idx >= 0).any(1).double(), (gold >= 0).double()
        soft, hard = torch.log_softmax(z / tau, 1), torch.log_softmax(z, 1)
        entropy = torch.special.entr(q).sum(1)
        cross = -torch.where(target[:, :V] > 0, target[:, :V] * soft, 0.0).sum(1)
        loss = alpha * tau ** 2 * (cross - entropy)
        nll = -torch.gather(hard, 1, gold.clamp(min=0).unsqueeze(1)).squeeze(1)
        loss = loss + (1 - alpha) * torch.where(gold >= 0, nll, 0.0)
        d = (soft.exp() * taught.unsqueeze(1) - target[:, :V]) * (alpha * tau)
        del soft, target
        d += hard.exp() * ((1 - alpha) * known).unsqueeze(1)
        d[torch.arange(R, device=z.device), gold.clamp(min=0)] -= (1 - alpha) * known
        return {"loss": loss * s["scale"], "dlogits": d * s["scale"]}
    if kind == "lse":
        return {"lse": torch.logsumexp(f("logits"), 2)}
    # The search: a candidate's score is defined as rounded to 32 bits after each operation, so
    # that the order is the same for everybody; a stable descending sort keeps the lowest place first.
    B, K, V, S, H = (case[k] for k in "BKVSH")
    step = (s["logits"].double() - s["lse"].double().unsqueeze(2)).float()
    cand = (s["score"].double().unsqueeze(2) + step.double()).float().double()
    done = s["done"].bool()
    cand[done] = -math.inf
    cand[:, :, 0][done] = s["score"].double()[done]
    cand = torch.nan_to_num(cand, nan=-math.inf, neginf=-math.inf)
    value, place = torch.sort(cand.reshape(B, K * V), dim=1, descending=True, stable=True)
    value, place = value[:, :K], place[:, :K]
    dead = torch.isinf(value)
    own_beam = torch.arange(K, device=value.device).expand(B, K)
    parent = torch.where(dead, own_beam, torch.div(place, V, rounding_mode="floor"))
    token = torch.where(dead | torch.gather(done, 1, parent), -1, place.remainder(V))
    h, c = f("h").view(S, B, K, H), f("c").view(S, B, K, H)
    at = parent.view(1, B, K, 1).expand(S, B, K, H)
    p = torch.gather(s["p"].view(B, K), 1, parent).long()
    h, c = torch.gather(h, 2, at), torch.gather(c, 2, at)
    top = p.view(1, B, K, 1).expand(1, B, K, H)
    above = (torch.arange(S, device=p.device).view(S, 1, 1, 1) > p.view(1, B, K, 1)).expand(S, B, K, H)
    th, tc = torch.gather(h, 0, top)[0], torch.gather(c, 0, top)[0]
    return {"score_new": value, "parent": torch.where(dead, -1, parent).int(), "token": token.int(), "p_new": p.reshape(-1).int(),
            "h_new": h.masked_fill(above, 0).view(S, B * K, H), "c_new": c.masked_fill(above, 0).view(S, B * K, H),
            "top_h": th.reshape(B * K, H), "top_c": tc.reshape(B * K, H)}
