"""The operators around an EAT layer that this framework is measured on: the vocabulary head's
cross entropy (with its gradient), the RMS norm with the residual's addition (with its gradient and
an e4m3 output), and the router's balance loss with per-expert counts (and its gradient).

Widths come from `paper_2609_33614_gb300.workloads` (256, 2048, 4096, 1408; 8 to 64 experts, 2 to 8
selected); vocabularies are generic.  `run` computes plain torch operations in 32 bits where `own`
is false, and calls the framework's operators where it is true.  Every draw follows from the seed.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
EPS = 1e-6
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _head(name, op, dtype, tokens, vocab, d, ignored=0.0):
    return dict(name=name, op=op, dtype=dtype, tokens=tokens, vocab=vocab, d=d, ignored=ignored)


def _norm(name, op, dtype, tokens, d, residual, fp8=False):
    return dict(name=name, op=op, dtype=dtype, tokens=tokens, d=d, residual=residual, fp8=fp8)


def _balance(name, tokens, experts, k, masked=0.0):
    return dict(name=name, op="balance", tokens=tokens, experts=experts, k=k, masked=masked)


def listed():
    return [
        # perplexity of one sequence being generated: the vocabulary matrix streamed for one token
        _head("nll_bf16_decode_1", "nll", "bf16", 1, 50257, 2048),
        # a full decode batch on an e4m3 vocabulary matrix
        _head("nll_fp8_decode_64", "nll", "fp8", 64, 100003, 4096),
        # scoring one ragged prompt
        _head("nll_bf16_prompt_777", "nll", "bf16", 777, 32003, 2048, 0.1),
        # scoring a batch of prompts in 8 bits
        _head("nll_fp8_prompt_4096", "nll", "fp8", 4096, 65536, 4096),
        # a step of a small model on a ragged batch, most of whose prompt tokens carry no loss
        _head("train_ragged_333", "train", "bf16", 333, 5003, 256, 0.4),
        # a training step's head at full size
        _head("train_8192", "train", "bf16", 8192, 65536, 2048, 0.05),
        # before a layer, for one token: the call is all latency
        _norm("norm_bf16_decode_1", "norm", "bf16", 1, 4096, True),
        # before an 8-bit product, for a prompt batch
        _norm("norm_fp8_prefill_16384", "norm", "bf16", 16384, 2048, True, True),
        # training: forward and gradient, the residual's gradient joined in
        _norm("norm_bf16_train_4095", "norm_train", "bf16", 4095, 4096, True),
        # the fp32 layer's width, a small step, first norm of a stack (no residual yet)
        _norm("norm_f32_train_64", "norm_train", "f32", 64, 256, False),
        # router of a small layer, few tokens
        _balance("balance_64x8", 64, 8, 2),
        # router of a training batch, padding masked
        _balance("balance_16384x64", 16384, 64, 8, 0.1),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


HEAD_WORK = 8192 * 65536 * 2048
HEAD_LOGITS = 8192 * 65536
HEAD_WIDTHS = (256, 576, 1024, 1408, 2048, 4096)


def draw(rng):
    op = rng.choice(("nll", "nll", "nll", "train", "train", "norm", "norm", "norm_train",
                     "norm_train", "balance", "balance"))
    if op in ("nll", "train"):
        dtype = rng.choice(("bf16", "fp8")) if op == "nll" else "bf16"
        d = rng.choice(HEAD_WIDTHS)
        tokens = _log_int(rng, 1, 8192)
        vocab = _log_int(rng, 500, 131072)
        vocab = min(vocab, HEAD_WORK // (tokens * d), HEAD_LOGITS // tokens)
        case = _head("", op, dtype, tokens, vocab, d,
                     rng.choice((0.0, 0.0, 0.1, 0.5)) if tokens >= 16 else 0.0)
    elif op in ("norm", "norm_train"):
        d = _log_int(rng, 64, 8192)
        if rng.random() < 0.6:
            d = rng.choice((256, 1024, 1408, 2048, 4096, 8192))
        tokens = min(_log_int(rng, 1, 16384), 16384 * 4096 // d)
        case = _norm("", op, rng.choice(("bf16", "bf16", "f32")), tokens, d,
                     rng.random() < 0.75, op == "norm" and rng.random() < 0.4)
    else:
        experts = rng.choice((8, 60, 64, 128, 256, _log_int(rng, 2, 256)))
        tokens = _log_int(rng, 1, 65536)
        case = _balance("", tokens, experts, min(experts // 2, rng.choice((1, 2, 4, 6, 8))),
                        rng.choice((0.0, 0.1, 0.5)) if tokens >= 16 else 0.0)
    del case["name"]
    return case


# ------------------------------------------------------------------------------------- inputs
def _gen(seed, k):
    return torch.Generator(DEV).manual_seed(1_000_003 * (seed + 1) + 7919 * k)


def _randn(seed, k, *shape):
    return torch.randn(*shape, generator=_gen(seed, k), device=DEV, dtype=torch.float32)


def _rand(seed, k, *shape):
    return torch.rand(*shape, generator=_gen(seed, k), device=DEV, dtype=torch.float32)


def _rows_e4m3(w):
    """e4m3 rows with one fp32 scale each (row maximum / 448)."""
    amax = w.abs().amax(dim=1)
    scale = torch.where(amax > 0, amax / 448.0, torch.ones_like(amax))
    return (w / scale[:, None]).to(torch.float8_e4m3fn), scale


def _head_inputs(case, seed):
    """Vocabulary rows N(0, 0.02^2); hidden states N(0, 1) that lean towards their target's row, so
    that target probabilities reach from about 1 / V to nearly 1; `ignored` of the targets are -1."""
    T, V, d = case["tokens"], case["vocab"], case["d"]
    w = _randn(seed, 1, V, d).mul_(0.02)
    u = _rand(seed, 2, T)
    y = (float(V) ** u - 1.0).clamp_(0, V - 1).to(torch.int64)  # frequent words first
    lean = 12.0 * _rand(seed, 3, T, 1)
    wy = w[y]
    x = _randn(seed, 4, T, d) + lean * wy / wy.square().sum(1, keepdim=True)
    drop = _rand(seed, 5, T) < case["ignored"]
    target = torch.where(drop, -1, y).to(torch.int32)
    if case["dtype"] == "fp8":
        (xq, xs), (wq, ws) = _rows_e4m3(x), _rows_e4m3(w)
        return dict(x=xq, x_scale=xs, w=wq, w_scale=ws, target=target)
    # the mean over the tokens that carry a loss
    g = (~drop).float() / max(1, int((~drop).sum()))
    return dict(x=x.to(torch.bfloat16), w=w.to(torch.bfloat16), target=target, g=g)


def _norm_inputs(case, seed):
    T, d, dt = case["tokens"], case["d"], TYPES[case["dtype"]]
    # a residual stream grows over the layers and has a few large channels
    big = 1.0 + 20.0 * (_rand(seed, 1, d) < 0.01)
    return dict(x=_randn(seed, 2, T, d).to(dt),
                residual=(3.0 * _randn(seed, 3, T, d) * big).to(dt) if case["residual"] else None,
                gamma=1.0 + 0.2 * _randn(seed, 4, d),
                dy=_randn(seed, 5, T, d).mul_(1e-3).to(dt),
                dres=_randn(seed, 6, T, d).mul_(1e-3).to(dt))


def _balance_inputs(case, seed):
    T, E, k = case["tokens"], case["experts"], case["k"]
    logits = _randn(seed, 1, T, E) + 0.7 * _randn(seed, 2, E)
    top = logits.topk(k, dim=1).indices.sort(1).values.to(torch.int32)
    # a variable number of experts per token: -1 after the last
    n = (1 + _rand(seed, 3, T, 1) * k).to(torch.int32).clamp_(max=k)
    idx = torch.where(torch.arange(k, device=DEV) < n, top, -1).to(torch.int32)
    mask = None
    if case["masked"]:
        mask = _rand(seed, 4, T) >= case["masked"]
    return dict(logits=logits, idx=idx.contiguous(), mask=mask,
                g=torch.full((1,), 0.01, device=DEV))


def _inputs(case, seed):
    make = {"nll": _head_inputs, "train": _head_inputs, "norm": _norm_inputs,
            "norm_train": _norm_inputs, "balance": _balance_inputs}
    return make[case["op"]](case, seed)


class State:
    pass


def prepare(case, seed):
    st = State()
    st.case = case
    st.__dict__.update(_inputs(case, seed))
    if own and case["op"] in ("nll", "train"):
        # a program keeps one handle for its vocabulary matrix
        from paper_2609_33614_gb300 import eat
        st.head = eat.EatHead(st.w, case["tokens"], w_scale=getattr(st, "w_scale", None),
                              grad=case["op"] == "train")
    return st


# ------------------------------------------------------------------- plain form, in 32 bits
def _plain_head(st):
    x, w = st.x.float(), st.w.float()
    if st.case["dtype"] == "fp8":
        x, w = x * st.x_scale[:, None], w * st.w_scale[:, None]
    logits = x @ w.T
    counted = st.target >= 0
    y = st.target.clamp(min=0).to(torch.int64)[:, None]
    ly = logits.gather(1, y)[:, 0]
    # -log p_y = log(1 + sum over the others of exp(l - l_y)), exact for a confident token too
    others = logits.scatter(1, y, -torch.inf)
    top = others.amax(1)
    r = top + others.sub_(top[:, None]).exp_().sum(1).log() - ly
    nll = r.clamp(min=0) + torch.log1p(torch.exp(-r.abs()))
    lse = ly + nll
    out = {"nll": torch.where(counted, nll, 0.0), "lse": torch.where(counted, lse, 0.0)}
    if st.case["op"] == "train":
        p = logits.sub_(lse[:, None]).exp_()
        p.scatter_add_(1, y, torch.full_like(y, -1, dtype=torch.float32))
        p.mul_(torch.where(counted, st.g, 0.0)[:, None])
        out["dx"] = (p @ w).to(st.x.dtype)
        out["dw"] = (p.T @ x).to(st.w.dtype)
    return out


def _plain_norm(st):
    s = st.x.float()
    if st.residual is not None:
        s = s + st.residual.float()
    y = s * (1.0 / torch.sqrt(s.square().mean(1, keepdim=True) + EPS)) * st.gamma
    h = s.to(st.x.dtype)
    if st.case["fp8"]:
        amax = y.abs().amax(1)
        scale = torch.where(amax > 0, amax / 448.0, 1.0)
        return {"h": h, "q": (y / scale[:, None]).to(torch.float8_e4m3fn), "scale": scale}
    out = {"h": h, "y": y.to(st.x.dtype)}
    if st.case["op"] == "norm_train":
        s, dy = h.float(), st.dy.float()
        rstd = 1.0 / torch.sqrt(s.square().mean(1, keepdim=True) + EPS)
        n, gd = s * rstd, dy * st.gamma
        dx = rstd * (gd - n * (gd * n).mean(1, keepdim=True))
        if st.residual is not None:
            dx = dx + st.dres.float()
        out["dx"] = dx.to(st.x.dtype)
        out["dgamma"] = (dy * n).sum(0)
    return out


def _plain_balance(st):
    T, E = st.logits.shape
    counted = torch.ones(T, dtype=torch.bool, device=DEV) if st.mask is None else st.mask
    n = counted.sum()
    live = (st.idx >= 0) & counted[:, None]
    counts = torch.zeros(E + 1, dtype=torch.int32, device=DEV)
    counts.index_add_(0, torch.where(live, st.idx, E).flatten(),
                      torch.ones(st.idx.numel(), dtype=torch.int32, device=DEV))
    counts = counts[:E]
    e = (st.logits - st.logits.amax(1, keepdim=True)).exp()
    p = torch.where(counted[:, None], e / e.sum(1, keepdim=True), 0.0)
    f = counts / counts.sum().clamp(min=1)
    n1 = n.clamp(min=1)
    loss = E * (f * (p.sum(0) / n1)).sum()
    dlogits = st.g * (E / n1) * p * (f - (p * f).sum(1, keepdim=True))
    return {"loss": loss.reshape(1), "counts": counts, "dlogits": dlogits}


# -------------------------------------------------------------------- the framework's calls
def _own_head(st):
    if st.case["op"] == "train":
        nll, lse, dx, dw = st.head.nll_grad(st.x, st.target, st.g)
        return {"nll": nll, "lse": lse, "dx": dx, "dw": dw}
    nll, lse = st.head.nll(st.x, st.target, x_scale=getattr(st, "x_scale", None))
    return {"nll": nll, "lse": lse}


def _own_norm(st):
    from paper_2609_33614_gb300 import eat
    if st.case["fp8"]:
        q, scale, h = eat.rms_norm_fp8(st.x, st.gamma, EPS, residual=st.residual)
        return {"h": h, "q": q, "scale": scale}
    y, h = eat.rms_norm(st.x, st.gamma, EPS, residual=st.residual)
    out = {"h": h, "y": y}
    if st.case["op"] == "norm_train":
        out["dx"], out["dgamma"] = eat.rms_norm_grad(
            h, st.gamma, EPS, st.dy, dres=st.dres if st.residual is not None else None)
    return out


def _own_balance(st):
    from paper_2609_33614_gb300 import eat
    loss, counts, n = eat.balance_loss(st.logits, st.idx, mask=st.mask)
    dlogits = eat.balance_grad(st.logits, counts, n, st.g, mask=st.mask)
    return {"loss": loss, "counts": counts, "dlogits": dlogits}


def run(state):
    op = state.case["op"]
    if op in ("nll", "train"):
        return _own_head(state) if own else _plain_head(state)
    if op in ("norm", "norm_train"):
        return _own_norm(state) if own else _plain_norm(state)
    return _own_balance(state) if own else _plain_balance(state)


# ------------------------------------------------------------- 64-bit values (plain torch)
def _exact_head(case, i):
    x, w = i["x"].double(), i["w"].double()
    if case["dtype"] == "fp8":
        x *= i["x_scale"].double()[:, None]
        w *= i["w_scale"].double()[:, None]
    train = case["op"] == "train"
    nll, lse, dx = [], [], []
    dw = torch.zeros_like(w) if train else None
    step = max(1, (1 << 28) // case["vocab"])  # 2 GiB of logits at a time
    for a in range(0, case["tokens"], step):
        xa, ya = x[a:a + step], i["target"][a:a + step].to(torch.int64)
        logits = torch.mm(xa, w.t())
        z = torch.logsumexp(logits, dim=1)
        keep = (ya >= 0).double()
        ly = logits[torch.arange(len(ya), device=DEV), ya.clamp(min=0)]
        nll.append((z - ly) * keep)
        lse.append(z * keep)
        if train:
            p = torch.softmax(logits, dim=1)
            p[torch.arange(len(ya), device=DEV), ya.clamp(min=0)] -= 1.0
            p *= (i["g"][a:a + step].double() * keep)[:, None]
            dx.append(torch.mm(p, w))
            dw.addmm_(p.t(), xa)
            del p
        del logits
    out = {"nll": torch.cat(nll), "lse": torch.cat(lse)}
    if train:
        out["dx"], out["dw"] = torch.cat(dx), dw
    return out


def _exact_norm(case, i):
    s = i["x"].double()
    if i["residual"] is not None:
        s = s + i["residual"].double()
    gamma = i["gamma"].double()
    y = gamma * s / (s.pow(2).mean(-1, keepdim=True) + EPS).sqrt()
    if case["fp8"]:
        top = y.abs().max(dim=-1).values
        scale = top / 448.0
        scale[top == 0] = 1.0
        return {"h": s, "q": y / scale[:, None], "scale": scale}
    out = {"h": s, "y": y}
    if case["op"] == "norm_train":
        # of the sum as it is stored
        s = s.to(TYPES[case["dtype"]]).double().requires_grad_()
        gamma = gamma.clone().requires_grad_()
        f = gamma * s / (s.pow(2).mean(-1, keepdim=True) + EPS).sqrt()
        f.backward(i["dy"].double())
        out["dx"] = s.grad + (i["dres"].double() if i["residual"] is not None else 0.0)
        out["dgamma"] = gamma.grad
    return out


def _exact_balance(case, i):
    z = i["logits"].double().requires_grad_()
    T, E = z.shape
    rows = torch.arange(T, device=DEV) if i["mask"] is None else i["mask"].nonzero()[:, 0]
    chosen = i["idx"][rows].flatten()
    counts = torch.bincount(chosen[chosen >= 0].to(torch.int64), minlength=E)
    if len(rows) == 0 or int(counts.sum()) == 0:
        return {"loss": torch.zeros(1, dtype=torch.float64, device=DEV),
                "counts": counts.to(torch.int32), "dlogits": torch.zeros_like(z)}
    share = counts.double() / counts.sum()
    loss = E * (torch.softmax(z[rows], dim=1).mean(0) * share).sum()
    (i["g"].double()[0] * loss).backward()
    return {"loss": loss.detach().reshape(1), "counts": counts.to(torch.int32),
            "dlogits": z.grad}


def exact(case, seed):
    i = _inputs(case, seed)
    if case["op"] in ("nll", "train"):
        return _exact_head(case, i)
    if case["op"] in ("norm", "norm_train"):
        return _exact_norm(case, i)
    return _exact_balance(case, i)


# ------------------------------------------------------------------------------------- work
def work(case):
    T = case["tokens"]
    if case["op"] in ("nll", "train"):
        V, d = case["vocab"], case["d"]
        eb, sb = (1, 4) if case["dtype"] == "fp8" else (2, 0)
        nbytes = (V + T) * (d * eb + sb) + T * 12
        if case["op"] == "nll":
            return {"bytes": nbytes, "flops": 2 * T * V * d}
        # the logits, dx and dw: three products; dx and dw written
        return {"bytes": nbytes + (V + T) * d * eb + T * 4, "flops": 6 * T * V * d}
    if case["op"] in ("norm", "norm_train"):
        d, eb = case["d"], {"f32": 4, "bf16": 2}[case["dtype"]]
        res = case["residual"]  # read it, write the sum
        nbytes = T * d * eb * (3 if res else 1) + d * 4
        nbytes += T * d + T * 4 if case["fp8"] else T * d * eb
        flops = 6 * T * d
        if case["op"] == "norm_train":  # dy (and the residual's gradient) in, dx out; h is at hand
            nbytes += T * d * eb * (3 if res else 2) + d * 4
            flops += 12 * T * d
        return {"bytes": nbytes, "flops": flops}
    E, k = case["experts"], case["k"]
    return {"bytes": 2 * T * E * 4 + T * k * 4 + T + E * 4, "flops": 12 * T * E}
