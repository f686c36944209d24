"""What training and serving the experts of a router's choice takes, and this framework is measured on:
tokens sorted by expert and back (with weights, and the gradients of both), matrix products in e4m3
with a scale for each block of 128 (one matrix, or one per expert; a training step of such a layer with
its quantisations), and the gated activation between two of them (with its gradient).

Widths come from `paper_2609_33614_gb300.workloads` (256, 2048, 4096, 1024, 1408, 14336; 8 to 64
experts, 2 to 8 selected).  `run` computes plain torch operations in 32 bits where `own` is false, and
calls the framework's operators where it is true.  Every draw follows from the seed.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
E4M3 = torch.float8_e4m3fn
BLOCK = 128
FEW = 32  # up to so many tokens every one selects all of its k experts


def _sort(name, dtype, tokens, d, experts, k, masked=0.0, fp8=False, train=False):
    return dict(name=name, op="sort", dtype=dtype, tokens=tokens, d=d, experts=experts, k=k,
                masked=masked, fp8=fp8, train=train)


def _mm(name, tokens, experts, k, n, d):
    """experts == 0: one matrix for all tokens."""
    return dict(name=name, op="mm", tokens=tokens, experts=experts, k=k, n=n, d=d)


def _linear(name, tokens, experts, k, n, d):
    return dict(_mm(name, tokens, experts, k, n, d), op="linear")


def _glu(name, rows, f, fp8=False, train=False):
    return dict(name=name, op="glu", rows=rows, f=f, fp8=fp8, train=train)


def listed():
    return [
        # one token being generated: the call is all latency
        _sort("sort_decode_1", "bf16", 1, 2048, 64, 8),
        # a prompt batch whose expert products are in 8 bits
        _sort("sort_fp8_prefill_4096", "bf16", 4096, 2048, 60, 4, fp8=True),
        # the fp32 layer's width, a small ragged step with padding
        _sort("sort_f32_train_333", "f32", 333, 256, 8, 2, masked=0.3, train=True),
        # a training step at full size, padding masked
        _sort("sort_train_8191", "bf16", 8191, 2048, 64, 8, masked=0.1, train=True),
        # gate and up projections of one token: the weights of two experts are read
        _mm("mm_experts_decode_1", 1, 8, 2, 28672, 4096),
        # a decode batch over many narrow experts
        _mm("mm_experts_decode_32", 32, 64, 8, 2048, 2048),
        # one matrix for a ragged prompt
        _mm("mm_dense_777", 777, 0, 1, 4096, 1408),
        # gate and up projections of a prompt batch
        _mm("mm_experts_prefill_4096", 4096, 60, 4, 2816, 2048),
        # forward and both gradients of a small layer, weights quantised after the optimizer's step
        _linear("linear_train_ragged_333", 333, 8, 2, 512, 256),
        # the same of a training step at full size
        _linear("linear_train_4096", 4096, 64, 8, 2048, 2048),
        # between the two products of a decode batch, in 8 bits for the second
        _glu("glu_fp8_decode_8", 8, 14336, fp8=True),
        # training: forward and gradient
        _glu("glu_train_16383", 16383, 1408, train=True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


ROUTERS = ((8, 2), (60, 4), (64, 6), (64, 8), (16, 4))
MM_WORK = 32768 * 2048 * 2048
MM_WEIGHTS = 64 * 2048 * 2048


def draw(rng):
    op = rng.choice(("sort", "sort", "sort", "mm", "mm", "mm", "linear", "linear", "glu", "glu"))
    if op == "sort":
        experts, k = rng.choice(ROUTERS + ((_log_int(rng, 4, 256), rng.choice((1, 2, 3, 4))),))
        d = rng.choice((256, 1024, 1408, 2048, 4096, _log_int(rng, 64, 4096)))
        tokens = min(_log_int(rng, 1, 16384), 8191 * 2048 * 8 // (d * k))
        train = rng.random() < 0.5
        dtype = rng.choice(("bf16", "bf16", "f32"))
        case = _sort("", dtype, tokens, d, experts, k,
                     rng.choice((0.0, 0.1, 0.5)) if tokens >= 16 else 0.0,
                     not train and rng.random() < 0.5, train)
    elif op in ("mm", "linear"):
        experts, k = rng.choice(ROUTERS + ((0, 1), (0, 1), (_log_int(rng, 2, 32), 1)))
        d = rng.choice((256, 1024, 1408, 2048, 4096, 16 * _log_int(rng, 8, 300)))
        n = rng.choice((512, 2048, 2816, 4096, 16 * _log_int(rng, 8, 300)))
        if op == "mm" and rng.random() < 0.3:
            n = _log_int(rng, 64, 8192)
        n = min(n, MM_WEIGHTS // (max(1, experts) * d) // 16 * 16)
        tokens = min(_log_int(rng, 1, 8192), MM_WORK // (n * d * k))
        case = (_mm if op == "mm" else _linear)("", tokens, experts, k, n, d)
    else:
        f = rng.choice((256, 1024, 1408, 14336, _log_int(rng, 64, 14336)))
        rows = min(_log_int(rng, 1, 32768), 16383 * 1408 // f)
        train = rng.random() < 0.5
        case = _glu("", rows, f, not train and rng.random() < 0.6, train)
    del case["name"]
    return case


# ------------------------------------------------------------------------------------- inputs
def _gen(seed, k):
    return torch.Generator(DEV).manual_seed(1_000_003 * (seed + 1) + 7919 * k)


def _randn(seed, k, *shape):
    return torch.randn(*shape, generator=_gen(seed, k), device=DEV, dtype=torch.float32)


def _rand(seed, k, *shape):
    return torch.rand(*shape, generator=_gen(seed, k), device=DEV, dtype=torch.float32)


def _routing(seed, T, E, k):
    """Selected experts [T, k] int32 (ascending, -1 after the last: a variable number per token) and
    their weights, which sum to 1."""
    logits = _randn(seed, 1, T, E) + 0.7 * _randn(seed, 2, E)
    top = logits.topk(k, dim=1)
    idx, order = top.indices.sort(1)
    n = (1 + _rand(seed, 3, T, 1) * k).to(torch.int32).clamp_(max=k)
    if T <= FEW:
        n.fill_(k)
    live = torch.arange(k, device=DEV) < n
    w = torch.where(live, top.values.gather(1, order).exp(), 0.0)
    return torch.where(live, idx, -1).to(torch.int32).contiguous(), w / w.sum(1, keepdim=True)


def _big_channels(seed, k, d):
    """Hidden states have a few large channels."""
    return 1.0 + 20.0 * (_rand(seed, k, d) < 0.01)


def _sort_inputs(case, seed):
    T, d, E, k, dt = case["tokens"], case["d"], case["experts"], case["k"], TYPES[case["dtype"]]
    idx, w = _routing(seed, T, E, k)
    mask = _rand(seed, 4, T) >= case["masked"] if case["masked"] else None
    return dict(idx=idx, w=w, mask=mask, x=(_randn(seed, 5, T, d) * _big_channels(seed, 6, d)).to(dt),
                out=_randn(seed, 7, T * k, d).to(dt),  # what the experts made of the sorted rows
                dy=_randn(seed, 8, T, d).mul_(1e-3).to(dt),
                din=_randn(seed, 9, T * k, d).mul_(1e-3).to(dt))  # gradient of the sorted rows


def _matmul_inputs(case, seed):
    """Rows sorted by expert (zeros behind the last), and weights N(0, 0.02^2) whose rows differ in size."""
    T, E, k, n, d = (case[c] for c in ("tokens", "experts", "k", "n", "d"))
    M = T * k
    if E:
        idx, _ = _routing(seed, T, E, k)
        counts = torch.bincount(idx[idx >= 0].long(), minlength=E)
        offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).to(torch.int32)
    else:
        offsets = torch.tensor([0, M], device=DEV, dtype=torch.int32)
    live = torch.arange(M, device=DEV)[:, None] < offsets[-1]
    x = torch.where(live, _randn(seed, 5, M, d) * _big_channels(seed, 6, d), 0.0)
    w = _randn(seed, 7, max(1, E), n, d).mul_(0.02).mul_(0.5 + _rand(seed, 8, max(1, E), n, 1))
    i = dict(offsets=offsets, most=int((offsets[1:] - offsets[:-1]).max()))
    if case["op"] == "linear":
        g = torch.where(live, _randn(seed, 9, M, n).mul_(1e-3), 0.0)
        i.update(x=x.to(torch.bfloat16), w=w.to(torch.bfloat16), dy=g.to(torch.bfloat16))
    else:
        i["xq"], i["xs"] = _plain_quant_rows(x.to(torch.bfloat16))
        i["wq"], i["ws"] = _plain_quant_tiles(w)
    if not E:
        i.update({n: i[n][0] for n in ("w", "wq", "ws") if n in i})
    return i


def _glu_inputs(case, seed):
    R, f = case["rows"], case["f"]
    return dict(gu=_randn(seed, 1, R, 2 * f).mul_(1.5).to(torch.bfloat16),
                dh=_randn(seed, 2, R, f).mul_(1e-3).to(torch.bfloat16))


def _inputs(case, seed):
    make = {"sort": _sort_inputs, "mm": _matmul_inputs, "linear": _matmul_inputs, "glu": _glu_inputs}
    return make[case["op"]](case, seed)


class State:
    pass


def prepare(case, seed):
    st = State()
    st.case = case
    st.__dict__.update(_inputs(case, seed))
    return st


# ------------------------------------------------------------------- plain form, in 32 bits
def _scales(top):
    return torch.where(top > 1e-35, top / 448.0, 1.0)


def _plain_quant_rows(x):
    """[M, K] -> e4m3 [M, K] and a scale for each 128 elements of a row, [ceil(K / 128), M]."""
    M, K = x.shape
    kb = -(-K // BLOCK)
    v = torch.nn.functional.pad(x.float(), (0, kb * BLOCK - K)).view(M, kb, BLOCK)
    scale = _scales(v.abs().amax(2))
    q = (v / scale[:, :, None]).view(M, kb * BLOCK)[:, :K].to(E4M3)
    return q.contiguous(), scale.t().contiguous()


def _plain_quant_tiles(w):
    """[E, N, K] -> e4m3 [E, N, K] and a scale for each 128 x 128 tile."""
    E, N, K = w.shape
    nb, kb = -(-N // BLOCK), -(-K // BLOCK)
    v = torch.nn.functional.pad(w.float(), (0, kb * BLOCK - K, 0, nb * BLOCK - N))
    v = v.view(E, nb, BLOCK, kb, BLOCK)
    scale = _scales(v.abs().amax((2, 4)))
    q = (v / scale[:, :, None, :, None]).view(E, nb * BLOCK, kb * BLOCK)[:, :N, :K].to(E4M3)
    return q.contiguous(), scale


def _of_rows(q, scale):
    return q.float() * scale.t().repeat_interleave(BLOCK, 1)[:, :q.shape[1]]


def _of_tiles(q, scale):
    s = scale.repeat_interleave(BLOCK, -2).repeat_interleave(BLOCK, -1)
    return q.float() * s[..., :q.shape[-2], :q.shape[-1]]


def _spread(x, offsets, most):
    """Rows sorted by expert -> [E, most, ...], zeros behind an expert's last, and where they were."""
    at = offsets[:-1, None].long() + torch.arange(most, device=DEV)
    live = at < offsets[1:, None]
    at = torch.where(live, at, 0)
    return torch.where(live[..., None], x[at], 0.0), at, live


def _plain_product(x, w, offsets, most):
    """x [M, K], w [E, N, K] or [N, K] in 32 bits -> [M, N] in bf16."""
    if w.dim() == 2:
        return (x @ w.T).to(torch.bfloat16)
    M, E = x.shape[0], w.shape[0]
    if M < E:  # few rows: their own experts' matrices alone
        r = torch.arange(M, device=DEV)
        e = torch.searchsorted(offsets[1:].contiguous(), r, right=True, out_int32=True)
        y = (w[e.clamp(max=E - 1).long()] @ x[:, :, None])[..., 0]
        return torch.where((e < E)[:, None], y, 0.0).to(torch.bfloat16)
    v, at, live = _spread(x, offsets, most)
    y = torch.zeros(M + 1, w.shape[1], device=DEV)
    y[torch.where(live, at, M)] = v @ w.transpose(1, 2)
    return y[:M].to(torch.bfloat16)


def _plain_sort(st):
    T, k = st.idx.shape
    E, M = st.case["experts"], T * k
    e = st.idx.long()
    live = (e >= 0) & (e < E)
    if st.mask is not None:
        live &= st.mask[:, None]
    key = torch.where(live, e, E).flatten()
    order = key.argsort(stable=True)
    ends = (key[None, :] == torch.arange(E, device=DEV)[:, None]).sum(1).cumsum(0)
    offsets = torch.cat([ends.new_zeros(1), ends]).to(torch.int32)
    rank = torch.empty_like(order)
    rank[order] = torch.arange(M, device=DEV)
    slot = torch.where(live, rank.view(T, k), -1).to(torch.int32)
    filled = (torch.arange(M, device=DEV) < offsets[-1])[:, None]
    rows = torch.where(filled, st.x[order // k], 0.0).to(st.x.dtype)
    out = {"offsets": offsets, "slot": slot}
    if st.case["fp8"]:
        out["q"], out["scale"] = _plain_quant_rows(rows)
    else:
        out["rows"] = rows
    at = torch.where(live, slot, 0).long()
    mine = torch.where(live[..., None], st.out[at].float(), 0.0)
    out["y"] = (mine * st.w[..., None]).sum(1).to(st.x.dtype)
    if st.case["train"]:
        dy = st.dy.float()
        out["dw"] = torch.where(live, (mine * dy[:, None]).sum(2), 0.0)
        wr = st.w.flatten()[order][:, None]
        out["dout"] = torch.where(filled, dy[order // k] * wr, 0.0).to(st.x.dtype)
        din = torch.where(live[..., None], st.din[at].float(), 0.0)
        out["dx"] = din.sum(1).to(st.x.dtype)
    return out


def _plain_linear(st):
    x, dy, offsets, most = st.x, st.dy, st.offsets, st.most
    dense = st.w.dim() == 2
    wq, ws = _plain_quant_tiles(st.w[None] if dense else st.w)
    w = _of_tiles(wq, ws)
    w = w[0] if dense else w
    y = _plain_product(_of_rows(*_plain_quant_rows(x)), w, offsets, most)
    dx = _plain_product(_of_rows(*_plain_quant_rows(dy)), w.transpose(-1, -2).contiguous(), offsets,
                        most)
    # the weights' gradient sums over rows: blocks of 128 rows of an expert, padded with zeros
    most = -(-most // BLOCK) * BLOCK
    a, b = (_of_columns(_spread(v.float(), offsets, most)[0]) for v in (dy, x))
    dw = (a.transpose(1, 2) @ b).to(torch.bfloat16)
    return {"y": y, "dx": dx, "dw": dw[0] if dense else dw}


def _of_columns(v):
    """[E, 128 m, C], quantised in blocks of 128 rows of a column, as the values it then stands for."""
    E, R, C = v.shape
    v = v.view(E, R // BLOCK, BLOCK, C)
    scale = _scales(v.abs().amax(2, keepdim=True))
    return ((v / scale).to(E4M3).float() * scale).view(E, R, C)


def _plain_glu(st):
    f = st.case["f"]
    gate, up = st.gu[:, :f].float(), st.gu[:, f:].float()
    s = 1.0 / (1.0 + torch.exp(-gate))
    h = gate * s * up
    if st.case["fp8"]:
        q, scale = _plain_quant_rows(h)
        return {"q": q, "scale": scale}
    out = {"h": h.to(torch.bfloat16)}
    if st.case["train"]:
        dh = st.dh.float()
        dgate = dh * up * s * (1.0 + gate * (1.0 - s))
        out["dgu"] = torch.cat([dgate, dh * gate * s], 1).to(torch.bfloat16)
    return out


# -------------------------------------------------------------------- the framework's calls
def _own_sort(st):
    from paper_2609_33614_gb300 import eat
    offsets, slot = eat.expert_sort(st.idx, st.case["experts"], mask=st.mask)
    out = {"offsets": offsets, "slot": slot}
    if st.case["fp8"]:
        out["q"], out["scale"] = eat.expert_gather_fp8(st.x, slot, offsets)
    else:
        out["rows"] = eat.expert_gather(st.x, slot, offsets)
    out["y"] = eat.expert_combine(st.out, slot, st.w)
    if st.case["train"]:
        out["dout"], out["dw"] = eat.expert_combine_grad(st.dy, st.out, slot, offsets, st.w)
        out["dx"] = eat.expert_combine(st.din, slot)
    return out


def _own_mm(st):
    from paper_2609_33614_gb300 import eat
    offsets = st.offsets if st.case["experts"] else None
    return {"y": eat.block_mm(st.xq, st.xs, st.wq, st.ws, offsets=offsets)}


def _own_linear(st):
    from paper_2609_33614_gb300 import eat
    offsets = st.offsets if st.case["experts"] else None
    wq, ws = eat.quant_tiles(st.w)
    xq, xs, xcq, xcs = eat.quant_rows_columns(st.x, offsets=offsets)
    y = eat.block_mm(xq, xs, wq, ws, offsets=offsets)
    gq, gs, gcq, gcs = eat.quant_rows_columns(st.dy, offsets=offsets)
    dx = eat.block_mm(gq, gs, wq, ws, offsets=offsets, transposed=True)
    dw = eat.block_mm_grad(gcq, gcs, xcq, xcs, offsets=offsets)
    return {"y": y, "dx": dx, "dw": dw}


def _own_glu(st):
    from paper_2609_33614_gb300 import eat
    if st.case["fp8"]:
        q, scale = eat.swiglu_fp8(st.gu)
        return {"q": q, "scale": scale}
    out = {"h": eat.swiglu(st.gu)}
    if st.case["train"]:
        out["dgu"] = eat.swiglu_grad(st.gu, st.dh)
    return out


def run(state):
    op = state.case["op"]
    if op == "sort":
        return _own_sort(state) if own else _plain_sort(state)
    if op == "mm":
        if own:
            return _own_mm(state)
        return {"y": _plain_product(_of_rows(state.xq, state.xs), _of_tiles(state.wq, state.ws),
                                    state.offsets, state.most)}
    if op == "linear":
        return _own_linear(state) if own else _plain_linear(state)
    return _own_glu(state) if own else _plain_glu(state)


# ------------------------------------------------------------- 64-bit values (plain torch)
def _exact_blocks(v):
    """64-bit values with blocks of 128 along the last axis -> v / scale, and the scales."""
    n = v.shape[-1]
    parts = v.split(BLOCK, dim=-1)
    top = torch.stack([p.abs().max(dim=-1).values for p in parts], dim=-1)
    scale = top / 448
    scale[top <= 1e-35] = 1.0
    return v / scale.repeat_interleave(BLOCK, dim=-1)[..., :n], scale


def _exact_sort(case, i):
    T, k, E = case["tokens"], case["k"], case["experts"]
    M, x = T * k, i["x"].double()
    flat = i["idx"].flatten().cpu()
    if i["mask"] is not None:
        flat = torch.where(i["mask"].cpu().repeat_interleave(k), flat, -1)
    lists = [(flat == e).nonzero()[:, 0] for e in range(E)]
    ends = torch.tensor([0] + [len(v) for v in lists]).cumsum(0)
    entry = torch.cat(lists)  # of each row
    n = len(entry)
    slot = torch.full((M,), -1, dtype=torch.int32)
    slot[entry] = torch.arange(n, dtype=torch.int32)
    entry = entry.to(DEV)
    rows = torch.zeros(M, x.shape[1], dtype=torch.float64, device=DEV)
    rows[:n] = x[entry // k]
    out = {"offsets": ends.to(torch.int32), "slot": slot.view(T, k)}
    if case["fp8"]:
        out["q"], scale = _exact_blocks(rows)
        out["scale"] = scale.t().contiguous()
    else:
        out["rows"] = rows
    made, w = i["out"].double()[:n], i["w"].double().flatten()[entry][:, None]
    out["y"] = torch.zeros_like(x).index_add_(0, entry // k, w * made)
    if case["train"]:
        g = i["dy"].double()[entry // k]
        dw = torch.zeros(M, dtype=torch.float64, device=DEV)
        dw[entry] = (g * made).sum(1)
        out["dw"] = dw.view(T, k)
        out["dout"] = torch.zeros_like(rows)
        out["dout"][:n] = w * g
        out["dx"] = torch.zeros_like(x).index_add_(0, entry // k, i["din"].double()[:n])
    return out


def _exact_wide(scale, n):
    return scale.double().repeat_interleave(BLOCK, dim=-1)[..., :n]


def _exact_mm(case, i):
    x = i["xq"].double() * _exact_wide(i["xs"].t(), case["d"])
    wq, ws = (i["wq"], i["ws"]) if case["experts"] else (i["wq"][None], i["ws"][None])
    y = torch.zeros(len(x), case["n"], dtype=torch.float64, device=DEV)
    ends = i["offsets"].tolist()
    for e in range(len(wq)):
        a, b = ends[e], ends[e + 1]
        if a == b:
            continue
        s = _exact_wide(_exact_wide(ws[e], case["d"]).t(), case["n"]).t()
        y[a:b] = torch.mm(x[a:b], (wq[e].double() * s).t())
    return {"y": y}


def _exact_rounded(v):
    """What blocks of 128 along the last axis stand for once they are held in e4m3."""
    q, scale = _exact_blocks(v)
    return q.to(E4M3).double() * scale.repeat_interleave(BLOCK, dim=-1)[..., :v.shape[-1]]


def _exact_linear(case, i):
    E = case["experts"]
    w_all = i["w"] if E else i["w"][None]
    x, g = i["x"].double(), i["dy"].double()
    xr, gr = _exact_rounded(x), _exact_rounded(g)
    y = torch.zeros(len(x), case["n"], dtype=torch.float64, device=DEV)
    dx = torch.zeros_like(x)
    dw = torch.zeros(w_all.shape, dtype=torch.float64, device=DEV)
    ends = i["offsets"].tolist()
    for e in range(len(w_all)):
        a, b = ends[e], ends[e + 1]
        if a == b:
            continue
        w = w_all[e].double()
        for r in range(0, case["n"], BLOCK):
            for c in range(0, case["d"], BLOCK):
                t = w[r:r + BLOCK, c:c + BLOCK]
                s = t.abs().max() / 448
                t.copy_((t / s).to(E4M3).double() * s)
        y[a:b] = torch.mm(xr[a:b], w.t())
        dx[a:b] = torch.mm(gr[a:b], w)
        dw[e] = torch.mm(_exact_rounded(g[a:b].t().contiguous()),
                         _exact_rounded(x[a:b].t().contiguous()).t())
    return {"y": y, "dx": dx, "dw": dw if E else dw[0]}


def _exact_glu(case, i):
    v = i["gu"].double().requires_grad_()
    gate, up = v.split(case["f"], dim=1)
    h = gate * torch.sigmoid(gate) * up
    if case["fp8"]:
        q, scale = _exact_blocks(h.detach())
        return {"q": q, "scale": scale.t().contiguous()}
    out = {"h": h.detach()}
    if case["train"]:
        h.backward(i["dh"].double())
        out["dgu"] = v.grad
    return out


def exact(case, seed):
    i = _inputs(case, seed)
    return {"sort": _exact_sort, "mm": _exact_mm, "linear": _exact_linear,
            "glu": _exact_glu}[case["op"]](case, i)


# ------------------------------------------------------------------------------------- work
def _rows(case):
    """Selections of a call, on average."""
    T, k = case["tokens"], case["k"]
    return T * k if T <= FEW or not case["experts"] else T * (k + 1) // 2


def work(case):
    if case["op"] == "glu":
        n = case["rows"] * case["f"]
        if case["fp8"]:
            return {"bytes": 5 * n + n // 32, "flops": 8 * n}
        return {"bytes": (6 + 10 * case["train"]) * n, "flops": (6 + 12 * case["train"]) * n}
    T, k, d = case["tokens"], case["k"], case["d"]
    M, R = T * k, _rows(case)
    if case["op"] == "sort":
        eb = {"f32": 4, "bf16": 2}[case["dtype"]]
        live = 1.0 - case["masked"]
        R = R * live
        # x read once; sorted rows written (zeros behind the last); the experts' rows and y
        nbytes = T * live * d * eb + R * d * eb + T * d * eb + M * 12 + case["experts"] * 4
        nbytes += M * d + M * d // 32 if case["fp8"] else M * d * eb
        flops = 2 * R * d
        if case["train"]:  # dy read, dout written; din read, dx written
            nbytes += T * live * d * eb + M * d * eb + R * d * eb + T * d * eb + 2 * M * 4
            flops += 4 * R * d
        return {"bytes": int(nbytes), "flops": int(flops)}
    n, E = case["n"], case["experts"]
    # experts that are selected at all: k of one token, on average of more
    met = 1 if not E else k if T == 1 else E * (1.0 - (1.0 - 1.0 / E) ** R)
    if case["op"] == "mm":
        nbytes = met * n * d + R * d + M * n * 2
        return {"bytes": int(nbytes * (1 + 1 / 4096)), "flops": 2 * R * n * d}
    # bf16 weights, rows and gradient in; y, dx and the weights' gradient out
    nbytes = 4 * max(1, E) * n * d + 2 * R * (n + d) + 2 * M * (n + d)
    return {"bytes": nbytes, "flops": 6 * R * n * d}
