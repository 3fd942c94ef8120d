"""Timed cases of packed attention, the RMS norm and the balance loss: what surrounds a MoE layer's gate
and experts in a training step and in serving.

Kinds of case:
  prompt   causal attention of packed prompts with grouped heads (xs_attention_packed)
  serve    the same for a few new tokens of each request over a cache of keys and values
  train    the same with its gradients (xs_attention_packed, xs_attention_packed_backward)
  norm     residual addition and RMS norm with an E4M3 result (xs_rmsnorm), or its gradients
           (xs_rmsnorm_backward)
  balance  a router's per-expert counts and balance loss (xs_balance_loss), or its gradient added to
           the gate's (xs_balance_loss_backward)

`own` selects the library's calls; otherwise run() computes the plain form with torch operations in
32 bits. Inputs are drawn on the GPU from the seed, the lengths of packed sequences from the case.
"""
from __future__ import annotations

import math
import random

import torch

own = False

BLOCK = 128
AMAX_FLOOR = 2.0 ** -60
F8 = torch.float8_e4m3fn
EPS = 1e-6
ALPHA = 1e-2


def listed():
    return [
        # one request's next token, a short cache: the smallest call
        dict(name="serve_one", kind="serve", n_seq=1, new=1, cap=512, heads=8, kv_heads=1, dim=128, layout="token"),
        # a decode step of 32 requests, caches of up to 16384 tokens
        dict(name="serve_batch", kind="serve", n_seq=32, new=1, cap=16384, heads=32, kv_heads=8, dim=128, layout="token"),
        # a few drafted or chunked tokens a request, an odd number
        dict(name="serve_chunk", kind="serve", n_seq=7, new=61, cap=8192, heads=32, kv_heads=8, dim=128, layout="head"),
        # a prefill of ragged prompts
        dict(name="prompt_ragged", kind="prompt", n_seq=12, total=16381, heads=32, kv_heads=8, dim=128, layout="token"),
        # one long prompt, the local heads of a sequence-parallel rank
        dict(name="prompt_long", kind="prompt", n_seq=1, total=16384, heads=8, kv_heads=8, dim=128, layout="head"),
        # a training step's packed documents
        dict(name="train_packed", kind="train", n_seq=4, total=8192, heads=32, kv_heads=8, dim=128, layout="token"),
        # a training step of small heads, short ragged documents
        dict(name="train_short", kind="train", n_seq=19, total=4093, heads=16, kv_heads=4, dim=64, layout="token"),
        # a decode step's activations in front of an E4M3 product
        dict(name="norm_decode", kind="norm", direction="forward", rows=24, cols=7168, residual=True, bf16=False, fp8=True, weight="bf16"),
        # a training step's, with the bf16 values that a weight's gradient takes; an odd batch
        dict(name="norm_train", kind="norm", direction="forward", rows=16381, cols=7168, residual=True, bf16=True, fp8=True, weight="bf16"),
        dict(name="norm_grad", kind="norm", direction="backward", rows=16381, cols=7168, residual=True, bf16=True, fp8=False, weight="bf16"),
        # a training step's router: eight packed sequences, the logits of a gate in fp32
        dict(name="balance_train", kind="balance", direction="forward", T=32768, n_seq=8, E=256, k=8, score="sigmoid", dtype="f32"),
        # its gradient, logits as a bf16 GEMM leaves them, an odd batch
        dict(name="balance_grad", kind="balance", direction="backward", T=32765, n_seq=1, E=256, k=8, score="softmax", dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["serve", "serve", "prompt", "prompt", "train", "train", "norm", "norm", "balance"])
    if kind == "norm":
        bf16 = rng.random() < 0.5
        return dict(kind="norm", direction=rng.choice(["forward", "backward"]), rows=_log(rng, 1, 16384), cols=8 * _log(rng, 16, 896),
                    residual=rng.random() < 0.7, bf16=bf16, fp8=not bf16 or rng.random() < 0.5, weight=rng.choice(["bf16", "f32"]))
    if kind == "balance":
        E = rng.choice([8, 60, 64, 128, 160, 256, 384, 512])
        T = _log(rng, 1, 32768)
        return dict(kind="balance", direction=rng.choice(["forward", "backward"]), T=T, n_seq=rng.choice([1, 1, 3, 8, 24]), E=E,
                    k=rng.randint(1, min(10, E)), score=rng.choice(["sigmoid", "softmax"]), dtype=rng.choice(["f32", "bf16"]))
    kv = rng.choice([1, 2, 4, 8])
    case = dict(kind=kind, heads=kv * rng.choice([1, 2, 4]), kv_heads=kv, dim=rng.choice([64, 128, 128]),
                layout=rng.choice(["token", "head"]))
    if kind == "serve":
        return dict(case, n_seq=_log(rng, 1, 24), new=rng.choice([1, 1, 1, 2, 5, _log(rng, 1, 60)]), cap=_log(rng, 64, 8192))
    if kind == "prompt":
        return dict(case, n_seq=_log(rng, 1, 16), total=_log(rng, 17, 12000))
    return dict(case, n_seq=_log(rng, 1, 16), total=_log(rng, 17, 7000))


# ----------------------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(g, shape, std=1.0, spread=0.0, dtype=torch.bfloat16):
    """N(0, std^2), rows scaled by exp(U(-spread, spread)), drawn in slices of the first dimension."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    step = max(1, (1 << 26) // max(1, out[0].numel()))
    for i in range(0, shape[0], step):
        n = min(step, shape[0] - i)
        part = torch.randn((n,) + tuple(shape[1:]), generator=g, device="cuda").mul_(std)
        if spread:
            part *= torch.empty((n,) + (1,) * (len(shape) - 1), device="cuda").uniform_(-spread, spread, generator=g).exp_()
        out[i:i + n] = part
    return out


def _lengths(n, total):
    """n ragged lengths that sum to total: exponential shares, about a tenth of them empty."""
    rng = random.Random(1000003 * n + total)
    share = [0.0 if n > 1 and rng.random() < 0.1 else rng.expovariate(1.0) for _ in range(n)]
    share[0] = max(share[0], 0.1)
    ends, at = [], 0.0
    for x in share:
        at += x
        ends.append(round(at / sum(share) * total))
    ends[-1] = total
    return [b - a for a, b in zip([0] + ends[:-1], ends)]


def _spans(case):
    """(first query, queries, first key, keys) of every sequence."""
    if case["kind"] == "serve":
        rng = random.Random(1000003 * case["n_seq"] + case["cap"])
        low = min(case["new"], case["cap"])
        return [(s * case["new"], case["new"], s * (case["cap"] + case["new"]), case["new"] + _log(rng, low, case["cap"]))
                for s in range(case["n_seq"])]
    at, out = 0, []
    for n in _lengths(case["n_seq"], case["total"]):
        out.append((at, n, at, n))
        at += n
    return out


def _rows(case):
    """Rows of q and of k."""
    if case["kind"] == "serve":
        return case["n_seq"] * case["new"], case["n_seq"] * (case["cap"] + case["new"])
    return case["total"], case["total"]


def _heads(x, layout):
    """x [rows][heads][dim], laid out so in memory ("token") or as [heads][rows][dim] ("head")."""
    return x if layout == "token" else x.transpose(0, 1).contiguous().transpose(0, 1)


def _attention_inputs(case, seed):
    g = _gen(seed)
    Tq, Tk = _rows(case)
    names = [("q", Tq, case["heads"]), ("k", Tk, case["kv_heads"]), ("v", Tk, case["kv_heads"])]
    if case["kind"] == "train":
        names.append(("d_o", Tq, case["heads"]))
    return {n: _heads(_normal(g, (rows, h, case["dim"])), case["layout"]) for n, rows, h in names}


def _norm_inputs(case, seed):
    g = _gen(seed)
    shape = (case["rows"], case["cols"])
    s = dict(w=_normal(g, (1, case["cols"]), 0.1, dtype=torch.float32)[0].add_(1.0))
    if case["weight"] == "bf16":
        s["w"] = s["w"].bfloat16()
    s["x"] = _normal(g, shape, spread=0.5)
    if case["direction"] == "backward":
        s["dy"] = _normal(g, shape, 1e-3, spread=0.5)
    if case["residual"]:
        s["r"] = _normal(g, shape, 1e-3 if case["direction"] == "backward" else 1.0, spread=0.5)
    return s


def _balance_inputs(case, seed):
    g = _gen(seed)
    T, E = case["T"], case["E"]
    logits = torch.randn((T, E), generator=g, device="cuda") + 0.5 * torch.randn((E,), generator=g, device="cuda")
    if case["dtype"] == "bf16":
        logits = logits.bfloat16()
    idx = torch.sort(logits.float(), dim=-1, descending=True, stable=True)[1][:, :case["k"]]
    lens = _lengths(case["n_seq"], T)
    seq = torch.repeat_interleave(torch.arange(case["n_seq"]), torch.tensor(lens)).cuda()
    d_loss = torch.randn((case["n_seq"],), generator=g, device="cuda")
    d_gate = ALPHA / E * case["n_seq"] / T * torch.randn((T, E), generator=g, device="cuda")     # about the loss's own gradient
    return logits, idx, lens, seq, d_loss, d_gate.to(logits.dtype)


def _starts(lens):
    return torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device="cuda")


def prepare(case, seed):
    kind = case["kind"]
    f32 = dict(dtype=torch.float32, device="cuda")
    status = torch.zeros((1,), dtype=torch.int32, device="cuda")
    if kind in ("prompt", "serve", "train"):
        s = _attention_inputs(case, seed)
        spans = _spans(case)
        s["spans"] = spans
        s["q_start"] = torch.tensor([x[0] for x in spans] + [_rows(case)[0]], dtype=torch.int32, device="cuda")
        s["k_start"] = torch.tensor([x[2] for x in spans] + [_rows(case)[1]], dtype=torch.int32, device="cuda")
        s["k_rows"] = torch.tensor([x[3] for x in spans], dtype=torch.int32, device="cuda") if kind == "serve" else None
        zeros = lambda x: _heads(torch.zeros(x.shape, dtype=x.dtype, device="cuda"), case["layout"])
        s["out"] = dict(o=zeros(s["q"]), lse=torch.zeros((case["heads"], _rows(case)[0]), **f32))
        if kind == "train":
            s["out"] |= dict(dq=zeros(s["q"]), dk=zeros(s["k"]), dv=zeros(s["v"]))
    elif kind == "norm":
        s = _norm_inputs(case, seed)
        rows, cols = case["rows"], case["cols"]
        bf = dict(dtype=torch.bfloat16, device="cuda")
        if case["direction"] == "backward":
            s["out"] = dict(dx=torch.zeros((rows, cols), **bf), dw=torch.zeros((cols,), **f32))
        else:
            s["out"] = {}
            if case["residual"]:
                s["out"]["h"] = torch.zeros((rows, cols), **bf)
            if case["bf16"]:
                s["out"]["y"] = torch.zeros((rows, cols), **bf)
            if case["fp8"]:
                blocks = -(-cols // BLOCK)
                s["scales"] = torch.zeros((rows, -(-blocks // 4) * 4), **f32)
                s["out"] |= dict(codes=torch.zeros((rows, blocks * BLOCK), dtype=F8, device="cuda"), scales=s["scales"][:, :blocks])
    else:
        logits, idx, lens, seq, d_loss, d_gate = _balance_inputs(case, seed)
        s = dict(logits=logits, idx=idx.int(), lens=lens, rows=torch.tensor(lens, dtype=torch.float32, device="cuda"), seq=seq,
                 q_start=_starts(lens))
        if case["direction"] == "backward":
            s |= dict(d_loss=d_loss, d_gate=d_gate, counts=_counts(case, lens, idx).int(), out=dict(d_logits=torch.zeros_like(logits)))
        else:
            s["out"] = dict(counts=torch.zeros((case["n_seq"], case["E"]), dtype=torch.int32, device="cuda"),
                            mean=torch.zeros((case["n_seq"], case["E"]), **f32), loss=torch.zeros((case["n_seq"],), **f32))
    return dict(s, case=case, status=status)


# ----------------------------------------------------------------------------- plain forms
def _plain_attention(s):
    c, out = s["case"], s["out"]
    H, K, D = c["heads"], c["kv_heads"], c["dim"]
    G = H // K
    rows = lambda x, at, n: x[at:at + n].float().reshape(n, K, -1, D).permute(1, 2, 0, 3).reshape(K, -1, D)
    back = lambda x, n: x.reshape(K, -1, n, D).permute(2, 0, 1, 3).reshape(n, -1, D)
    for q0, n, k0, m in s["spans"]:
        if not n:
            continue
        q, k, v = rows(s["q"], q0, n), rows(s["k"], k0, m), rows(s["v"], k0, m)
        hidden = torch.arange(m, device=q.device) > torch.arange(n, device=q.device)[:, None] + (m - n)
        x = (q @ k.transpose(1, 2)).view(K, G, n, m).mul_(D ** -0.5).masked_fill_(hidden, -math.inf).view(K, G * n, m)
        top = x.amax(-1, keepdim=True)
        p = x.sub_(top).exp_()
        total = p.sum(-1, keepdim=True)
        p /= total
        o = p @ v
        out["o"][q0:q0 + n] = back(o, n)
        out["lse"][:, q0:q0 + n] = (top + total.log()).view(H, n)
        if c["kind"] == "train":
            d_o = rows(s["d_o"], q0, n)
            ds = (d_o @ v.transpose(1, 2)).sub_((d_o * o).sum(-1, keepdim=True)).mul_(p).mul_(D ** -0.5)
            out["dq"][q0:q0 + n] = back(ds @ k, n)
            out["dk"][k0:k0 + m] = back(ds.transpose(1, 2) @ q, m)
            out["dv"][k0:k0 + m] = back(p.transpose(1, 2) @ d_o, m)
    return out


def _quantize_rows(x):
    """1 x 128 blocks of fp32 x: E4M3 values (zero columns up to whole blocks) and fp32 scales."""
    more = -x.shape[1] % BLOCK
    v = (torch.nn.functional.pad(x, (0, more)) if more else x).view(x.shape[0], -1, BLOCK)
    s = v.abs().amax(-1).clamp_min(AMAX_FLOOR) / 448.0
    return (v / s[..., None]).to(F8).view(x.shape[0], -1), s


def _plain_norm(s):
    c, out, w = s["case"], s["out"], s["w"].float()
    if c["direction"] == "forward":
        h = s["x"].float()
        if c["residual"]:
            out["h"].copy_(h + s["r"].float())
            h = out["h"].float()
        y = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS) * w
        if c["bf16"]:
            out["y"].copy_(y)
        if c["fp8"]:
            codes, scales = _quantize_rows(y)
            out["codes"].copy_(codes)
            out["scales"].copy_(scales)
        return out
    h, dy = s["x"].float(), s["dy"].float()
    inv = torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS)
    unit = h * inv
    g = dy * w
    dx = inv * (g - unit * (g * unit).mean(-1, keepdim=True))
    out["dx"].copy_(dx + s["r"].float() if c["residual"] else dx)
    torch.sum(dy * unit, 0, out=out["dw"])
    return out


def _sums(x, lens):
    """Sums over each sequence's rows."""
    return torch.stack([part.sum(0) for part in x.split(lens)])


def _counts(case, lens, idx):
    return _sums(torch.zeros((case["T"], case["E"]), device=idx.device).scatter_(1, idx, 1.0), lens)


def _shares(case, logits):
    """Scores that sum to one over a token's experts, and the scores."""
    if case["score"] == "softmax":
        p = torch.softmax(logits, -1)
        return p, p
    p = torch.sigmoid(logits)
    return p / p.sum(-1, keepdim=True), p


def _plain_balance(s):
    c, out, n = s["case"], s["out"], s["rows"][:, None]
    p, score = _shares(c, s["logits"].float())
    if c["direction"] == "forward":
        counts = _counts(c, s["lens"], s["idx"].long())
        out["counts"].copy_(counts)
        out["mean"].copy_(_sums(p, s["lens"]) / n.clamp_min(1))
        torch.mul((counts / (c["k"] * n.clamp_min(1)) * out["mean"]).sum(-1), ALPHA * c["E"], out=out["loss"])
        return out
    f = s["counts"] * (ALPHA * c["E"] / c["k"]) * s["d_loss"][:, None] / n.clamp_min(1) ** 2
    f = f[s["seq"]]
    grad = p * (f - (f * p).sum(-1, keepdim=True))
    if c["score"] == "sigmoid":
        grad *= 1 - score
    out["d_logits"].copy_(s["d_gate"].float() + grad)
    return out


# ----------------------------------------------------------------------------- the library's calls
def _own_call(s):
    """A call without arguments but the stream: descriptors and workspaces that a program keeps."""
    from paper_2607_23264_amd import xstage as X
    c, kind, out, ptr = s["case"], s["case"]["kind"], s["out"], X.ptr
    if kind in ("prompt", "serve", "train"):
        a = X.attn_packed(s["q"], s["k"], s["v"], out["o"], s["q_start"], s["k_start"], k_rows=s["k_rows"], lse=out["lse"],
                          max_k=c["cap"] + c["new"] if kind == "serve" else 0)
        ws = X.workspace(X.xs_attention_packed_workspace_bytes, a)
        forward = lambda st: X.xs_attention_packed(a, ptr(ws), ws.numel(), ptr(s["status"]), st)
        if kind != "train":
            return X, forward
        g = X.attn_packed_grads(s["d_o"], out["dq"], out["dk"], out["dv"])
        bs = X.workspace(X.xs_attention_packed_backward_workspace_bytes, a)
        return X, lambda st: forward(st) or X.xs_attention_packed_backward(a, g, ptr(bs), bs.numel(), ptr(s["status"]), st)
    if kind == "norm":
        rows, cols = c["rows"], c["cols"]
        wt = X.XS_TYPE_BF16 if c["weight"] == "bf16" else X.XS_TYPE_F32
        if c["direction"] == "backward":
            ws = X.workspace(X.xs_rmsnorm_backward_workspace_bytes, rows, cols)
            return X, lambda st: X.xs_rmsnorm_backward(ptr(s["dy"]), cols, ptr(s.get("r")), cols, ptr(s["x"]), cols, ptr(s["w"]), wt,
                                                       EPS, rows, cols, ptr(out["dx"]), cols, ptr(out["dw"]), ptr(ws), ws.numel(), st)
        pair = (ptr(out["codes"]), out["codes"].shape[1], ptr(s["scales"]), s["scales"].shape[1]) if c["fp8"] else (None, 0, None, 0)
        return X, lambda st: X.xs_rmsnorm(ptr(s["x"]), cols, ptr(s.get("r")), cols, ptr(s["w"]), wt, EPS, rows, cols,
                                          ptr(out.get("h")), cols, ptr(out.get("y")), cols, *pair, st)
    T, E = c["T"], c["E"]
    gate = X.gate(E, c["k"], score=X.XS_SCORE_SIGMOID if c["score"] == "sigmoid" else X.XS_SCORE_SOFTMAX,
                  logits_type=X.XS_TYPE_BF16 if c["dtype"] == "bf16" else X.XS_TYPE_F32)
    if c["direction"] == "backward":
        return X, lambda st: X.xs_balance_loss_backward(gate, ptr(s["logits"]), E, T, ptr(s["q_start"]), c["n_seq"], ALPHA, ptr(s["counts"]),
                                                        ptr(s["d_loss"]), ptr(s["d_gate"]), E, ptr(out["d_logits"]), E, ptr(s["status"]), st)
    ws = X.workspace(X.xs_balance_loss_workspace_bytes, T, E, c["n_seq"])
    return X, lambda st: X.xs_balance_loss(gate, ptr(s["logits"]), E, T, ptr(s["idx"]), ptr(s["q_start"]), c["n_seq"], ALPHA,
                                           ptr(out["counts"]), ptr(out["mean"]), ptr(out["loss"]), ptr(ws), ws.numel(), ptr(s["status"]), st)


def run(s):
    kind = s["case"]["kind"]
    if own:
        if "call" not in s:
            s["call"] = _own_call(s)
        X, call = s["call"]
        X.check(call(torch.cuda.current_stream().cuda_stream), kind)
        return s["out"]
    return {"norm": _plain_norm, "balance": _plain_balance}.get(kind, _plain_attention)(s)


# ----------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    kind = case["kind"]
    if kind == "norm":
        n, w = case["rows"] * case["cols"], case["cols"] * (2 if case["weight"] == "bf16" else 4)
        if case["direction"] == "backward":
            return {"bytes": n * (8 if case["residual"] else 6) + w + 4 * case["cols"], "flops": 0}
        return {"bytes": n * (2 + (4 if case["residual"] else 0) + (2 if case["bf16"] else 0) + (1 + 4 / BLOCK if case["fp8"] else 0)) + w,
                "flops": 0}
    if kind == "balance":
        T, E, k, b = case["T"], case["E"], case["k"], 2 if case["dtype"] == "bf16" else 4
        if case["direction"] == "backward":
            return {"bytes": 3 * T * E * b + 4 * case["n_seq"] * E, "flops": 0}
        return {"bytes": T * (E * b + 4 * k) + 8 * case["n_seq"] * E, "flops": 0}
    H, K, D = case["heads"], case["kv_heads"], case["dim"]
    spans = _spans(case)
    pairs = sum(n * (m - n) + n * (n + 1) // 2 for _, n, _, m in spans)
    q, k = sum(x[1] for x in spans) * H, sum(x[3] for x in spans) * K
    if kind == "train":     # o, d_o and the gradients too; five products more
        return {"bytes": 2 * D * (4 * q + 4 * k) + 4 * q, "flops": 14.0 * D * H * pairs}
    return {"bytes": 2 * D * (2 * q + 2 * k) + 4 * q, "flops": 4.0 * D * H * pairs}


# ----------------------------------------------------------------------------- 64-bit results
def _exact_attention(case, seed):
    t = _attention_inputs(case, seed)
    train, D, G = case["kind"] == "train", case["dim"], case["heads"] // case["kv_heads"]
    f64 = dict(dtype=torch.float64, device="cuda")
    out = dict(o=torch.zeros(t["q"].shape, **f64), lse=torch.zeros((case["heads"], t["q"].shape[0]), **f64))
    if train:
        out |= {d: torch.zeros(t[n].shape, **f64) for d, n in (("dq", "q"), ("dk", "k"), ("dv", "v"))}
    for q0, n, k0, m in _spans(case):
        if not n:
            continue
        for h in range(case["heads"]):
            q, k, v = (x.double().requires_grad_(train) for x in (t["q"][q0:q0 + n, h], t["k"][k0:k0 + m, h // G], t["v"][k0:k0 + m, h // G]))
            score = torch.mm(q, k.T) / math.sqrt(D)
            score = score + torch.full((n, m), -math.inf, **f64).triu(m - n + 1)
            lse = torch.logsumexp(score, -1)
            o = torch.mm(torch.exp(score - lse[:, None]), v)
            out["o"][q0:q0 + n, h], out["lse"][h, q0:q0 + n] = o.detach(), lse.detach()
            if train:
                dq, dk, dv = torch.autograd.grad(o, (q, k, v), t["d_o"][q0:q0 + n, h].double())
                out["dq"][q0:q0 + n, h] = dq
                out["dk"][k0:k0 + m, h // G] += dk
                out["dv"][k0:k0 + m, h // G] += dv
    return out


def _nearest(v):
    """v (fp64, at most 448) rounded to E4M3 values, ties to even."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(v / step) * step


def _exact_norm(case, seed):
    t = _norm_inputs(case, seed)
    x, w = t["x"].double(), t["w"].double()
    if case["direction"] == "backward":
        x, w = x.requires_grad_(True), w.requires_grad_(True)
        y = x / torch.sqrt(torch.mean(x ** 2, -1, keepdim=True) + EPS) * w
        dx, dw = torch.autograd.grad(y, (x, w), t["dy"].double())
        return dict(dx=dx + t["r"].double() if case["residual"] else dx, dw=dw)
    out = {}
    if case["residual"]:
        x = x + t["r"].double()
        out["h"] = x
        x = x.bfloat16().double()
    y = x / torch.sqrt(torch.mean(x ** 2, -1, keepdim=True) + EPS) * w
    if case["bf16"]:
        out["y"] = y
    if case["fp8"]:
        rows, cols = y.shape
        blocks = -(-cols // BLOCK)
        full = torch.zeros((rows, blocks * BLOCK), dtype=torch.float64, device="cuda")
        full[:, :cols] = y
        full = full.view(rows, blocks, BLOCK)
        scales = full.abs().max(-1)[0].clamp_min(AMAX_FLOOR) / 448
        out |= dict(codes=_nearest(full / scales[..., None]).view(rows, -1), scales=scales)
    return out


def _exact_balance(case, seed):
    logits, idx, lens, seq, d_loss, d_gate = _balance_inputs(case, seed)
    n, E = torch.tensor(lens, dtype=torch.float64, device="cuda").clamp_min(1)[:, None], case["E"]
    x = logits.double().requires_grad_(True)
    if case["score"] == "softmax":
        p = torch.exp(x - torch.logsumexp(x, -1, keepdim=True))
    else:
        p = 1 / (1 + torch.exp(-x))
        p = p / p.sum(-1, keepdim=True)
    member = (seq[:, None] == torch.arange(case["n_seq"], device="cuda")).double()
    mean = torch.mm(member.T, p) / n
    share = torch.mm(member.T, torch.zeros_like(p).scatter(1, idx, 1.0)) / (case["k"] * n)
    loss = ALPHA * E * (share * mean).sum(-1)
    if case["direction"] == "forward":
        return dict(counts=None, mean=mean.detach(), loss=loss.detach())
    (grad,) = torch.autograd.grad((loss * d_loss.double()).sum(), x)
    return dict(d_logits=grad + d_gate.double())


def exact(case, seed):
    return {"norm": _exact_norm, "balance": _exact_balance}.get(case["kind"], _exact_attention)(case, seed)
