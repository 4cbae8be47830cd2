"""Performance cases of the operators for training adapters over frozen weights held in 8 bits.

Five kinds of case:
  norm      RMSNorm of x + residual with an int8 output and a scale per row, as in front of an 8-bit projection
  norm_bwd  its gradient with respect to x (= residual) and the gain
  product   int8 codes of tokens times int8 codes of a weight, a scale per token and per channel
  layer     rows to int8 codes, then the product: a projection whose input no norm has quantised (attention output,
            MLP down projection), or the input gradient of a layer (the weight's channel scales enter as column factors)
  distill   loss over the vocabulary against a teacher's top logits and the labels, with its gradient

All inputs are synthetic and made on the GPU from the seed.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5
TINY = 1e-36            # rows whose largest magnitude is below this are held as zero


# ---- cases ---------------------------------------------------------------------------------
def _norm(name, M, d, dtype="bf16", residual=True, want_y=False):
    c = {"kind": "norm", "M": M, "d": d, "dtype": dtype, "residual": residual, "want_y": want_y}
    return dict(c, name=name) if name else c


def _norm_bwd(name, M, d, dtype="bf16", residual=True, want_dg=False):
    c = {"kind": "norm_bwd", "M": M, "d": d, "dtype": dtype, "residual": residual, "want_dg": want_dg}
    return dict(c, name=name) if name else c


def _product(name, M, K, N, dtype="bf16", bias=False, residual=False):
    c = {"kind": "product", "M": M, "K": K, "N": N, "dtype": dtype, "bias": bias, "residual": residual}
    return dict(c, name=name) if name else c


def _layer(name, M, K, N, dtype="bf16", bias=False, residual=False, backward=False):
    c = {"kind": "layer", "M": M, "K": K, "N": N, "dtype": dtype, "bias": bias, "residual": residual, "backward": backward}
    return dict(c, name=name) if name else c


def _distill(name, M, V, k, dtype="bf16", temperature=2.0, labels=True):
    c = {"kind": "distill", "M": M, "V": V, "k": k, "dtype": dtype, "temperature": temperature, "labels": labels}
    return dict(c, name=name) if name else c


def listed():
    return [
        # a single token of the narrowest model: the call itself
        _norm("norm_one_token", 1, 128, dtype="fp32"),
        # the norm in front of a Llama-2-7B-shaped block's projections, a batch of eight sequences of 1024; the bf16 output is
        # kept for the adapters
        _norm("norm_llama", 8192, 4096, want_y=True),
        # odd rows and width, fp32
        _norm_bwd("norm_bwd_odd", 1665, 1001, dtype="fp32"),
        # the same block's backward pass with a trained gain
        _norm_bwd("norm_bwd_llama", 8192, 4096, want_dg=True),
        # one token through a 4096-wide projection: the weight's bytes
        _product("product_one_token", 1, 4096, 4096),
        # the QKV projection of a GPT-2-small-shaped block at a row count that is a multiple of nothing
        _product("product_ragged", 1665, 768, 2304, bias=True),
        # a Llama-2-7B-shaped up projection over eight sequences of 1024
        _product("product_llama_up", 8192, 4096, 11008),
        # the attention output projection of a GPT-2-medium-shaped block: bias, residual
        _layer("layer_attn_out", 4096, 1024, 1024, bias=True, residual=True),
        # input gradient of a Llama-2-7B-shaped up projection
        _layer("layer_input_grad", 4096, 11008, 4096, backward=True),
        # a small fp32 vocabulary
        _distill("distill_tiny_fp32", 512, 1024, 8, dtype="fp32"),
        # a Llama-shaped vocabulary, rows and temperature of no convenient value, teacher only
        _distill("distill_llama", 1665, 32000, 20, temperature=1.5, labels=False),
        # the GPT-2 vocabulary, eight sequences of 512, the teacher's 64 largest logits and the labels
        _distill("distill_gpt2", 4096, 50257, 64),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "norm_bwd", "product", "layer", "distill"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    flag = lambda: rng.random() < 0.5  # noqa: E731
    cost = 2 if dtype == "fp32" else 1
    if kind in ("norm", "norm_bwd"):
        d = _log_int(rng, 8, 8192)
        if flag():
            d = max(8, d // 8 * 8)
        M = _log_int(rng, 1, max(1, min(32768, 8192 * 4096 // (cost * d))))
        return _norm(None, M, d, dtype, flag(), flag()) if kind == "norm" else _norm_bwd(None, M, d, dtype, flag(), flag())
    if kind in ("product", "layer"):
        K, N = _log_int(rng, 16, 11008), _log_int(rng, 16, 11008)
        if flag():
            K, N = max(16, K // 16 * 16), max(16, N // 8 * 8)
        most = (8192 if kind == "product" else 4096) * 4096 * 11008 // cost
        M = _log_int(rng, 1, max(1, min(16384, most // (K * max(N, K // 2, 1024)))))
        if kind == "product":
            return _product(None, M, K, N, dtype, flag(), flag())
        backward = flag()
        return _layer(None, M, K, N, dtype, not backward and flag(), flag(), backward)
    V = _log_int(rng, 64, 50257)
    M = _log_int(rng, 1, max(1, min(16384, 4096 * 50257 // (cost * V))))
    return _distill(None, M, V, _log_int(rng, 1, 64), dtype, rng.choice([1.0, 1.5, 2.0, 4.0, round(rng.uniform(0.5, 5.0), 2)]), flag())


# ---- inputs --------------------------------------------------------------------------------
_DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(1000003 * seed + 17)
    dt = _DTYPES[case["dtype"]]
    randn = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    rand = lambda *s: torch.rand(*s, device="cuda", generator=g)  # noqa: E731
    st = {"case": case}
    if case["kind"] in ("norm", "norm_bwd"):
        M, d = case["M"], case["d"]
        # a residual stream: a few channels far larger than the others, rows of different size, a row of padding
        channel = 1.0 + 15.0 * (rand(d) < 0.01)
        st["x"] = (randn(M, d) * channel * torch.exp(0.5 * randn(M, 1))).to(dt)
        st["g"] = (1.0 + 0.2 * randn(d)).to(dt)
        st["residual"] = (randn(M, d) * channel).to(dt) if case["residual"] else None
        if case["kind"] == "norm":
            if M > 4:
                st["x"][M // 3] = 0
                if case["residual"]:
                    st["residual"][M // 3] = 0
        else:
            st["dy"] = (1e-3 * randn(M, d)).to(dt)
            st["residual"] = (1e-3 * randn(M, d)).to(dt) if case["residual"] else None
        return st
    if case["kind"] in ("product", "layer"):
        M, K, N = case["M"], case["K"], case["N"]
        st["bias"] = (0.05 * randn(N)).to(dt) if case["bias"] else None
        st["residual"] = randn(M, N).to(dt) if case["residual"] else None
        # codes of weights drawn N(0, 0.02): magnitude 127 at about four standard deviations
        pad = (K + 15) // 16 * 16              # rows of codes start on 16-byte boundaries
        codes = lambda rows: (randn(rows, pad)[:, :K] * 32).round_().clamp_(-127, 127).to(torch.int8)  # noqa: E731
        hold = lambda c: torch.zeros(c.shape[0], pad, dtype=torch.int8, device="cuda")[:, :K].copy_(c)  # noqa: E731
        st["w"] = hold(codes(N))
        if case["kind"] == "product":
            st["x"] = hold(codes(M))
            st["x_scales"] = (0.02 + 0.03 * rand(M))
            st["w_scales"] = 6e-4 * (0.5 + rand(N))
        else:
            st["x"] = randn(M, K).to(dt)
            if M > 4:
                st["x"][M // 3] = 0
            # backward: x is dL/dy and the weight is the transposed one, whose channels are the columns
            st["col_scale"] = 6e-4 * (0.5 + rand(K)) if case["backward"] else None
            st["w_scales"] = None if case["backward"] else 6e-4 * (0.5 + rand(N))
        return st
    M, V, k = case["M"], case["V"], case["k"]
    st["logits"] = (2.5 * randn(M, V)).to(dt)
    # the teacher's largest logits: its own vocabulary entries, sorted by size; some rows hold fewer (index -1)
    st["top_idx"] = torch.argsort(rand(M, max(V // 16, k) if V < 4096 else 4096), dim=1)[:, :k].to(torch.int32).contiguous()
    st["top_idx"] = (st["top_idx"] * (max(1, V // 4096)) % V).to(torch.int32)
    st["top_logits"] = (6.0 + 2.0 * randn(M, k)).sort(dim=1, descending=True).values.contiguous()
    if k > 2:
        st["top_idx"][:: 7, k // 2:] = -1
    if M > 4:
        st["top_idx"][M // 3] = -1             # a row for which the teacher gave nothing
    if case["labels"]:
        y = torch.randint(0, V, (M,), device="cuda", generator=g, dtype=torch.int32)
        st["labels"] = torch.where(rand(M) < 0.1, torch.full_like(y, -100), y)      # padding
        st["labels"][0] = V // 2
    else:
        st["labels"] = None
    st["weights"] = (0.5, 0.5) if case["labels"] else (0.0, 1.0)
    return st


# ---- plain forms ---------------------------------------------------------------------------
def _plain_codes(v, top):
    """int8 codes of the rows of v (fp32) whose largest magnitudes are `top`."""
    live = (top >= TINY) & torch.isfinite(top)
    inv = torch.where(live, torch.full_like(top, 127.0).div(top), torch.zeros_like(top))
    return torch.where(live[:, None], torch.round(v * inv[:, None]), torch.zeros_like(v))


def _plain_scales(top, size):
    return torch.where(torch.isfinite(top), torch.where(top >= TINY, size, torch.zeros_like(size)), torch.full_like(size, float("nan")))


def _plain_norm(st):
    dt = st["x"].dtype
    s = st["x"].float()
    if st["residual"] is not None:
        s = s + st["residual"].float()
    rstd = torch.rsqrt((s * s).mean(dim=1) + EPS)
    v = s * st["g"].float()
    top = v.abs().amax(dim=1)
    codes, scales = _plain_codes(v, top), _plain_scales(top, top * rstd / 127.0)
    out = {"values": (codes * scales[:, None]).bfloat16(), "scales": scales}
    if st["residual"] is not None:
        out["h"] = s.to(dt)
    if st["case"]["want_y"]:
        out["y"] = (v * rstd[:, None]).to(dt)
    return out


def _plain_norm_bwd(st):
    dt = st["x"].dtype
    h, dy = st["x"].float(), st["dy"].float()
    rstd = torch.rsqrt((h * h).mean(dim=1, keepdim=True) + EPS)
    w = dy * st["g"].float()
    dx = rstd * (w - h * (rstd * rstd) * (w * h).mean(dim=1, keepdim=True))
    if st["residual"] is not None:
        dx = dx + st["residual"].float()
    out = {"dx": dx.to(dt)}
    if st["case"]["want_dg"]:
        out["dg"] = (dy * h * rstd).sum(dim=0)
    return out


def _plain_product(st, x, x_scales, dt):
    y = (x @ st["w"].float().t()) * x_scales[:, None]
    if st["w_scales"] is not None:
        y = y * st["w_scales"]
    if st["bias"] is not None:
        y = y + st["bias"].float()
    if st["residual"] is not None:
        y = y + st["residual"].float()
    return {"y": y.to(dt)}


def _plain_layer(st):
    v = st["x"].float()
    if st["col_scale"] is not None:
        v = v * st["col_scale"]
    top = v.abs().amax(dim=1)
    return _plain_product(st, _plain_codes(v, top), _plain_scales(top, top / 127.0), st["x"].dtype)


def _plain_distill(st):
    T, (wc, wk) = st["case"]["temperature"], st["weights"]
    z, idx, t, labels = st["logits"].float(), st["top_idx"].long(), st["top_logits"].float() / T, st["labels"]
    M, V = z.shape
    rows = torch.ones(M, dtype=torch.bool, device=z.device) if labels is None else (labels >= 0) & (labels < V)
    n = rows.sum().clamp(min=1)
    keep = (idx >= 0) & (idx < V)
    idx = torch.where(keep, idx, torch.zeros_like(idx))
    t = torch.where(keep, t, torch.full_like(t, float("-inf")))
    some = keep.any(dim=1)
    q = torch.where(keep & some[:, None], torch.softmax(torch.where(some[:, None], t, torch.zeros_like(t)), dim=1), torch.zeros_like(t))
    logq = torch.where(keep, torch.log_softmax(torch.where(some[:, None], t, torch.zeros_like(t)), dim=1), torch.zeros_like(t))
    logp = torch.log_softmax(z / T, dim=1)
    kl = (q * (logq - logp.gather(1, idx))).sum(dim=1)
    d = wk * T * (logp.exp_() * some[:, None])
    d.scatter_add_(1, idx, -wk * T * q)
    row = wk * T * T * kl
    if labels is not None:
        y = torch.where(rows, labels, torch.zeros_like(labels)).long()[:, None]
        logp = torch.log_softmax(z, dim=1)
        row = row - wc * logp.gather(1, y)[:, 0]
        d += wc * logp.exp_()
        d.scatter_add_(1, y, torch.full_like(y, -wc, dtype=torch.float32))
    row = torch.where(rows, row, torch.zeros_like(row))
    d *= (rows / n)[:, None]
    return {"loss": (row.double().sum() / n).float(), "rows": row, "dlogits": d.to(st["logits"].dtype)}


# ---- one pass ------------------------------------------------------------------------------
def _own_norm(st):
    from paper_2407_00952_b200 import binding as B
    codes, scales, h, y = B.rmsnorm_quantize(st["x"], st["g"], residual=st["residual"], eps=EPS, want_y=st["case"]["want_y"])
    out = {"values": B.dequantize_rows(codes, scales, torch.bfloat16), "scales": scales}
    if h is not None:
        out["h"] = h
    if y is not None:
        out["y"] = y
    return out


def _own_norm_bwd(st):
    from paper_2407_00952_b200 import binding as B
    dx, dg = B.rmsnorm_bwd(st["dy"], st["x"], st["g"], resid=st["residual"], eps=EPS, want_dg=st["case"]["want_dg"])
    return {"dx": dx} if dg is None else {"dx": dx, "dg": dg}


def _own_product(st):
    from paper_2407_00952_b200 import binding as B
    return {"y": B.linear_i8(st["x"], st["x_scales"], st["w"], st["w_scales"], bias=st["bias"], residual=st["residual"],
                             dtype=_DTYPES[st["case"]["dtype"]])}


def _own_layer(st):
    from paper_2407_00952_b200 import binding as B
    codes, scales = B.quantize_rows(st["x"], col_scale=st["col_scale"])
    return {"y": B.linear_i8(codes, scales, st["w"], st["w_scales"], bias=st["bias"], residual=st["residual"], dtype=st["x"].dtype)}


def _own_distill(st):
    from paper_2407_00952_b200 import binding as B
    wc, wk = st["weights"]
    loss, rows, dlogits = B.distill_loss(st["logits"], st["top_idx"], st["top_logits"], labels=st["labels"],
                                         temperature=st["case"]["temperature"], ce_weight=wc, kd_weight=wk)
    return {"loss": loss, "rows": rows, "dlogits": dlogits}


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"norm": _own_norm, "norm_bwd": _own_norm_bwd, "product": _own_product, "layer": _own_layer, "distill": _own_distill}[kind](state)
    if kind == "product":
        return _plain_product(state, state["x"].float(), state["x_scales"], _DTYPES[state["case"]["dtype"]])
    return {"norm": _plain_norm, "norm_bwd": _plain_norm_bwd, "layer": _plain_layer, "distill": _plain_distill}[kind](state)


# ---- what a pass cannot do without ---------------------------------------------------------
def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "norm":
        n, r = case["M"] * case["d"], int(case["residual"])
        return {"bytes": n * (es * (1 + 2 * r + int(case["want_y"])) + 1) + 4 * case["M"] + es * case["d"], "flops": 6 * n}
    if case["kind"] == "norm_bwd":
        n, r = case["M"] * case["d"], int(case["residual"])
        return {"bytes": n * es * (3 + r) + (es + 4 * int(case["want_dg"])) * case["d"], "flops": 10 * n}
    if case["kind"] in ("product", "layer"):
        M, K, N = case["M"], case["K"], case["N"]
        x_bytes = M * K * (1 if case["kind"] == "product" else es)
        return {"bytes": x_bytes + N * K + es * M * N * (1 + int(case["residual"])) + 4 * (M + N) + es * N * int(case["bias"]), "flops": 2 * M * N * K}
    M, V = case["M"], case["V"]
    return {"bytes": 2 * es * M * V + M * (8 * case["k"] + 8), "flops": 8 * M * V}


# ---- the definitions in 64 bits ------------------------------------------------------------
def _codes64(v32):
    """Codes (as fp64) and largest magnitudes of rows whose rounding decisions the definition makes in fp32."""
    a = torch.max(torch.abs(v32), dim=1)[0]
    c = torch.zeros_like(v32)
    full = (a >= TINY).nonzero()[:, 0]
    c[full] = torch.clamp(torch.round(v32[full] * torch.true_divide(torch.full_like(a[full], 127.0), a[full]).unsqueeze(1)), -127, 127)
    return c.double(), a


def exact(case, seed):
    st = prepare(case, seed)
    f = lambda k: st[k].double()  # noqa: E731
    if case["kind"] == "norm":
        s32 = st["x"].float() if st["residual"] is None else st["x"].float() + st["residual"].float()
        s = f("x") if st["residual"] is None else f("x") + f("residual")
        scale = 1.0 / torch.sqrt(torch.sum(s ** 2, 1) / case["d"] + EPS)
        codes, a = _codes64(s32 * st["g"].float())
        steps = torch.max(torch.abs(s * f("g")), dim=1)[0] * scale / 127
        steps[a < TINY] = 0
        out = {"values": codes * steps[:, None], "scales": steps}
        if case["residual"]:
            out["h"] = s
        if case["want_y"]:
            out["y"] = s * f("g") * scale[:, None]
        return out
    if case["kind"] == "norm_bwd":
        h, up = f("x"), f("dy")
        size = torch.sqrt(torch.sum(h ** 2, 1, keepdim=True) / case["d"] + EPS)
        unit = h / size
        back = up * f("g")
        dx = (back - unit * torch.sum(back * unit, 1, keepdim=True) / case["d"]) / size
        out = {"dx": dx if st["residual"] is None else dx + f("residual")}
        if case["want_dg"]:
            out["dg"] = torch.einsum("mc,mc->c", up, unit)
        return out
    if case["kind"] in ("product", "layer"):
        if 2.0 * case["M"] * case["K"] * case["N"] > 1e14:
            return None
        if case["kind"] == "product":
            codes, step = f("x"), f("x_scales")
        else:
            v = st["x"].float() if st["col_scale"] is None else st["x"].float() * st["col_scale"]
            codes, a = _codes64(v)
            step = (f("x") if st["col_scale"] is None else f("x") * f("col_scale")).abs().max(dim=1)[0] / 127
            step[a < TINY] = 0
        y = torch.einsum("mk,nk->mn", codes * step[:, None], f("w") if st["w_scales"] is None else f("w") * f("w_scales")[:, None])
        for k in ("bias", "residual"):
            if st[k] is not None:
                y += f(k)
        return {"y": y}
    # distill: row by row in blocks, from the definition
    M, V, T, (wc, wk) = case["M"], case["V"], case["temperature"], st["weights"]
    y = st["labels"]
    valid = torch.ones(M, dtype=torch.bool, device="cuda") if y is None else (y >= 0) & (y < V)
    n = max(1, int(valid.sum()))
    rows, grads = [], []
    for a in range(0, M, 512):
        z, ix, t, ok = f("logits")[a:a + 512], st["top_idx"][a:a + 512].long(), f("top_logits")[a:a + 512], valid[a:a + 512]
        live = ((ix >= 0) & (ix < V)).double()
        e = live * torch.exp((t - t.max(dim=1, keepdim=True)[0]) / T)
        q = e / e.sum(dim=1, keepdim=True).clamp(min=1e-300)
        Q = torch.zeros_like(z).scatter_add_(1, ix.clamp(min=0), q)
        zt = z / T
        lse = torch.logsumexp(zt, 1, keepdim=True)
        has = live.any(dim=1, keepdim=True).double()
        grad = wk * T * (torch.exp(zt - lse) * has - Q)
        row = wk * T * T * (torch.special.xlogy(q, q).sum(1) - (Q * (zt - lse)).sum(1))
        if y is not None:
            one = torch.zeros_like(z).scatter_(1, y[a:a + 512].long().clamp(min=0)[:, None], 1.0)
            lse = torch.logsumexp(z, 1, keepdim=True)
            grad = grad + wc * (torch.exp(z - lse) - one)
            row = row + wc * (lse[:, 0] - (z * one).sum(1))
        rows.append(torch.where(ok, row, torch.zeros_like(row)))
        grads.append(grad * (ok.double() / n)[:, None])
    row = torch.cat(rows)
    return {"loss": row.sum() / n, "rows": row, "dlogits": torch.cat(grads)}
