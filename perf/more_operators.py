"""Operators of a language model's layers between the token table and the loss: cases, plain forms and 64-bit values.

Three operators with their gradients:

    product       out = act(x w^T + bias) + residual, pre = x w^T + bias          (w as [out, in] or as [in, out])
    product_grad  dz = dout * act'(pre), dx = dz w, dw = dz^T x, db = column sums of dz
    join          y = c x + gate * post(f), h = pre(y): a block's branch f joins the residual stream x behind a norm of its
                  own, and the next block's input is normed in the same pass.  post and pre are an RMS norm or a layer norm with
                  learned weights (a layer norm with biases too); gate is nothing, a vector or one vector per group of rows
    join_grad     gradients of x, f, both norms' weights, both biases and the gate from those of y and h
    logp          log probability of a given token per row of logits (scaled by 1 / temperature), the entropy of the row, and
                  its most probable tokens with their log probabilities (ties: the lowest token)
    logp_grad     gradient of the logits from those of the log probability and of the entropy

``run`` takes them through the package where ``own`` is true and through elementary torch operations in 32 bits where it
is false.
"""
import math

import torch

own = False

F32, BF16 = "float32", "bfloat16"
PRODUCT_MAX, JOIN_MAX, LOGITS_MAX = 16384 * 2048 * 8192, 65536 * 2048, 16384 * 50257


# ---- cases ------------------------------------------------------------------------------------------------------
def _product(name, op, tokens, n_in, n_out, act="none", bias=False, residual=False, layout="out_in", out=BF16, pre=False):
    return {"name": name, "op": op, "tokens": tokens, "n_in": n_in, "n_out": n_out, "act": act, "bias": bias, "residual": residual,
            "layout": layout, "out": out, "pre": pre}


def _join(name, op, groups, rows, dim, kind="rms", post=True, gate="none", stream=F32, branch=BF16, grad=BF16, scale=1.0):
    return {"name": name, "op": op, "groups": groups, "rows": rows, "dim": dim, "kind": kind, "post": post, "gate": gate,
            "stream": stream, "branch": branch, "grad": grad, "scale": scale}


def _logp(name, op, tokens, vocab, dtype=BF16, scale=1.0, top=0, ids="int64", ignored=0.0, masked=0.0, entropy=True):
    return {"name": name, "op": op, "tokens": tokens, "vocab": vocab, "dtype": dtype, "scale": scale, "top": top, "ids": ids,
            "ignored": ignored, "masked": masked, "entropy": entropy}


def listed():
    return [
        # one token of a decode loop through the LLaMA-1B-shaped feed-forward's first matrix
        _product("product_decode", "product", 1, 2048, 8192, act="silu"),
        # a training micro-batch of 16384 tokens through the same matrix, the values before the activation kept
        _product("product_up", "product", 16384, 2048, 8192, act="gelu", bias=True, pre=True),
        # a small odd model of the kind tests and ablations train: rows that are not multiples of 16 bytes
        _product("product_grad_odd", "product_grad", 1000, 513, 1001, act="gelu_tanh", bias=True, out=F32),
        # the way back through the LLaMA-1B-shaped second matrix, stored as [in, out]
        _product("product_grad_down", "product_grad", 16384, 8192, 2048, act="none", bias=True, layout="in_out"),
        # one token of a decode loop: the join between two blocks
        _join("join_decode", "join", 1, 1, 2048, gate="vector"),
        # 64 K tokens of the LLaMA-1B shape, a gate per sequence
        _join("join_long", "join", 32, 2048, 2048, gate="group"),
        # a small odd model, layer norms with biases, everything in fp32
        _join("join_grad_odd", "join_grad", 1, 300, 513, kind="layer", gate="vector", branch=F32, grad=F32, scale=0.7),
        # a micro-batch of the GPT-2-small shape on a bf16 stream
        _join("join_grad_batch", "join_grad", 16, 1024, 768, kind="layer", gate="vector", stream=BF16),
        # what a server returns beside one generated token: log probability, entropy, 20 alternatives
        _logp("logp_decode", "logp", 1, 50257, top=20, scale=1.25, ids="int32"),
        # scoring a micro-batch of the GPT-2-small shape, 5 alternatives, a twentieth of the positions ignored
        _logp("logp_batch", "logp", 16384, 50257, top=5, ignored=0.05),
        # a fine-tuning step on a few tokens of a small odd vocabulary, part of it masked
        _logp("logp_grad_odd", "logp_grad", 300, 4099, dtype=F32, masked=0.3, ignored=0.1, ids="int32"),
        # the loss's gradient of 16 K tokens of the LLaMA-1B-shaped vocabulary, with an entropy bonus
        _logp("logp_grad_batch", "logp_grad", 16384, 32000),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["product", "product_grad", "join", "join_grad", "logp", "logp_grad"])
    if op in ("product", "product_grad"):
        n_in, n_out = _log(rng, 48, 8192), _log(rng, 48, 8192)
        if rng.random() < 0.6:
            n_in, n_out = max(64, n_in // 64 * 64), max(64, n_out // 64 * 64)
        tokens = _log(rng, 1, min(16384, PRODUCT_MAX // (n_in * n_out)))
        act = rng.choice(["none", "none", "relu", "gelu", "gelu_tanh", "silu"])
        return {"op": op, "tokens": tokens, "n_in": n_in, "n_out": n_out, "act": act, "bias": rng.choice([True, False]),
                "residual": op == "product" and rng.choice([True, False]), "layout": rng.choice(["out_in", "out_in", "in_out"]),
                "out": rng.choice([BF16, BF16, F32]), "pre": op == "product" and act != "none" and rng.choice([True, False])}
    if op in ("join", "join_grad"):
        dim = _log(rng, 64, 8192)
        if rng.random() < 0.6:
            dim = max(64, dim // 64 * 64)
        most = JOIN_MAX // 2 if op == "join_grad" else JOIN_MAX
        rows = _log(rng, 1, min(65536, most // dim))
        groups = rng.choice([1, 2, 5, 16, 64])
        groups = groups if groups <= rows else 1
        stream, branch = rng.choice([(F32, BF16), (F32, BF16), (BF16, BF16), (F32, F32)])
        return {"op": op, "groups": groups, "rows": rows // groups, "dim": dim, "kind": rng.choice(["rms", "rms", "layer"]),
                "post": rng.choice([True, False]), "gate": rng.choice(["none", "vector", "group"]), "stream": stream,
                "branch": branch, "grad": rng.choice([BF16, F32]), "scale": rng.choice([1.0, 0.5])}
    vocab = _log(rng, 256, 131072)
    tokens = _log(rng, 1, min(65536, LOGITS_MAX // vocab))
    dtype = rng.choice([BF16, BF16, F32])
    if dtype == F32:
        tokens = max(1, tokens // 2)
    return {"op": op, "tokens": tokens, "vocab": vocab, "dtype": dtype, "scale": rng.choice([1.0, 1.0, 1.25, 0.5]),
            "top": rng.choice([0, 1, 5, 20]) if op == "logp" else 0, "ids": rng.choice(["int32", "int64"]),
            "ignored": rng.choice([0.0, 0.05, 0.3]), "masked": rng.choice([0.0, 0.0, 0.3]), "entropy": rng.choice([True, True, False])}


_SIZE = {F32: 4, BF16: 2, "int32": 4, "int64": 8}


def work(case):
    op = case["op"]
    if op == "product":
        m, k, n = case["tokens"], case["n_in"], case["n_out"]
        size = _SIZE[case["out"]]
        bytes_ = 2 * (m * k + k * n) + m * n * size * (2 if case["residual"] else 1) + (4 * n if case["bias"] else 0) + (2 * m * n if case["pre"] else 0)
        return {"bytes": bytes_, "flops": 2 * m * k * n}
    if op == "product_grad":
        m, k, n = case["tokens"], case["n_in"], case["n_out"]
        size = _SIZE[case["out"]]
        bytes_ = 2 * (m * k + k * n + m * n + m * k) + k * n * size + (2 * m * n if case["act"] != "none" else 0) + (n * size if case["bias"] else 0)
        return {"bytes": bytes_, "flops": 4 * m * k * n}
    if op in ("join", "join_grad"):
        n = case["groups"] * case["rows"] * case["dim"]
        s, b = _SIZE[case["stream"]], _SIZE[case["branch"]]
        if op == "join":                     # x and f in, y and h out
            return {"bytes": n * 2 * (s + b), "flops": 12 * n}
        # y, the gradients of y and h in, those of x and f out; f itself where its norm or the gate needs it
        return {"bytes": n * (3 * s + (3 if case["post"] or case["gate"] != "none" else 2) * b), "flops": 30 * n}
    kept = case["tokens"] * (1.0 - case["ignored"])
    n = kept * case["vocab"]
    if op == "logp":
        return {"bytes": n * _SIZE[case["dtype"]] + case["tokens"] * (_SIZE[case["ids"]] + 8 + 8 * case["top"]), "flops": 6 * n}
    return {"bytes": (n + case["tokens"] * case["vocab"]) * _SIZE[case["dtype"]] + case["tokens"] * (_SIZE[case["ids"]] + 16), "flops": 8 * n}


# ---- inputs -----------------------------------------------------------------------------------------------------
def _dtype(name):
    return getattr(torch, name)


def _normal(gen, shape, dtype, std=1.0, mean=0.0):
    return torch.empty(shape, device="cuda", dtype=_dtype(dtype)).normal_(mean, std, generator=gen)


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)
    if case["op"] in ("product", "product_grad"):
        m, k, n = case["tokens"], case["n_in"], case["n_out"]
        s["x"] = _normal(gen, (m, k), BF16)
        s["w"] = _normal(gen, (n, k) if case["layout"] == "out_in" else (k, n), BF16, k ** -0.5)
        if case["op"] == "product":
            s["b"] = _normal(gen, (n,), F32, 0.1) if case["bias"] else None
            s["r"] = _normal(gen, (m, n), case["out"]) if case["residual"] else None
        else:
            s["dout"] = _normal(gen, (m, n), BF16, m ** -0.5)
            s["before"] = _normal(gen, (m, n), BF16) if case["act"] != "none" else None
        return s
    if case["op"] in ("join", "join_grad"):
        n, d = case["groups"] * case["rows"], case["dim"]
        layer, gate = case["kind"] == "layer", case["gate"]
        s["f"] = _normal(gen, (n, d), case["branch"], 0.5, 0.1)
        s["pre_w"], s["pre_b"] = _normal(gen, (d,), F32, 0.1, 1.0), _normal(gen, (d,), F32, 0.1) if layer else None
        s["post_w"] = _normal(gen, (d,), F32, 0.1, 0.5) if case["post"] else None
        s["post_b"] = _normal(gen, (d,), F32, 0.1) if case["post"] and layer else None
        s["g"] = None if gate == "none" else _normal(gen, (case["groups"] if gate == "group" else 1, d), F32, 0.3, 0.5)
        if case["op"] == "join":
            s["x"] = _normal(gen, (n, d), case["stream"], 2.0)
        else:
            s["y"] = _normal(gen, (n, d), case["stream"], 2.0)
            s["dy"], s["dh"] = _normal(gen, (n, d), case["stream"], 0.01), _normal(gen, (n, d), case["branch"], 0.01)
        return s
    n, v = case["tokens"], case["vocab"]
    x = torch.empty((n, v), device="cuda", dtype=_dtype(case["dtype"])).normal_(0.0, 2.5, generator=gen)
    ids = torch.randint(0, v, (n,), generator=gen, device="cuda")
    # a trained model gives most given tokens a high logit
    raised = torch.rand((n, 1), generator=gen, device="cuda") * 14.0
    x.scatter_(1, ids[:, None], raised.to(x.dtype))
    if case["masked"]:                       # tokens that a grammar or a filter forbids
        x.masked_fill_((torch.rand(v, generator=gen, device="cuda") < case["masked"])[None, :], float("-inf"))
    if case["ignored"]:
        ids[torch.rand(n, generator=gen, device="cuda") < case["ignored"]] = -1
    s["x"], s["token_ids"] = x, ids.to(_dtype(case["ids"]))
    if case["op"] == "logp_grad":
        s["dlogp"] = _normal(gen, (n,), F32, 0.5, -1.0) / n
        s["dentropy"] = _normal(gen, (n,), F32, 0.01) / n if case["entropy"] else None
        s["rowmax"], s["logsum"], s["ent"] = _row_values(x, case["scale"], torch.float64)
    return s


def _row_values(x, scale, dtype):
    """Largest logit, log of the sum of exp(scale (x - largest)) and entropy of every row, in fp32, a slab of rows at a time."""
    out = []
    step = max(1, (1 << 26) // x.shape[1])
    for i in range(0, x.shape[0], step):
        z = x[i:i + step].to(dtype)
        m = z.amax(1, keepdim=True)
        t = scale * (z - m)
        e = t.exp()
        total = e.sum(1)
        h = total.log() - torch.where(e > 0, e * t, 0.0).sum(1) / total
        out.append((m[:, 0].float(), total.log().float(), h.float()))
    return tuple(torch.cat(c) for c in zip(*out))


def prepare(case, seed):
    s = _inputs(case, seed)
    return _with_plan(s, case) if own else s


def _with_plan(s, case):
    """The plan, output buffers and workspace that a program keeps."""
    from paper_2605_04711_b200 import binding as B
    op, empty = case["op"], lambda shape, dtype: torch.empty(shape, dtype=_dtype(dtype), device="cuda")
    if op in ("product", "product_grad"):
        m, k, n = case["tokens"], case["n_in"], case["n_out"]
        p = s["plan"] = B.Linear(k, n, act=case["act"], layout=case["layout"])
        if op == "product":
            s["result"], s["kept"] = empty((m, n), case["out"]), empty((m, n), BF16) if case["pre"] else None
            s["ws"] = empty((p.workspace_bytes(m),), "uint8")
        else:
            s["dx"], s["dw"] = empty((m, k), BF16), empty(s["w"].shape, case["out"])
            s["db"] = empty((n,), case["out"]) if case["bias"] else None
            s["ws"] = empty((p.grad_workspace_bytes(m),), "uint8")
        return s
    if op in ("join", "join_grad"):
        n, d = case["groups"] * case["rows"], case["dim"]
        p = s["plan"] = B.Join(d, kind=case["kind"], scale=case["scale"])
        if op == "join":
            s["out_y"], s["out_h"] = empty((n, d), case["stream"]), empty((n, d), case["branch"])
        else:
            s["dx"], s["df"] = empty((n, d), case["stream"]), empty((n, d), case["branch"])
            for name, of in (("dpre_w", "pre_w"), ("dpre_b", "pre_b"), ("dpost_w", "post_w"), ("dpost_b", "post_b"), ("dg", "g")):
                s[name] = None if s[of] is None else empty(s[of].shape, case["grad"])
            s["ws"] = empty((p.grad_workspace_bytes(n),), "uint8")
        return s
    n = case["tokens"]
    s["plan"] = B.LogProbs(case["vocab"], scale=case["scale"], top=case["top"])
    if op == "logp":
        s["out"] = s["plan"].buffers(n, "cuda")
    else:
        s["stats"] = torch.stack([s["rowmax"], s["logsum"], s["ent"]], 1).contiguous()
        s["dx"] = torch.empty_like(s["x"])
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------
def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    op = s["op"]
    if op == "product":
        s["plan"].product(s["x"], s["w"], bias=s["b"], residual=s["r"], out=s["result"], pre=s["kept"], ws=s["ws"])
        return {"out": s["result"], "pre": s["kept"]} if s["pre"] else {"out": s["result"]}
    if op == "product_grad":
        s["plan"].grad(s["x"], s["w"], s["dout"], pre=s["before"], dx=s["dx"], dw=s["dw"], db=s["db"], ws=s["ws"])
        return _named(dx=s["dx"], dw=s["dw"], db=s["db"])
    if op == "join":
        s["plan"].join(s["x"], s["f"], s["pre_w"], pre_b=s["pre_b"], post_w=s["post_w"], post_b=s["post_b"], gate=s["g"], y=s["out_y"], h=s["out_h"])
        return {"y": s["out_y"], "h": s["out_h"]}
    if op == "join_grad":
        s["plan"].grad(s["y"], s["f"], s["dh"], s["pre_w"], dy=s["dy"], post_w=s["post_w"], post_b=s["post_b"], gate=s["g"], dx=s["dx"], df=s["df"],
                       dpre_w=s["dpre_w"], dpre_b=s["dpre_b"], dpost_w=s["dpost_w"], dpost_b=s["dpost_b"], dgate=s["dg"], ws=s["ws"])
        return _named(dx=s["dx"], df=s["df"], dpre_w=s["dpre_w"], dpre_b=s["dpre_b"], dpost_w=s["dpost_w"], dpost_b=s["dpost_b"], dgate=s["dg"])
    if op == "logp":
        out = s["plan"].logprobs(s["x"], s["token_ids"], out=s["out"])
        got = {"logp": out.logp, "entropy": out.entropy}
        return got | {"top_ids": out.top_ids, "top_logp": out.top_logp} if s["top"] else got
    return s["plan"].grad(s["x"], s["token_ids"], s["stats"], s["dlogp"], dentropy=s["dentropy"], dlogits=s["dx"])


def _named(**outputs):
    return {k: v for k, v in outputs.items() if v is not None}


def _act(z, act):
    if act == "relu":
        return z.clamp(min=0.0)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if act == "gelu_tanh":
        c = math.sqrt(2.0 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * z * z)
    s = 1.0 / (1.0 + torch.exp(-z))
    return s * (1.0 + z * (1.0 - s))


_EPS = 1e-6


def _hat(v, kind):
    """The row without its mean (a layer norm) over its standard deviation or root mean square, and one over that."""
    c = v - v.mean(1, keepdim=True) if kind == "layer" else v
    r = (c.square().mean(1, keepdim=True) + _EPS).rsqrt()
    return c * r, r


def _hat_grad(dhat, hat, r, kind):
    inner = dhat - hat * (dhat * hat).mean(1, keepdim=True)
    return r * (inner - dhat.mean(1, keepdim=True) if kind == "layer" else inner)


def _plain(s):
    op = s["op"]
    if op == "product":
        x, w = s["x"].float(), s["w"].float()
        z = x @ (w.t() if s["layout"] == "out_in" else w)
        if s["b"] is not None:
            z = z + s["b"]
        a = _act(z, s["act"])
        out = (a if s["r"] is None else a + s["r"].float()).to(_dtype(s["out"]))
        return {"out": out, "pre": z.to(torch.bfloat16)} if s["pre"] else {"out": out}
    if op == "product_grad":
        x, w, dz = s["x"].float(), s["w"].float(), s["dout"].float()
        if s["before"] is not None:
            dz = dz * _act_slope(s["before"].float(), s["act"])
        out_in = s["layout"] == "out_in"
        dx = (dz @ (w if out_in else w.t())).to(torch.bfloat16)
        dw = (dz.t() @ x if out_in else x.t() @ dz).to(_dtype(s["out"]))
        return _named(dx=dx, dw=dw, db=dz.sum(0).to(_dtype(s["out"])) if s["bias"] else None)
    if op in ("join", "join_grad"):
        f, kind, groups, d = s["f"].float(), s["kind"], s["groups"], s["dim"]
        u, fhat, fr = f, None, None
        if s["post"]:
            fhat, fr = _hat(f, kind)
            u = fhat * s["post_w"] if s["post_b"] is None else fhat * s["post_w"] + s["post_b"]
        spread = lambda t: t.view(groups, -1, d) if s["gate"] == "group" else t.view(1, -1, d)
        if op == "join":
            if s["g"] is not None:
                u = (spread(u) * s["g"][:, None, :]).view(-1, d)
            y = s["scale"] * s["x"].float() + u
            h = _hat(y, kind)[0] * s["pre_w"]
            if s["pre_b"] is not None:
                h = h + s["pre_b"]
            return {"y": y.to(_dtype(s["stream"])), "h": h.to(_dtype(s["branch"]))}
        t = _dtype(s["grad"])
        dh = s["dh"].float()
        yhat, yr = _hat(s["y"].float(), kind)
        dy = s["dy"].float() + _hat_grad(dh * s["pre_w"], yhat, yr, kind)
        du, dg = dy, None
        if s["g"] is not None:
            dg = spread(dy * u).sum(1).to(t)
            du = (spread(dy) * s["g"][:, None, :]).view(-1, d)
        df, dpost_w, dpost_b = du, None, None
        if s["post"]:
            dpost_w = (du * fhat).sum(0).to(t)
            dpost_b = None if s["post_b"] is None else du.sum(0).to(t)
            df = _hat_grad(du * s["post_w"], fhat, fr, kind)
        return _named(dx=(s["scale"] * dy).to(_dtype(s["stream"])), df=df.to(_dtype(s["branch"])), dpre_w=(dh * yhat).sum(0).to(t),
                      dpre_b=None if s["pre_b"] is None else dh.sum(0).to(t), dpost_w=dpost_w, dpost_b=dpost_b, dgate=dg)
    x, ids, v = s["x"].float(), s["token_ids"].long(), s["vocab"]
    kept = (ids >= 0) & (ids < v)
    at = torch.where(kept, ids, 0)[:, None]
    if op == "logp":
        m = x.amax(1, keepdim=True)
        t = (x - m) * s["scale"]
        e = t.exp()
        total = e.sum(1, keepdim=True)
        logsum = total.log()
        logp = torch.where(kept, (t.gather(1, at) - logsum)[:, 0], 0.0)
        entropy = (logsum - torch.where(e > 0, e * t, 0.0).sum(1, keepdim=True) / total)[:, 0]
        got = {"logp": logp, "entropy": torch.where(kept, entropy, 0.0)}
        if not s["top"]:
            return got
        best, best_logp, left = [], [], x.clone()
        for _ in range(s["top"]):            # the first of the largest that are left
            i = left.argmax(1, keepdim=True)
            best.append(torch.where(kept, i[:, 0], -1).to(torch.int32))
            best_logp.append(torch.where(kept, (t.gather(1, i) - logsum)[:, 0], 0.0))
            left.scatter_(1, i, float("-inf"))
        return got | {"top_ids": torch.stack(best, 1), "top_logp": torch.stack(best_logp, 1)}
    logq = (x - s["rowmax"][:, None]) * s["scale"] - s["logsum"][:, None]
    p = logq.exp()
    grad = -s["dlogp"][:, None] * p
    if s["dentropy"] is not None:
        grad = grad - s["dentropy"][:, None] * torch.where(p > 0, p * (logq + s["ent"][:, None]), 0.0)
    grad.scatter_add_(1, at, s["dlogp"][:, None])
    return torch.where(kept[:, None], grad * s["scale"], 0.0).to(s["x"].dtype)


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------
def exact(case, seed):
    s = _inputs(case, seed)
    return {"product": _exact_product, "product_grad": _exact_product_grad, "join": _exact_join, "join_grad": _exact_join_grad,
            "logp": _exact_logp, "logp_grad": _exact_logp_grad}[case["op"]](s)


def _slope64(z, act):
    """The activation and its derivative, the derivative by automatic differentiation."""
    z = z.double().requires_grad_(True)
    f = {"none": lambda q: q * 1.0, "relu": torch.relu, "gelu": lambda q: q * torch.special.ndtr(q),
         "gelu_tanh": lambda q: q * torch.sigmoid(math.sqrt(8.0 / math.pi) * (q + 0.044715 * q.pow(3))), "silu": lambda q: q * torch.sigmoid(q)}[act]
    with torch.enable_grad():
        a = f(z)
        return a.detach(), torch.autograd.grad(a.sum(), z)[0]


def _exact_product(s):
    w = s["w"].double() if s["layout"] == "in_out" else s["w"].double().t()
    z = torch.mm(s["x"].double(), w)
    if s["b"] is not None:
        z += s["b"].double()
    out = torch.empty_like(z)
    for rows, to in zip(z.split(4096), out.split(4096)):
        to.copy_(_slope64(rows, s["act"])[0])
    if s["r"] is not None:
        out += s["r"].double()
    return {"out": out, "pre": z} if s["pre"] else {"out": out}


def _exact_product_grad(s):
    dz = s["dout"].double()
    if s["before"] is not None:
        for rows, b in zip(dz.split(4096), s["before"].split(4096)):
            rows.mul_(_slope64(b, s["act"])[1])
    x, w = s["x"].double(), s["w"].double()
    if s["layout"] == "out_in":
        dx, dw = torch.mm(dz, w), torch.mm(dz.t(), x)
    else:
        dx, dw = torch.mm(dz, w.t()), torch.mm(x.t(), dz)
    return {"dx": dx, "dw": dw, "db": torch.mv(dz.t(), torch.ones(dz.shape[0], dtype=torch.float64, device="cuda"))} if s["bias"] else {"dx": dx, "dw": dw}


def _norm64(v, w, b, kind):
    if kind == "layer":
        var, mean = torch.var_mean(v, 1, correction=0, keepdim=True)
        n = (v - mean) / torch.sqrt(var + _EPS)
    else:
        n = v / torch.sqrt((v * v).sum(1, keepdim=True) / v.shape[1] + _EPS)
    n = n * w.double()
    return n if b is None else n + b.double()


def _join_slabs(s):
    """Row ranges of one group each, of at most about 2^24 elements."""
    step = max(1, (1 << 24) // s["dim"])
    for g in range(s["groups"]):
        for lo in range(g * s["rows"], (g + 1) * s["rows"], step):
            yield (g if s["gate"] == "group" else 0), slice(lo, min(lo + step, (g + 1) * s["rows"]))


def _branch64(s, f, g):
    u = _norm64(f, s["post_w"], s["post_b"], s["kind"]) if s["post"] else f
    return u if s["g"] is None else u * s["g"][g].double()


def _exact_join(s):
    y = torch.empty(s["f"].shape, dtype=torch.float64, device="cuda")
    h = torch.empty_like(y)
    for g, rows in _join_slabs(s):
        y[rows] = s["x"][rows].double() * s["scale"] + _branch64(s, s["f"][rows].double(), g)
        h[rows] = _norm64(y[rows], s["pre_w"], s["pre_b"], s["kind"])
    return {"y": y, "h": h}


def _exact_join_grad(s):
    """By automatic differentiation: of <h(y), dh> by y and the weights, then of <u(f), dy> by f and the rest."""
    wide = lambda t: None if t is None else t.double().requires_grad_(True)
    q = dict(s) | {k: wide(s[k]) for k in ("pre_w", "pre_b", "post_w", "post_b", "g")}
    leaves = [k for k in ("pre_w", "pre_b", "post_w", "post_b", "g") if q[k] is not None]
    dx = torch.empty(s["f"].shape, dtype=torch.float64, device="cuda")
    df = torch.empty_like(dx)
    for g, rows in _join_slabs(s):
        y, f = s["y"][rows].double().requires_grad_(True), s["f"][rows].double().requires_grad_(True)
        with torch.enable_grad():
            _norm64(y, q["pre_w"], q["pre_b"], s["kind"]).backward(s["dh"][rows].double())
            dy = s["dy"][rows].double() + y.grad
            (_branch64(q, f, g) * 1.0).backward(dy)
        dx[rows], df[rows] = dy * s["scale"], f.grad
    grads = {k: q[k].grad for k in leaves}
    return _named(dx=dx, df=df, dpre_w=grads["pre_w"], dpre_b=grads.get("pre_b"), dpost_w=grads.get("post_w"), dpost_b=grads.get("post_b"), dgate=grads.get("g"))


def _exact_logp(s):
    n, v, k = s["tokens"], s["vocab"], s["top"]
    dev, f64 = "cuda", torch.float64
    logp, entropy = torch.zeros(n, dtype=f64, device=dev), torch.zeros(n, dtype=f64, device=dev)
    top_ids, top_logp = torch.full((n, k), -1, dtype=torch.int32, device=dev), torch.zeros((n, k), dtype=f64, device=dev)
    step = max(1, (1 << 25) // v)
    for lo in range(0, n, step):
        ids = s["token_ids"][lo:lo + step].long()
        rows = torch.nonzero((ids >= 0) & (ids < v)).flatten()
        if rows.numel() == 0:
            continue
        x = s["x"][lo:lo + step][rows]
        logq = torch.log_softmax(x.double() * s["scale"], 1)
        logp[lo + rows] = logq.gather(1, ids[rows][:, None])[:, 0]
        entropy[lo + rows] = torch.special.entr(logq.exp()).sum(1)
        if k:
            order = torch.sort(x.float(), stable=True, dim=1, descending=True)[1][:, :k]
            top_ids[lo + rows], top_logp[lo + rows] = order.to(torch.int32), logq.gather(1, order)
    got = {"logp": logp, "entropy": entropy}
    return got | {"top_ids": top_ids, "top_logp": top_logp} if k else got


def _exact_logp_grad(s):
    n, v = s["tokens"], s["vocab"]
    out = torch.zeros((n, v), dtype=torch.float64, device="cuda")
    step = max(1, (1 << 25) // v)
    for lo in range(0, n, step):
        ids = s["token_ids"][lo:lo + step].long()
        rows = torch.nonzero((ids >= 0) & (ids < v)).flatten()
        if rows.numel() == 0:
            continue
        q = torch.softmax(s["x"][lo:lo + step][rows].double() * s["scale"], 1)
        d = -q * s["dlogp"][lo + rows].double()[:, None]
        d[torch.arange(rows.numel(), device="cuda"), ids[rows]] += s["dlogp"][lo + rows].double()
        if s["dentropy"] is not None:
            e = torch.special.entr(q)        # -q log q, zero at q = 0
            d += s["dentropy"][lo + rows].double()[:, None] * (e - q * e.sum(1, keepdim=True))
        out[lo + rows] = d * s["scale"]
    return out
