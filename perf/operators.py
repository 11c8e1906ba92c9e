"""The token table's and the gradient clip's operators: cases, plain forms and 64-bit values.

Four operators of one training step of a language model, around the optimizer step of this library:

    lookup   out[t, :] = scale * table[ids[t], :]                         (zeros where ids[t] is outside the table)
    grad     dtable[v, :] = scale * sum over t with ids[t] = v of dout[t, :]   (nothing for the pad row and ids outside)
    norm     norms[0] = sqrt(sum_i n_i^2), norms[1 + i] = n_i = sqrt(sum of block i's squared gradient)
    clip     dst_i = min(1, max_norm / (norms[0] + 1e-6)) * src_i for every block i, and the norms

``run`` takes them through the package where ``own`` is true and through elementary torch operations in 32 bits where
it is false.
"""
import math

import torch

own = False

F32, BF16 = "float32", "bfloat16"
TOKENS_MAX, LOOKUP_MAX, GRAD_MAX, PARAMS_MAX = 131072, 131072 * 2048, 65536 * 2048, 1139345408


# ---- cases ------------------------------------------------------------------------------------------------------
def _lookup(name, tokens, vocab, dim, scale=1.0, table=F32, out=BF16, ids="int64", ignored=0.0):
    return {"name": name, "op": "lookup", "tokens": tokens, "vocab": vocab, "dim": dim, "scale": scale, "table": table,
            "out": out, "ids": ids, "pad": 0.0, "ignored": ignored}


def _grad(name, tokens, vocab, dim, scale=1.0, act=BF16, grad=BF16, ids="int64", pad=0.0, ignored=0.0):
    return {"name": name, "op": "grad", "tokens": tokens, "vocab": vocab, "dim": dim, "scale": scale, "act": act,
            "grad": grad, "ids": ids, "pad": pad, "ignored": ignored}


def _blocks(name, op, layers, width, ff, vocab, positions, bias, src=BF16, dst=BF16, max_norm=1.0):
    return {"name": name, "op": op, "layers": layers, "width": width, "ff": ff, "vocab": vocab, "positions": positions,
            "bias": bias, "src": src, "dst": dst, "max_norm": max_norm}


def listed():
    return [
        # one token of a decode loop: the table of the LLaMA-1B-shaped workload, fp32 master weights, bf16 activations
        _lookup("lookup_decode", 1, 32000, 2048, scale=math.sqrt(2048.0)),
        # odd width, odd vocabulary, everything in fp32: a small model of the kind tests and ablations train
        _lookup("lookup_odd", 1000, 4099, 513, out=F32, ids="int32", ignored=0.02),
        # a training micro-batch of the GPT-2-small-shaped workload: 16 sequences of 1024
        _lookup("lookup_batch", 16384, 50257, 768),
        # 128 K tokens of a long-context step on the LLaMA-1B-shaped table
        _lookup("lookup_long", 131072, 32000, 2048, scale=math.sqrt(2048.0)),
        # a fine-tuning step on a few tokens, odd width, fp32 throughout
        _grad("grad_odd", 64, 1000, 257, act=F32, grad=F32, ids="int32", ignored=0.05),
        # the token table's gradient of the same micro-batch of the GPT-2-small-shaped workload
        _grad("grad_batch", 16384, 50257, 768),
        # 64 K tokens, a tenth of them padding, scaled embeddings: the LLaMA-1B-shaped table
        _grad("grad_long", 65536, 32000, 2048, scale=math.sqrt(2048.0), ids="int32", pad=0.1),
        # norm for the training log, 20 small tensors
        _blocks("norm_small", "norm", 2, 256, 1024, 1000, 0, False),
        # norm of every gradient of the GPT-2-small shape: 148 tensors, 124 M parameters
        _blocks("norm_gpt2_small", "norm", 12, 768, 3072, 50257, 1024, True),
        # clipping at the same small shape: launch latency
        _blocks("clip_small", "clip", 2, 256, 1024, 1000, 0, False),
        # gradients accumulated over micro-batches in fp32, clipped into the bf16 arrays that the optimizer step reads
        _blocks("clip_accumulated", "clip", 12, 768, 3072, 50257, 1024, True, src=F32),
        # every gradient of the LLaMA-1B shape: 146 tensors, 1.14 G parameters
        _blocks("clip_llama_1b", "clip", 16, 2048, 8192, 32000, 0, False),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["lookup", "grad", "norm", "clip"])
    if op in ("lookup", "grad"):
        vocab, dim = _log(rng, 256, 65536), _log(rng, 32, 4096)
        if rng.random() < 0.5:
            dim = max(32, dim // 64 * 64)
        case = {"op": op, "vocab": vocab, "dim": dim, "scale": rng.choice([1.0, math.sqrt(float(dim))]),
                "ids": rng.choice(["int32", "int64"]), "ignored": rng.choice([0.0, 0.0, 0.01, 0.2])}
        if op == "lookup":
            tokens = _log(rng, 1, min(TOKENS_MAX, LOOKUP_MAX // dim))
            return case | {"tokens": tokens, "table": rng.choice([F32, F32, BF16]), "out": rng.choice([BF16, BF16, F32]), "pad": 0.0}
        tokens = _log(rng, 1, min(TOKENS_MAX, GRAD_MAX // dim))
        return case | {"tokens": tokens, "act": rng.choice([BF16, BF16, F32]), "grad": rng.choice([BF16, BF16, F32]),
                       "pad": rng.choice([0.0, 0.1, 0.5])}
    width = _log(rng, 96, 2048)
    if rng.random() < 0.5:
        width = width // 32 * 32
    ff = rng.choice([4 * width, (8 * width) // 3])
    vocab, bias = _log(rng, 256, 50257), rng.choice([True, False])
    positions = rng.choice([0, 512, 1024])
    case = {"op": op, "width": width, "ff": ff, "vocab": vocab, "positions": positions, "bias": bias}
    per_layer = 4 * width * width + 3 * width * ff + 16 * width
    most = max(1, min(24, (PARAMS_MAX - width * (vocab + positions + 2)) // per_layer))
    src, dst = rng.choice([(BF16, BF16), (BF16, BF16), (F32, BF16), (F32, F32)])
    if src == F32 and most > 8:
        most = 8                                  # fp32 arrays move twice the bytes
    return case | {"layers": rng.randint(1, most), "src": src, "dst": dst, "max_norm": rng.choice([0.1, 1.0, 1.0, 1e6])}


def _shapes(case):
    """Rows and columns of every block, in forward order (a vector has one column)."""
    d, ff, vec = case["width"], case["ff"], lambda n: (n, 1)
    out = [(case["vocab"], d)] + ([(case["positions"], d)] if case["positions"] else [])
    for _ in range(case["layers"]):
        if case["bias"]:
            out += [vec(d), vec(d), (d, 3 * d), vec(3 * d), (d, d), vec(d), vec(d), vec(d), (d, ff), vec(ff), (ff, d), vec(d)]
        else:
            out += [vec(d)] + [(d, d)] * 4 + [vec(d), (ff, d), (ff, d), (d, ff)]
    return out + ([vec(d), vec(d)] if case["bias"] else [vec(d)])


def _layout(case):
    """Offsets and lengths of the blocks in one flat buffer, every start a multiple of 128 elements, and its length."""
    offs, lens, cur = [], [], 0
    for r, c in _shapes(case):
        offs.append(cur)
        lens.append(r * c)
        cur += (r * c + 127) // 128 * 128
    return offs, lens, cur


def _rank_probabilities(vocab):
    """A token's probability by frequency rank r: log((r + 2) / (r + 1)) / log(vocab + 1), close to 1 / rank."""
    r = torch.arange(vocab, dtype=torch.float64)
    return torch.log1p(1.0 / (r + 1.0)) / math.log(vocab + 1.0)


def work(case):
    if case["op"] in ("lookup", "grad"):
        n, v, d = case["tokens"], case["vocab"], case["dim"]
        size = {F32: 4, BF16: 2, "int32": 4, "int64": 8}
        kept = n * (1.0 - case["ignored"]) * (1.0 - case["pad"])
        if case["op"] == "lookup":     # the distinct rows that the tokens name are read once
            rows = float((1.0 - (1.0 - _rank_probabilities(v)).pow(kept)).sum())
            return {"bytes": rows * d * size[case["table"]] + n * size[case["ids"]] + n * d * size[case["out"]], "flops": n * d}
        return {"bytes": kept * d * size[case["act"]] + n * size[case["ids"]] + v * d * size[case["grad"]], "flops": n * d}
    total = sum(r * c for r, c in _shapes(case))
    read = total * (4 if case["src"] == F32 else 2)
    if case["op"] == "norm":
        return {"bytes": read, "flops": 2 * total}
    return {"bytes": read + total * (4 if case["dst"] == F32 else 2), "flops": 3 * total}


# ---- inputs -----------------------------------------------------------------------------------------------------
def _dtype(name):
    return getattr(torch, name)


def _ids(case, gen):
    """Token ids whose frequency falls like 1 / rank, ranks spread over the vocabulary; row 0 is the pad row, -1 marks
    ignored positions."""
    n, v = case["tokens"], case["vocab"]
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    rank = (torch.exp(u * math.log(v + 1.0)) - 1.0).long().clamp_(0, v - 1)
    ids = torch.randperm(v, generator=gen, device="cuda")[rank]
    if case["pad"]:
        ids[torch.rand(n, generator=gen, device="cuda") < case["pad"]] = 0
    if case["ignored"]:
        ids[torch.rand(n, generator=gen, device="cuda") < case["ignored"]] = -1
    return ids.to(_dtype(case["ids"]))


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)
    if case["op"] in ("lookup", "grad"):
        n, v, d = case["tokens"], case["vocab"], case["dim"]
        s["token_ids"] = _ids(case, gen)
        s["pad_id"] = 0 if case["pad"] else -1
        if case["op"] == "lookup":
            s["weights"] = torch.empty((v, d), device="cuda", dtype=_dtype(case["table"])).normal_(0.0, 0.02, generator=gen)
        else:
            s["dout"] = torch.empty((n, d), device="cuda", dtype=_dtype(case["act"])).normal_(0.0, 1e-3, generator=gen)
        return s
    offs, lens, total = _layout(case)
    flat = torch.empty(total, device="cuda", dtype=_dtype(case["src"])).normal_(0.0, 1.0, generator=gen)
    scales = (10.0 ** (torch.rand(len(offs), generator=gen, device="cuda") * 2.0 - 4.0)).tolist()
    for i, (o, n) in enumerate(zip(offs, lens)):
        flat[o:o + n] *= scales[i]
        flat[o + n:offs[i + 1] if i + 1 < len(offs) else total] = 0
    s["flat"], s["grads"] = flat, [flat[o:o + n] for o, n in zip(offs, lens)]
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    return _with_plan(s, case) if own else s


def _with_plan(s, case):
    """The plan or handle, workspace and output buffers that a program keeps."""
    from paper_2605_04711_b200 import binding as B
    dev = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")
    if case["op"] in ("lookup", "grad"):
        n, v, d = case["tokens"], case["vocab"], case["dim"]
        s["plan"] = B.Embedding(v, d, scale=case["scale"], pad_id=s["pad_id"])
        if case["op"] == "lookup":
            s["result"] = torch.empty((n, d), dtype=_dtype(case["out"]), device="cuda")
        else:
            s["result"] = torch.empty((v, d), dtype=_dtype(case["grad"]), device="cuda")
            s["ws"] = dev(s["plan"].grad_workspace_bytes(n))
        return s
    h = s["handle"] = B.Baoc([(r * c, r, c) for r, c in _shapes(case)], B.default_configs())
    s["ws"] = dev(h.clip_workspace_bytes())
    h.bind_clip_workspace(s["ws"])
    s["norms"] = torch.empty(1 + len(s["grads"]), dtype=torch.float32, device="cuda")
    s["src_table"] = B.pointer_table(s["grads"])
    if case["op"] == "clip":
        offs, lens, total = _layout(case)
        s["result"] = torch.zeros(total, dtype=_dtype(case["dst"]), device="cuda")
        s["dst_table"] = B.pointer_table([s["result"][o:o + n] for o, n in zip(offs, lens)])
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------
def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    if s["op"] == "lookup":
        return s["plan"].lookup(s["weights"], s["token_ids"], out=s["result"])
    if s["op"] == "grad":
        return s["plan"].grad(s["token_ids"], s["dout"], s["result"], ws=s["ws"])
    if s["op"] == "norm":
        return s["handle"].grad_norm(s["src_table"], s["norms"], dtype=_dtype(s["src"]))
    s["handle"].clip_grads(s["src_table"], s["dst_table"], s["max_norm"], s["norms"], src_dtype=_dtype(s["src"]), dst_dtype=_dtype(s["dst"]))
    return {"clipped": s["result"], "norms": s["norms"]}


def _plain(s):
    if s["op"] == "lookup":
        ids = s["token_ids"].long()
        inside = (ids >= 0) & (ids < s["vocab"])
        rows = s["weights"][torch.where(inside, ids, 0)].float() * s["scale"]
        return torch.where(inside[:, None], rows, 0.0).to(_dtype(s["out"]))
    if s["op"] == "grad":
        ids = s["token_ids"].long()
        kept = (ids >= 0) & (ids < s["vocab"]) & (ids != s["pad_id"])
        rows = torch.where(kept[:, None], s["dout"].float(), 0.0)
        total = torch.zeros((s["vocab"], s["dim"]), device="cuda").index_add_(0, torch.where(kept, ids, 0), rows)
        return (total * s["scale"]).to(_dtype(s["grad"]))
    squares = torch.stack([g.float().square().sum() for g in s["grads"]])
    total = squares.sum().sqrt()
    norms = torch.cat([total[None], squares.sqrt()])
    if s["op"] == "norm":
        return norms
    factor = (s["max_norm"] / (total + 1e-6)).clamp(max=1.0)
    return {"clipped": (s["flat"].float() * factor).to(_dtype(s["dst"])), "norms": norms}


def exact(case, seed):
    """The definitions in 64 bits."""
    s = _inputs(case, seed)
    if case["op"] == "lookup":
        out = torch.zeros((case["tokens"], case["dim"]), device="cuda", dtype=torch.float64)
        at = torch.nonzero(torch.logical_and(s["token_ids"] >= 0, s["token_ids"] < case["vocab"])).flatten()
        out[at] = s["weights"].index_select(0, s["token_ids"][at].long()).double() * case["scale"]
        return out
    if case["op"] == "grad":
        # the tokens in the order of their ids: a row's gradient is the difference of two running sums over them
        order = torch.argsort(s["token_ids"], stable=True)
        running = torch.zeros((case["tokens"] + 1, case["dim"]), device="cuda", dtype=torch.float64)
        torch.cumsum(s["dout"][order].double(), 0, out=running[1:])
        ends = torch.searchsorted(s["token_ids"][order].long(), torch.arange(case["vocab"], device="cuda"), right=True)
        starts = torch.searchsorted(s["token_ids"][order].long(), torch.arange(case["vocab"], device="cuda"))
        total = (running[ends] - running[starts]) * case["scale"]
        total[starts == ends] = 0.0
        if s["pad_id"] >= 0:
            total[s["pad_id"]] = 0.0
        return total
    norms = torch.stack([torch.linalg.vector_norm(g, dtype=torch.float64) for g in s["grads"]])
    norms = torch.cat([torch.linalg.vector_norm(norms)[None], norms])
    if case["op"] == "norm":
        return norms
    return {"clipped": s["flat"].double() * min(1.0, case["max_norm"] / (float(norms[0]) + 1e-6)), "norms": norms}
