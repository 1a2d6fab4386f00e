"""What the head in 8-bit floating point and the operators on either side of it are measured on: its product with a scale for
each block of 128, forward and backward; the selection of a beam search over its logits, and the reordering of what the beams
keep; and dropout of the hidden states in front of it, with a mask that is never stored.  Each with its plain form.

A block of 128 values (of a row of hidden states or gradients; 128 x 128 of the matrix) is held as e4m3 times a power of two,
the smallest 2^e >= 2^-127 with max |x| <= 448 2^e; products are of the values that these stand for.

A case is an operator (`op`) and its sizes:

  logits   N rows of hidden states, quantised within the call, against V e4m3 rows of D as a served head keeps them, and a bias
  train    logits of a head whose matrix is a parameter (quantised within the call), and the gradients of hidden states, matrix and
           bias from those of the logits: dH = q(dY) q(W), dW = q(dY)^T q(H) with dY and H in blocks along the rows, db = sum of dY
  select   B sequences of `beams` beams: the K best of score + log softmax(x / T) over beams and vocabulary, equal ones by beam and
           token; a finished beam goes on with its score and the end token alone; entries of -inf are excluded
  reorder  new[b, k] = old[b, parent[b, k]] for all that the beams keep: token histories, hidden states, keys and values of layers
  dropout  y = x / (1 - p) or 0, and the same of the gradient: element i is kept where 16-bit number i % 8 of the Philox4x32-10
           block at counter (i / 8, offset) with key `seed` is at least 65536 p, rounded; 1 - p is that of the rounded p

Sizes are those of the repository's own workloads (`paper_2603_25011_amd/inputs.py`), tests and sweeps: hidden sizes
up to 1024 with 768 as the ordinary one, 30522 and 250002 vocabulary entries, batches from one query to many documents.
"""
import math

import torch

own = False
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _product(name, op, N, D, V, dtype="bf16", out="f32"):
    return {"name": name, "op": op, "N": N, "D": D, "V": V, "dtype": dtype, "out": out}


def _select(name, B, beams, V, K, dtype="f32", temperature=1.0, excluded=0.0, finished=0.0, pitch=0):
    return {"name": name, "op": "select", "B": B, "beams": beams, "V": V, "K": K, "dtype": dtype, "temperature": temperature,
            "excluded": excluded, "finished": finished, "pitch": pitch}


def _reorder(name, B, beams, history, D, layers, heads, width, length):
    return {"name": name, "op": "reorder", "B": B, "beams": beams, "history": history, "D": D, "layers": layers, "heads": heads,
            "width": width, "length": length}


def _dropout(name, rows, cols, p, dtype="bf16"):
    return {"name": name, "op": "dropout", "rows": rows, "cols": cols, "p": p, "dtype": dtype}


def listed():
    return [
        # the last token of one query: the smallest product, latency counts
        _product("logits_one_token", "logits", 1, 768, 30522),
        # a few beams against the multilingual vocabulary: reading the matrix is what takes time
        _product("logits_few_tokens", "logits", 12, 1024, 250002, out="bf16"),
        # a teacher over a batch of documents
        _product("logits_documents", "logits", 8192, 768, 30522, out="bf16"),
        # a small float32 model with odd sizes
        _product("train_ragged_float32", "train", 2561, 312, 31091, dtype="f32"),
        # a training step on documents, logits and their gradients kept in bfloat16
        _product("train_documents", "train", 8192, 768, 30522, out="bf16"),
        # one query expanded with four beams: the smallest selection, latency counts
        _select("select_one_query", 1, 4, 30522, 8),
        # expansion of a batch of documents, logits in the type that the 8-bit product stores
        _select("select_documents", 64, 8, 30522, 16, dtype="bf16"),
        # multilingual beams, rows of a wider array, a tenth of the vocabulary excluded, a fifth of the beams at their end
        _select("select_multilingual", 24, 10, 250002, 20, temperature=0.7, excluded=0.1, finished=0.2, pitch=250016),
        # histories and last hidden states of one query's beams: latency counts
        _reorder("reorder_one_query", 1, 4, 33, 768, 0, 0, 0, 0),
        # keys and values of every layer of an expansion of documents
        _reorder("reorder_layers", 32, 8, 48, 768, 12, 12, 64, 40),
        # hidden states of one query
        _dropout("dropout_query", 32, 768, 0.1, dtype="f32"),
        # hidden states of a batch of documents
        _dropout("dropout_documents", 32768, 1024, 0.1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: sizes over the logarithm of their range, most hidden sizes those of encoders, now and then any
    multiple of 8 (dropout: any at all); no dearer than the largest case of its operator in `listed`."""
    while True:
        op = rng.choice(["logits", "logits", "train", "train", "select", "select", "reorder", "dropout"])
        dtype = "f32" if rng.random() < 0.3 else "bf16"
        D = rng.choice([128, 256, 312, 384, 512, 768, 768, 1024, 1024]) if rng.random() < 0.7 else 8 * rng.randint(8, 128)
        V = _log_int(rng, 1000, 250002)
        if op in ("logits", "train"):
            N = _log_int(rng, 1, 16) if op == "logits" and rng.random() < 0.4 else _log_int(rng, 1, 8192)
            c = _product("", op, N, D, V, dtype, rng.choice(["f32", "bf16"]))
            limit = 2561 * 312 * 31091 if op == "train" and "f32" in (c["dtype"], c["out"]) else 8192 * 768 * 30522
            if N * D * V > limit or N * V > 8192 * 30522:
                continue
        elif op == "select":
            beams = _log_int(rng, 1, 32)
            c = _select("", _log_int(rng, 1, 128), beams, V, min(64, rng.choice([1, 2]) * beams), dtype, rng.choice([1.0, 1.0, 0.7, 2.0]),
                        rng.choice([0.0, 0.0, 0.1, 0.5]), rng.choice([0.0, 0.2]), rng.choice([0, 0, V + rng.randint(1, 64)]))
            if c["B"] * beams * V > 24 * 10 * 250002:
                continue
        elif op == "reorder":
            layers = rng.choice([0, 1, 6, 12])
            c = _reorder("", _log_int(rng, 1, 64), _log_int(rng, 1, 16), rng.randint(1, 64), D, layers, rng.choice([1, 4, 12]) if layers else 0,
                         rng.choice([32, 48, 64]) if layers else 0, _log_int(rng, 1, 64) if layers else 0)
            if c["B"] * c["beams"] * layers * c["heads"] * c["width"] * c["length"] > 32 * 8 * 12 * 12 * 64 * 40:
                continue
        else:
            cols = D if rng.random() < 0.6 else rng.randint(1, 1024)
            c = _dropout("", _log_int(rng, 1, 32768), cols, rng.choice([0.1, 0.1, 0.15, 0.5, round(rng.random(), 3)]), dtype)
        del c["name"]
        return c


class State:
    """Inputs of one pass and the buffers that a program keeps beside them."""


def _normal(gen, shape, std, dtype):
    x = torch.empty(shape, dtype=dtype, device=DEV)
    for r in range(0, shape[0], 16384):
        n = min(16384, shape[0] - r)
        x[r:r + n] = torch.randn((n,) + tuple(shape[1:]), device=DEV, generator=gen).mul_(std).to(dtype)
    return x


def _up(n, m):
    return (n + m - 1) // m * m


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    s = State()
    s.case = dict(case)
    return {"logits": _prepare_product, "train": _prepare_product, "select": _prepare_select, "reorder": _prepare_reorder,
            "dropout": _prepare_dropout}[case["op"]](s, case, gen, int(seed))


def _prepare_product(s, case, gen, seed):
    N, D, V = case["N"], case["D"], case["V"]
    td, to = TYPES[case["dtype"]], TYPES[case["out"]]
    # hidden states behind a norm, a few channels larger than the others; a trained matrix, rows of different norms
    channels = torch.exp(torch.randn((D,), device=DEV, generator=gen).mul_(0.5))
    s.H = (_normal(gen, (N, D), 1.0, torch.float32) * channels).to(td)
    W = _normal(gen, (V, D), 0.05, torch.float32).mul_(torch.rand((V, 1), device=DEV, generator=gen).add_(0.5))
    s.bias = torch.randn((V,), device=DEV, generator=gen).mul_(0.1)
    if case["op"] == "train":
        s.H, s.W, s.bias = s.H.requires_grad_(True), W.to(td).requires_grad_(True), s.bias.requires_grad_(True)
        # gradients of a loss over a vocabulary: most next to nothing, a few of each row large, tokens of different weight
        s.dY = _normal(gen, (N, V), 3e-5 / N, to)
        hot = torch.randint(0, V, (N, min(V, 32)), device=DEV, generator=gen)
        s.dY.scatter_(1, hot, torch.randn(hot.shape, device=DEV, generator=gen).mul_(0.05 / N).to(to))
        s.dY.mul_(torch.rand((N, 1), device=DEV, generator=gen).add_(0.5).to(to))
        return s
    # the matrix as a loaded head keeps it: e4m3 rows padded with zeros to a multiple of 128, and the exponents (+ 127) of its blocks,
    # those of four blocks of a row beside each other, [blocks of 512 columns][rows][4]
    rows, cols = _up(V, 128), _up(D, 128)
    padded = torch.zeros((rows, cols), device=DEV)
    padded[:V, :D] = W
    tiles = padded.view(rows // 128, 128, cols // 128, 128)
    f, x = torch.frexp(tiles.abs().amax(dim=(1, 3)))
    e = (x - 9 + (f > 0.875).to(torch.int32)).clamp_(min=-127)
    s.W8 = (tiles * torch.exp2(-e.double()).float()[:, None, :, None]).to(torch.float8_e4m3fn).view(torch.uint8).view(rows, cols)[:V].contiguous()
    quads = torch.zeros((rows // 128, _up(cols, 512) // 128), dtype=torch.uint8, device=DEV)
    quads[:, :cols // 128] = (e + 127).to(torch.uint8)
    s.w_exp = quads.repeat_interleave(128, dim=0)[:V].view(V, -1, 4).transpose(0, 1).contiguous()
    s.out = torch.empty((N, V), dtype=to, device=DEV)
    s.ws = torch.empty((N * (cols + 4 * s.w_exp.shape[0]) + 1024,), dtype=torch.uint8, device=DEV)
    return s


def _prepare_select(s, case, gen, seed):
    B, beams, V, K = case["B"], case["beams"], case["V"], case["K"]
    td = TYPES[case["dtype"]]
    # logits as a head gives them: most near zero, a few of each row well above; beams of a sequence have much in common
    s.X = _normal(gen, (B * beams, case["pitch"] or V), 1.5, td)[:, :V]
    hot = torch.randint(0, V, (B, 1, min(V, 32)), device=DEV, generator=gen).expand(B, beams, -1).reshape(B * beams, -1)
    s.X.scatter_(1, hot, torch.rand(hot.shape, device=DEV, generator=gen).mul_(8.0).add_(2.0).to(td))
    if case["excluded"]:
        out = torch.rand(V, device=DEV, generator=gen) < case["excluded"]
        out[:min(V, 256)] = False
        s.X.masked_fill_(out, -math.inf)
    # scores of beams in order, as the step before left them
    s.scores = torch.rand((B, beams), device=DEV, generator=gen).mul_(2.0).cumsum(dim=1).neg_().sub_(5.0).contiguous()
    s.finished = None
    if case["finished"]:
        s.finished = torch.rand((B, beams), device=DEV, generator=gen) < case["finished"]
        s.finished[:, 0] = False
    s.end_id = 2
    s.values = torch.empty((B, K), dtype=torch.float32, device=DEV)
    s.parents = torch.empty((B, K), dtype=torch.int32, device=DEV)
    s.tokens = torch.empty((B, K), dtype=torch.int32, device=DEV)
    s.ws = torch.empty((32 << 20,), dtype=torch.uint8, device=DEV)
    return s


def _prepare_reorder(s, case, gen, seed):
    B, beams = case["B"], case["beams"]
    s.states = [torch.randint(0, 30522, (B, beams, case["history"]), device=DEV, generator=gen, dtype=torch.int32),
                _normal(gen, (B, beams, case["D"]), 1.0, torch.bfloat16)]
    for _ in range(2 * case["layers"]):
        s.states.append(_normal(gen, (B, beams, case["heads"], case["length"], case["width"]), 1.0, torch.bfloat16))
    # the better beams have the more children
    s.parents = torch.rand((B, beams), device=DEV, generator=gen).square_().mul_(beams).floor_().clamp_(max=beams - 1).to(torch.int32)
    s.out = [torch.empty_like(x) for x in s.states]
    return s


def _prepare_dropout(s, case, gen, seed):
    td = TYPES[case["dtype"]]
    s.x = _normal(gen, (case["rows"], case["cols"]), 1.0, td).requires_grad_(True)
    s.dy = _normal(gen, (case["rows"], case["cols"]), 1e-3, td)
    s.seed, s.offset = seed * 2654435761 % (1 << 62), seed % 1000003
    return s


def run(s):
    c = s.case
    if not own:
        with torch.no_grad():
            return {"logits": _plain_logits, "train": _plain_train, "select": _plain_select, "reorder": _plain_reorder,
                    "dropout": _plain_dropout}[c["op"]](s, c)
    from paper_2603_25011_amd import beam, dropout, fp8
    from paper_2603_25011_amd import binding as lsr
    kind = {"f32": lsr.LSR_F32, "bf16": lsr.LSR_BF16}
    if c["op"] == "logits":
        lsr.lsr_fp8_matmul(c["N"], c["V"], c["D"], kind[c["dtype"]], kind[c["out"]], s.H, c["D"], None,
                           s.W8, s.W8.shape[1], s.w_exp, s.bias, s.out, c["V"], s.ws)
        return s.out
    if c["op"] == "train":
        out = fp8.fp8_logits(s.H, s.W, s.bias, TYPES[c["out"]])
        dH, dW, db = torch.autograd.grad(out, (s.H, s.W, s.bias), s.dY)
        return {"logits": out.detach(), "dH": dH, "dW": dW, "db": db}
    if c["op"] == "select":
        lsr.lsr_beam_select(c["B"], c["beams"], c["V"], c["K"], kind[c["dtype"]], c["temperature"], s.X, s.X.stride(0), s.scores, s.finished,
                            s.end_id, s.values, s.parents, s.tokens, s.ws)
        return {"scores": s.values, "beams": s.parents, "tokens": s.tokens}
    if c["op"] == "reorder":
        return beam.beam_reorder(s.states, s.parents, out=s.out)
    y = dropout.dropout(s.x, c["p"], s.seed, s.offset)
    return {"y": y.detach(), "dx": torch.autograd.grad(y, s.x, s.dy)[0]}


def _blocks(x):
    """The values that rows of blocks of 128 stand for: e4m3 times a power of two for each block (x: [rows, columns], float32)."""
    rows, cols = x.shape
    t = torch.nn.functional.pad(x, (0, -cols % 128)).reshape(rows, -1, 128)
    f, e = torch.frexp(t.abs().amax(dim=2, keepdim=True))
    e = (e - 9 + (f > 0.875).to(torch.int32)).clamp_(min=-127).float()
    return ((t * torch.exp2(-e)).to(torch.float8_e4m3fn).float() * torch.exp2(e)).view(rows, -1)[:, :cols]


def _square_blocks(x):
    """The same with one power of two for each 128 x 128 of a matrix."""
    rows, cols = x.shape
    t = torch.nn.functional.pad(x, (0, -cols % 128, 0, -rows % 128))
    t = t.view(t.shape[0] // 128, 128, -1, 128)
    f, e = torch.frexp(t.abs().amax(dim=(1, 3), keepdim=True))
    e = (e - 9 + (f > 0.875).to(torch.int32)).clamp_(min=-127).float()
    return ((t * torch.exp2(-e)).to(torch.float8_e4m3fn).float() * torch.exp2(e)).view(t.shape[0] * 128, -1)[:rows, :cols]


def _plain_logits(s, c):
    scale = torch.exp2(s.w_exp.float() - 127.0).transpose(0, 1).reshape(c["V"], -1)[:, :s.W8.shape[1] // 128]
    w = (s.W8.view(torch.float8_e4m3fn).float().view(c["V"], -1, 128) * scale[:, :, None]).view(c["V"], -1)[:, :c["D"]]
    return (_blocks(s.H.float()) @ w.t() + s.bias).to(TYPES[c["out"]])


def _plain_train(s, c):
    h, w, g = s.H.float(), _square_blocks(s.W.float()), s.dY.float()
    out = (_blocks(h) @ w.t() + s.bias).to(s.dY.dtype)
    dH = (_blocks(g) @ w).to(s.H.dtype)
    dW = (_blocks(g.t()) @ _blocks(h.t()).t()).to(s.W.dtype)
    return {"logits": out, "dH": dH, "dW": dW, "db": g.sum(dim=0)}


def _plain_select(s, c):
    # scores in 64 bits: candidates of different beams lie close together
    B, beams, V, K = c["B"], c["beams"], c["V"], c["K"]
    z = s.X.double() / c["temperature"]
    most = z.amax(dim=1, keepdim=True)
    z = z - (most + (z - most).exp().sum(dim=1, keepdim=True).log())
    # the K best of each beam: one whole number for each logit that orders as the pair (value, lowest token first) does
    bits = s.X.float().contiguous().view(torch.int32)
    order = torch.where(bits < 0, bits ^ 0x7fffffff, bits).long()
    key = order * (1 << 32) + ((1 << 32) - 1 - torch.arange(V, device=DEV))
    best = (1 << 32) - 1 - (key.topk(min(K, V), dim=1).values & 0xffffffff)
    score = (z.gather(1, best) + s.scores.double().reshape(-1, 1)).view(B, beams, -1)
    best = best.view(B, beams, -1)
    if s.finished is not None:
        only = s.finished[:, :, None]
        first = torch.arange(best.shape[2], device=DEV) == 0
        score = torch.where(only, torch.where(first, s.scores.double()[:, :, None], -math.inf), score)
        best = torch.where(only, s.end_id, best)
    score, at = torch.sort(score.reshape(B, -1), dim=1, descending=True, stable=True)
    score, at = score[:, :K], at[:, :K]
    return {"scores": score.float(), "beams": (at // best.shape[2]).to(torch.int32), "tokens": best.reshape(B, -1).gather(1, at).to(torch.int32)}


def _plain_reorder(s, c):
    at = s.parents.long()
    batch = torch.arange(c["B"], device=DEV)[:, None]
    return [x[batch, at] for x in s.states]


def _plain_dropout(s, c):
    mask = (1 << 32) - 1
    n = c["rows"] * c["cols"]
    i = torch.arange((n + 7) // 8, device=DEV)
    v0, v1, v2, v3 = i & mask, i >> 32, torch.full_like(i, s.offset & mask), torch.full_like(i, s.offset >> 32)
    k0, k1 = s.seed & mask, s.seed >> 32
    for _ in range(10):
        a, b = v0 * 0xD2511F53, v2 * 0xCD9E8D57
        v0, v1, v2, v3 = ((b >> 32) & mask) ^ v1 ^ k0, b & mask, ((a >> 32) & mask) ^ v3 ^ k1, a & mask
        k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
    numbers = torch.stack([v0 & 0xffff, v0 >> 16, v1 & 0xffff, v1 >> 16, v2 & 0xffff, v2 >> 16, v3 & 0xffff, v3 >> 16], dim=1)
    least = round(c["p"] * 65536)
    keep = (numbers.view(-1)[:n] >= least).view(s.x.shape)
    scale = 65536.0 / (65536 - least) if least < 65536 else 0.0
    return {"y": torch.where(keep, s.x.float() * scale, 0.0).to(s.x.dtype), "dx": torch.where(keep, s.dy.float() * scale, 0.0).to(s.x.dtype)}


def work(case):
    """Every input read once, every output written once; two operations for each multiply-add of a product."""
    e = {"f32": 4, "bf16": 2}
    if case["op"] in ("logits", "train"):
        N, D, V = case["N"], case["D"], case["V"]
        h, o = e[case["dtype"]], e[case["out"]]
        if case["op"] == "logits":
            return {"bytes": N * D * h + V * D + 4 * V + N * V * o, "flops": 2.0 * N * D * V}
        return {"bytes": 2 * (N * D + V * D) * h + 8 * V + 2 * N * V * o, "flops": 6.0 * N * D * V}
    if case["op"] == "select":
        rows = case["B"] * case["beams"] - case["B"] * (case["beams"] - 1) * case["finished"]
        return {"bytes": rows * case["V"] * e[case["dtype"]] + 5 * case["B"] * case["beams"] + 12 * case["B"] * case["K"], "flops": 3.0 * rows * case["V"]}
    if case["op"] == "reorder":
        each = 4 * case["history"] + 2 * case["D"] + 4 * case["layers"] * case["heads"] * case["length"] * case["width"]
        return {"bytes": case["B"] * case["beams"] * (2 * each + 4), "flops": 0.0}
    n = case["rows"] * case["cols"]
    return {"bytes": 4 * n * e[case["dtype"]], "flops": 2.0 * n}


def _levels(x, rows, cols):
    """In float64: the nearest e4m3 value, ties to even, of every value of blocks of rows x cols, times the block's power of two."""
    n, m = x.shape
    out = torch.empty((n, m), dtype=torch.float64, device=DEV)
    step = rows * max(1, (1 << 24) // (rows * m))
    for r in range(0, n, step):
        t = x[r:r + step].double()
        t = torch.nn.functional.pad(t, (0, -m % cols, 0, -t.shape[0] % rows))
        t = t.view(t.shape[0] // rows, rows, -1, cols)
        most = t.abs().amax(dim=(1, 3), keepdim=True)
        e = torch.floor(torch.log2(most / 448.0)).clamp(min=-127.0)
        e = torch.where(most > torch.exp2(e) * 448.0, e + 1, e)
        e = torch.where((e > -127) & (most <= torch.exp2(e - 1) * 448.0), e - 1, e)
        y = t / torch.exp2(e)
        # spacing of e4m3: an eighth of the value's power of two, 2^-9 below 2^-6
        gap = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
        out[r:r + step] = (torch.round(y / gap) * gap * torch.exp2(e)).reshape(t.shape[0] * rows, -1)[:min(step, n - r), :m]
    return out


def exact(case, seed):
    """The same outputs in float64, from the definitions."""
    s = prepare(case, seed)
    with torch.no_grad():
        if case["op"] == "logits":
            D, V = case["D"], case["V"]
            h = _levels(s.H, 1, 128)
            out = torch.empty((case["N"], V), dtype=torch.float64, device=DEV)
            for v in range(0, V, 32768):
                w8 = s.W8[v:v + 32768].to(torch.int32)
                power, part = (w8 >> 3) & 15, (w8 & 7).double()
                w = torch.where(power > 0, (part + 8) * torch.exp2(power.double() - 10), part * 2.0 ** -9) * (1.0 - 2.0 * (w8 >> 7))
                e = torch.stack([s.w_exp[b // 4, v:v + 32768, b % 4] for b in range(w.shape[1] // 128)], dim=1).double() - 127
                w = (w * torch.exp2(e).repeat_interleave(128, dim=1))[:, :D]
                out[:, v:v + 32768] = h.mm(w.t().contiguous()) + s.bias[v:v + 32768].double()
            return out
        if case["op"] == "train":
            N, D, V = case["N"], case["D"], case["V"]
            h, w = _levels(s.H, 1, 128), _levels(s.W, 128, 128)
            ht = _levels(s.H, 128, 1)
            out = torch.empty((N, V), dtype=torch.float64, device=DEV)
            dH = torch.zeros((N, D), dtype=torch.float64, device=DEV)
            dW = torch.empty((V, D), dtype=torch.float64, device=DEV)
            db = torch.empty((V,), dtype=torch.float64, device=DEV)
            for v in range(0, V, 16384):
                part, g = w[v:v + 16384], s.dY[:, v:v + 16384]
                out[:, v:v + 16384] = h.mm(part.t().contiguous()) + s.bias[v:v + 16384].double()
                dH += _levels(g, 1, 128).mm(part)
                dW[v:v + 16384] = _levels(g, 128, 1).t().contiguous().mm(ht)
                db[v:v + 16384] = g.double().sum(dim=0)
            return {"logits": out, "dH": dH, "dW": dW, "db": db}
        if case["op"] == "select":
            B, beams, V, K = case["B"], case["beams"], case["V"], case["K"]
            values = torch.empty((B, K), dtype=torch.float64, device=DEV)
            at = torch.empty((B, K), dtype=torch.int64, device=DEV)
            for b in range(B):
                score = torch.log_softmax(s.X[b * beams:(b + 1) * beams].double() / case["temperature"], dim=1) + s.scores[b].double()[:, None]
                if s.finished is not None:
                    ends = torch.full_like(score, -math.inf)
                    ends[:, s.end_id] = s.scores[b].double()
                    score = torch.where(s.finished[b][:, None], ends, score)
                least = score.reshape(-1).topk(K).values[-1]
                where = (score.reshape(-1) >= least).nonzero()[:, 0]
                v, i = torch.sort(score.reshape(-1)[where], descending=True, stable=True)
                values[b], at[b] = v[:K], where[i[:K]]
            return {"scores": values, "beams": (at // V).int(), "tokens": (at % V).int()}
        if case["op"] == "reorder":
            return [torch.stack([x[b].double()[s.parents[b].long()] for b in range(case["B"])]) if x.is_floating_point()
                    else torch.stack([x[b][s.parents[b].long()] for b in range(case["B"])]) for x in s.states]
        # products of 32 bits by halves of the multiplier, a block of counters at a time
        def times(a, m):
            low, high = a * (m & 0xffff), a * (m >> 16)
            total = low + ((high & 0xffff) << 16)
            return (high >> 16) + (total >> 32), total & 0xffffffff
        n = case["rows"] * case["cols"]
        least = round(case["p"] * 65536)
        kept = []
        for first in range(0, (n + 7) // 8, 1 << 20):
            at = torch.arange(first, min((n + 7) // 8, first + (1 << 20)), device=DEV)
            x = [at % (1 << 32), at // (1 << 32), torch.zeros_like(at) + s.offset % (1 << 32), torch.zeros_like(at) + s.offset // (1 << 32)]
            for r in range(10):
                key = [(s.seed % (1 << 32) + r * 0x9E3779B9) % (1 << 32), (s.seed // (1 << 32) + r * 0xBB67AE85) % (1 << 32)]
                (h0, l0), (h1, l1) = times(x[0], 0xD2511F53), times(x[2], 0xCD9E8D57)
                x = [h1 ^ x[1] ^ key[0], l1, h0 ^ x[3] ^ key[1], l0]
            kept.append(torch.stack([w // (1 << (16 * h)) % (1 << 16) >= least for w in x for h in (0, 1)], dim=1).reshape(-1))
        kept = torch.cat(kept)[:n].reshape(s.x.shape)
        factor = kept.double() * (65536 / (65536 - least) if least < 65536 else 0.0)
        return {"y": s.x.double() * factor, "dx": s.dy.double() * factor}
