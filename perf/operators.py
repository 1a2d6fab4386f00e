"""What the operators around the dense logits of the head are measured on: the 8-bit product that gives them, the
choice of the largest ones, and the distillation loss that trains a head on them, each with its plain form.

A teacher's head runs in 8-bit integers (rows of hidden states quantised by token, its matrix by vocabulary entry),
the largest K logits of every token and the logarithm of the normaliser are kept, and a student's head is trained on
those: loss[n] = sum_j p_nj (log p_nj - log q_n[id_nj]) with q_n = softmax((W h_n + bias) / T).

A case is an operator (`op`) and its sizes:

  quantize  N rows of D values to int8, one scale for each row
  int8      N rows of hidden states, quantised within the call, against V int8 rows of D: logits with a bias
  top       the K largest of V logits for each of N rows, in order, ties to the lowest index, and logsumexp(x / T)
  eval      loss of N rows of a student and the logarithm of its normaliser, nothing kept for a gradient
  train     loss and the gradients of hidden states, matrix and bias

Sizes are those of the repository's own workloads (`paper_2603_25011_amd/inputs.py`), tests and sweeps: hidden sizes
up to 1024 with 768 as the ordinary one, 30522 and 250002 vocabulary entries, batches from one query to many documents.
"""
import math

import torch

own = False
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _case(name, op, N, D, V, K=0, dtype="bf16", out="f32", temperature=1.0, keep=1.0, mass=1.0, excluded=0.0, pitch=0):
    return {"name": name, "op": op, "N": N, "D": D, "V": V, "K": K, "dtype": dtype, "out": out,
            "temperature": temperature, "keep": keep, "mass": mass, "excluded": excluded, "pitch": pitch}


def listed():
    return [
        # a multilingual matrix as it is loaded: the largest array that is ever quantised
        _case("quantize_matrix", "quantize", 250002, 1024, 0),
        # the last token of one query: the smallest product, latency counts
        _case("int8_one_token", "int8", 1, 768, 30522),
        # a handful of positions against the multilingual vocabulary: reading the matrix is what takes time
        _case("int8_few_tokens", "int8", 12, 1024, 250002, out="bf16"),
        # a batch of odd sizes kept in float32, as the tests have them
        _case("int8_ragged", "int8", 197, 312, 31091, dtype="f32"),
        # a teacher over a batch of documents
        _case("int8_documents", "int8", 8192, 768, 30522, out="bf16"),
        # one query's logits: the smallest choice, latency counts
        _case("top_one_token", "top", 1, 0, 30522, K=64),
        # a teacher's logits of a batch of documents, in the type that the 8-bit product stores
        _case("top_documents", "top", 4096, 0, 30522, K=64, dtype="bf16", temperature=2.0),
        # multilingual logits, rows of a wider array, a tenth of the vocabulary excluded with -inf
        _case("top_multilingual", "top", 256, 0, 250002, K=128, dtype="f32", excluded=0.1, pitch=250016),
        # held-out loss of a batch of passages, the teacher's logits renormalised over the ones that are kept
        _case("eval_passages", "eval", 2048, 768, 30522, K=64),
        # a small float32 model with odd sizes, some of its positions chosen
        _case("train_ragged_float32", "train", 2561, 312, 31091, K=33, dtype="f32", keep=0.5, mass=0.9, temperature=2.0),
        # a training step on documents, every third position is padding
        _case("train_documents", "train", 16384, 768, 30522, K=64, keep=0.66, temperature=2.0),
        # the multilingual student at its largest
        _case("train_multilingual", "train", 4096, 1024, 250002, K=64, mass=0.9),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: sizes over the logarithm of their range, most hidden sizes those of encoders, now and then any
    multiple of 8; no dearer than the largest case of its operator in `listed`."""
    while True:
        op = rng.choice(["quantize", "int8", "int8", "top", "top", "eval", "train", "train"])
        dtype = "f32" if rng.random() < 0.3 else "bf16"
        D = rng.choice([128, 256, 312, 384, 512, 768, 768, 1024, 1024]) if rng.random() < 0.7 else 8 * rng.randint(8, 128)
        V = _log_int(rng, 1000, 250002)
        K = _log_int(rng, 1, 128)
        temperature = rng.choice([1.0, 1.0, 2.0, 4.0])
        c = None
        if op == "quantize":
            c = _case("", op, _log_int(rng, 1, 250002), D, 0, dtype=dtype)
        elif op == "int8":
            N = _log_int(rng, 1, 16) if rng.random() < 0.4 else _log_int(rng, 16, 8192)
            c = _case("", op, N, D, V, dtype=dtype, out=rng.choice(["f32", "bf16"]))
            if N * D * V > 8192 * 768 * 30522:
                continue
        elif op == "top":
            N = _log_int(rng, 1, 4096)
            c = _case("", op, N, 0, V, K=K, dtype=dtype, temperature=temperature,
                      excluded=rng.choice([0.0, 0.0, 0.1, 0.5]), pitch=rng.choice([0, 0, V + rng.randint(1, 64)]))
            if N * V > 4096 * 30522:
                continue
        else:
            N = _log_int(rng, 1, 16384)
            c = _case("", op, N, D, V, K=K, dtype=dtype, temperature=temperature,
                      keep=rng.choice([1.0, 1.0, 0.66, 0.15]), mass=rng.choice([1.0, 0.9, 0.6]))
            limit = 2561 * 312 * 31091 if dtype == "f32" else 4096 * 1024 * 250002
            if N * D * V > limit or N * V > 4096 * 250002:
                continue
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


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    N, D, V, K = case["N"], case["D"], case["V"], case["K"]
    td = TYPES[case["dtype"]]
    s = State()
    s.case = dict(case)
    if case["op"] == "quantize":
        # a trained matrix: entries of one spread, rows of different norms
        s.X = _normal(gen, (N, D), 0.02, td).mul_(torch.rand((N, 1), device=DEV, generator=gen).add_(0.5).to(td))
        return s
    if case["op"] == "top":
        # logits as a head gives them: most near zero, a few of each row well above
        pitch = case["pitch"] or V
        s.X = _normal(gen, (N, pitch), 1.5, td)[:, :V]
        hot = torch.randint(0, V, (N, min(V, 32)), device=DEV, generator=gen)
        s.X.scatter_(1, hot, torch.rand(hot.shape, device=DEV, generator=gen).mul_(8.0).add_(2.0).to(td))
        if case["excluded"]:
            # whole vocabulary entries are excluded; at least K stay
            out = torch.rand(V, device=DEV, generator=gen) < case["excluded"]
            out[:min(V, 2 * K)] = False
            s.X.masked_fill_(out, -math.inf)
        s.values = torch.empty((N, K), dtype=torch.float32, device=DEV)
        s.ids = torch.empty((N, K), dtype=torch.int32, device=DEV)
        s.lse = torch.empty((N,), dtype=torch.float32, device=DEV)
        s.ws = torch.empty((8 << 20,), dtype=torch.uint8, device=DEV)
        return s
    s.H = _normal(gen, (N, D), 1.0, td)
    W = _normal(gen, (V, D), 0.05, torch.float32 if case["op"] == "int8" else td)
    s.bias = torch.randn((V,), device=DEV, generator=gen).mul_(0.1)
    if case["op"] == "int8":
        # the matrix as a loaded model keeps it: int8 rows padded with zeros to a multiple of 128, one scale each
        s.w_scale = W.abs().amax(dim=1) / 127.0
        s.W8 = torch.zeros((V, (D + 127) // 128 * 128), dtype=torch.int8, device=DEV)
        for v in range(0, V, 16384):
            s.W8[v:v + 16384, :D] = torch.round(W[v:v + 16384] / s.w_scale[v:v + 16384, None]).to(torch.int8)
        s.out = torch.empty((N, V), dtype=TYPES[case["out"]], device=DEV)
        s.ws = torch.empty((N * (s.W8.shape[1] + 4) + 256,), dtype=torch.uint8, device=DEV)
        return s
    s.W = W
    # a teacher's choice: distinct vocabulary entries, frequent (low) ones more often; its logits fall off from a peak
    k = min(K, V)
    ids = torch.rand((N, k), device=DEV, generator=gen).mul_(math.log(V - k + 1)).exp_().floor_().long() - 1
    ids = ids.clamp_(0, V - k).sort(dim=1).values + torch.arange(k, device=DEV)
    ids = ids.gather(1, torch.rand((N, k), device=DEV, generator=gen).argsort(dim=1))
    s.ids = ids.to(torch.int32)
    s.logits = torch.randn((N, k), device=DEV, generator=gen).mul_(2.5).sort(dim=1, descending=True).values.contiguous()
    # the normaliser over the teacher's whole vocabulary: the kept logits hold `mass` of it on average
    s.teacher_lse = None
    if case["mass"] < 1.0:
        share = torch.rand((N,), device=DEV, generator=gen).mul_(2.0 * (1.0 - case["mass"])).neg_().add_(1.0)
        s.teacher_lse = torch.logsumexp(s.logits / case["temperature"], dim=1) - share.log()
    s.mask = None
    if case["keep"] < 1.0:
        s.mask = torch.rand((N,), device=DEV, generator=gen) < case["keep"]
    if case["op"] == "train":
        s.dloss = torch.rand((N,), device=DEV, generator=gen).add_(0.5).div_(N)
        for t in (s.H, s.W, s.bias):
            t.requires_grad_(True)
    return s


def run(s):
    c = s.case
    if not own:
        with torch.no_grad():
            return {"quantize": _plain_quantize, "int8": _plain_int8, "top": _plain_top,
                    "eval": _plain_distill, "train": _plain_distill}[c["op"]](s, c)
    from paper_2603_25011_amd import binding as lsr
    from paper_2603_25011_amd import distill
    kind = {"f32": lsr.LSR_F32, "bf16": lsr.LSR_BF16}
    if c["op"] == "quantize":
        q, scale = distill.quantize_rows(s.X)
        return {"values": (q[:, :c["D"]] * scale[:, None]), "scale": scale}
    if c["op"] == "int8":
        lsr.lsr_int8_matmul(c["N"], c["V"], c["D"], kind[c["dtype"]], kind[c["out"]], s.H, c["D"], None,
                            s.W8, s.W8.shape[1], s.w_scale, s.bias, s.out, c["V"], s.ws)
        return s.out
    if c["op"] == "top":
        lsr.lsr_top_logits(c["N"], c["V"], c["K"], kind[c["dtype"]], c["temperature"], s.X, s.X.stride(0),
                           s.values, s.ids, s.lse, s.ws)
        return {"values": s.values, "ids": s.ids, "lse": s.lse}
    loss, lse = distill.lsr_distill(s.H, s.W, s.bias, s.ids, s.logits, s.teacher_lse, s.mask, c["temperature"])
    if c["op"] == "eval":
        return {"loss": loss, "lse": lse}
    dH, dW, db = torch.autograd.grad(loss, (s.H, s.W, s.bias), s.dloss)
    return {"loss": loss.detach(), "dH": dH, "dW": dW, "db": db}


def _plain_quantize(s, c):
    x = s.X.float()
    most = x.abs().amax(dim=1, keepdim=True)
    scale = most / 127.0
    return {"values": torch.round((x * 127.0) / most) * scale, "scale": scale[:, 0]}


def _plain_int8(s, c):
    x = s.H.float()
    most = x.abs().amax(dim=1, keepdim=True)
    q = torch.round((x * 127.0) / most)
    acc = q @ s.W8[:, :c["D"]].float().t()
    return (acc * ((most / 127.0) * s.w_scale) + s.bias).to(s.out.dtype)


def _plain_top(s, c):
    # one whole number for each logit that orders as the pair (value, lowest index first) does
    x = s.X.float()
    bits = x.view(torch.int32) if x.is_contiguous() else x.contiguous().view(torch.int32)
    order = torch.where(bits < 0, bits ^ 0x7fffffff, bits).long()
    key = order * (1 << 32) + ((1 << 32) - 1 - torch.arange(c["V"], device=DEV))
    best = key.topk(c["K"], dim=1).values
    ids = (1 << 32) - 1 - (best & 0xffffffff)
    x = x / c["temperature"]
    most = x.amax(dim=1, keepdim=True)
    lse = most[:, 0] + (x - most).exp().sum(dim=1).log()
    return {"values": s.X.gather(1, ids).float(), "ids": ids.to(torch.int32), "lse": lse}


def _plain_distill(s, c):
    t = c["temperature"]
    h, w = s.H.float(), s.W.float()
    z = (h @ w.t() + s.bias) / t
    most = z.amax(dim=1, keepdim=True)
    lse = most[:, 0] + (z - most).exp().sum(dim=1).log()
    x = s.logits / t
    if s.teacher_lse is None:
        top = x.amax(dim=1, keepdim=True)
        norm = top + (x - top).exp().sum(dim=1, keepdim=True).log()
    else:
        norm = s.teacher_lse[:, None]
    ids = s.ids.long()
    p = (x - norm).exp()
    loss = (p * ((x - norm) - (z.gather(1, ids) - lse[:, None]))).sum(dim=1)
    if s.mask is not None:
        loss, lse = loss * s.mask, lse * s.mask
    if c["op"] == "eval":
        return {"loss": loss, "lse": lse}
    g = s.dloss / t
    if s.mask is not None:
        g = g * s.mask
    d = (z - lse[:, None]).exp().mul_((g * p.sum(dim=1))[:, None])
    d.scatter_add_(1, ids, -p * g[:, None])
    return {"loss": loss, "dH": (d @ w).to(s.H.dtype), "dW": (d.t() @ h).to(s.W.dtype), "db": d.sum(dim=0)}


def work(case):
    """Every input read once, every output written once; two operations for each multiply-add of the product, and in
    training those of the two products that its gradients are.  Rows that the mask leaves out are not counted."""
    N, D, V, K = case["N"], case["D"], case["V"], case["K"]
    e = 4 if case["dtype"] == "f32" else 2
    o = 4 if case["out"] == "f32" else 2
    if case["op"] == "quantize":
        return {"bytes": N * D * (e + 1) + 4 * N, "flops": 3.0 * N * D}
    if case["op"] == "int8":
        return {"bytes": N * D * e + V * D + 8 * V + N * V * o, "flops": 2.0 * N * D * V}
    if case["op"] == "top":
        return {"bytes": N * V * e + 8 * N * K + 4 * N, "flops": 3.0 * N * V}
    rows = N * case["keep"]
    b = rows * D * e + V * D * e + 4 * V + 8 * rows * K + 8 * N
    if case["op"] == "train":
        return {"bytes": b + N * D * e + V * D * e + 4 * V + 4 * rows, "flops": 6.0 * rows * D * V}
    return {"bytes": b, "flops": 2.0 * rows * D * V}


def exact(case, seed):
    """The same outputs in float64, from the definitions, a block of rows at a time."""
    s = prepare(case, seed)
    op, t = case["op"], float(case["temperature"])
    with torch.no_grad():
        if op in ("quantize", "int8"):
            def levels(x):
                # 127 x first: what lies half-way between two levels then stays there, and goes to the even one
                most = x.double().abs().max(dim=1).values
                return torch.round(x.double() * 127 / most.unsqueeze(1)), most / 127
        if op == "quantize":
            parts = [levels(x) for x in s.X.split(16384)]
            return {"values": torch.cat([q * a.unsqueeze(1) for q, a in parts]), "scale": torch.cat([a for _, a in parts])}
        if op == "int8":
            out = torch.empty((case["N"], case["V"]), dtype=torch.float64, device=DEV)
            q, a = levels(s.H)
            for v in range(0, case["V"], 32768):
                w = s.W8[v:v + 32768, :case["D"]].double() * s.w_scale[v:v + 32768].double().unsqueeze(1)
                out[:, v:v + 32768] = (q * a.unsqueeze(1)).mm(w.t().contiguous()) + s.bias[v:v + 32768].double()
            return out
        if op == "top":
            values, ids, lse = [], [], []
            for x in s.X.split(256):
                v, i = torch.sort(x.double(), dim=1, descending=True, stable=True)
                values.append(v[:, :case["K"]])
                ids.append(i[:, :case["K"]].int())
                lse.append(torch.logsumexp(x.double() / t, dim=1))
            return {"values": torch.cat(values), "ids": torch.cat(ids), "lse": torch.cat(lse)}
        N, D, V = case["N"], case["D"], case["V"]
        W, bias = s.W.detach().double(), s.bias.detach().double()
        Wt = W.t().contiguous()
        train = op == "train"
        loss = torch.zeros(N, dtype=torch.float64, device=DEV)
        norms = torch.zeros(N, dtype=torch.float64, device=DEV)
        dH = torch.zeros((N, D), dtype=torch.float64, device=DEV) if train else None
        dW, db = (torch.zeros_like(W), torch.zeros_like(bias)) if train else (None, None)
        rows = torch.arange(N, device=DEV) if s.mask is None else s.mask.nonzero()[:, 0]
        for r in rows.split(1024):
            h = s.H.detach()[r].double()
            logq = torch.log_softmax(torch.addmm(bias, h, Wt) / t, dim=1)
            teacher = s.logits[r].double() / t
            if s.teacher_lse is None:
                logp = torch.log_softmax(teacher, dim=1)
            else:
                logp = teacher - s.teacher_lse[r].double().unsqueeze(1)
            at = s.ids[r].long()
            loss[r] = (logp.exp() * (logp - logq.gather(1, at))).sum(dim=1)
            norms[r] = ((h * W[at[:, 0]]).sum(dim=1) + bias[at[:, 0]]) / t - logq.gather(1, at[:, :1])[:, 0]
            if train:
                # softmax times the teacher's mass, less the teacher's probabilities
                g = logq.exp_().mul_(logp.exp().sum(dim=1, keepdim=True)).scatter_add_(1, at, -logp.exp())
                g.mul_((s.dloss[r].double() / t).unsqueeze(1))
                dH[r] = g.mm(W)
                dW.add_(g.t().contiguous().mm(h))
                db.add_(g.sum(dim=0))
    if train:
        return {"loss": loss, "dH": dH, "dW": dW, "db": db}
    return {"loss": loss, "lse": norms}
