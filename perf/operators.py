"""Operators on a matrix of logits: the log probabilities of given tokens with their entropy and
top alternatives, their gradient, and distillation from a teacher's top logits.

A case is one call on logits [rows][vocab] that are on the device already, as the tied LM head
leaves them. Where `own` is false the operators are computed from elementary torch operations
in 32 bits; where it is true by the library's kernels.
"""
import math

import torch

own = False

DEV = "cuda"
F32, F64 = torch.float32, torch.float64
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
QWEN, GEMMA = 151936, 262144  # the vocabularies of mebp_inputs.CONFIGS


def _case(op, rows, vocab, dtype, **kw):
    c = {"op": op, "rows": rows, "vocab": vocab, "dtype": dtype, "pad": 0, "masked": 0, "tau": 1.0}
    c.update(kw)
    return c


def listed():
    cases = {
        # one decoded token: its log probability and the usual number of alternatives; latency
        "logprobs-1x151936-f32-k20": _case("logprobs", 1, QWEN, "f32", top=20),
        # a phone-sized batch, scored for its perplexity and entropy: no alternatives asked for
        "logprobs-256x151936-f32": _case("logprobs", 256, QWEN, "f32", top=0),
        # a teacher's pass that records the alternatives a student is distilled from
        "logprobs-2048x262144-bf16-k64": _case("logprobs", 2048, GEMMA, "bf16", top=64),
        # odd sizes and pitch: every row starts at another alignment; columns masked off
        "logprobs-333x50257-f16-k5": _case("logprobs", 333, 50257, "f16", top=5, pad=6, masked=57, tau=0.7),
        # policy-gradient step: gradients of log probabilities and entropies
        "logprobs-grad-1024x151936-bf16": _case("logprobs_grad", 1024, QWEN, "bf16", grad="bf16"),
        # the same, small and ragged, in fp32
        "logprobs-grad-77x32001-f32": _case("logprobs_grad", 77, 32001, "f32", grad="f32", pad=2, tau=0.8),
        # validation loss of a distilled student: no gradient
        "distill-loss-512x151936-f16-k32": _case("distill", 512, QWEN, "f16", top=32, tau=2.0, alpha=0.7),
        # a few tokens, no gradient: latency
        "distill-loss-3x262144-bf16-k16": _case("distill", 3, GEMMA, "bf16", top=16, tau=1.0, alpha=1.0),
        # a small vocabulary and few tokens: the smallest training call
        "distill-grad-64x1000-f32-k8": _case("distill", 64, 1000, "f32", grad="f32", top=8, tau=2.0, alpha=0.5),
        # a phone-sized step as the LM head runs it: fp32 logits, bf16 gradients for the products
        "distill-grad-255x151936-f32-bf16-k32": _case("distill", 255, QWEN, "f32", grad="bf16", top=32, tau=1.0, alpha=1.0),
        # ordinary training batch in 16 bits, with the hard label mixed in
        "distill-grad-1024x151936-bf16-k16": _case("distill", 1024, QWEN, "bf16", grad="bf16", top=16, tau=2.0, alpha=0.7, masked=271),
        # the largest: a micro-batch over the large vocabulary, fp32 both ways
        "distill-grad-2048x262144-f32-k64": _case("distill", 2048, GEMMA, "f32", grad="f32", top=64, tau=1.5, alpha=0.9),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def draw(rng):
    def log(lo, hi):
        return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))

    op = rng.choice(["logprobs", "logprobs_grad", "distill", "distill_grad"])
    dtype = rng.choice(["f32", "f16", "bf16"])
    vocab = rng.choice([QWEN, GEMMA, log(1000, 262144), log(1000, 262144)])
    # rows: over the whole range, below the largest listed case's bytes
    rows = min(log(1, 4096), (1 << 29) // vocab)
    kw = {"pad": rng.choice([0, 0, 1, 8]), "masked": rng.choice([0, 0, rng.randrange(1, vocab // 8)]),
          "tau": round(rng.choice([1.0, rng.uniform(0.5, 3.0)]), 2)}
    if op == "logprobs":
        kw["top"] = rng.choice([0, 1, 5, 20, 64, rng.randrange(1, 65)])
    if op.startswith("distill"):
        kw["top"] = rng.choice([1, 8, 16, 32, 64, rng.randrange(1, 65)])
        kw["alpha"] = rng.choice([1.0, round(rng.uniform(0.1, 0.95), 2)])
    if op.endswith("_grad"):
        # gradients in fp16 only of fp16 logits
        kw["grad"] = rng.choice(["f32", "bf16", dtype])
    return _case("distill" if op == "distill_grad" else op, rows, vocab, dtype, **kw)


# ------------------------------------------------------------------------------- inputs
def _matrix(case, dtype):
    """[rows][vocab] of a buffer whose rows are `pad` elements further apart."""
    return torch.zeros((case["rows"], case["vocab"] + case["pad"]), dtype=TYPES[dtype], device=DEV)[:, :case["vocab"]]


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    n, v, k = case["rows"], case["vocab"], case.get("top", 0)

    def normal(*shape, std=1.0, mean=0.0):
        return torch.randn(shape, generator=gen, device=DEV) * std + mean

    def integers(hi, *shape):
        return torch.randint(0, hi, shape, generator=gen, device=DEV)

    # distinct likely tokens in each row, the target among them or not: the model is sure of some
    # rows and not of others
    real = v - case["masked"]
    kk = max(k, 8)
    step = 1 + integers(max(1, real // kk), n, 1)
    ids = (integers(real, n, 1) + step * torch.arange(kk, device=DEV)) % real
    z = _matrix(case, case["dtype"])
    for r in range(0, n, 256):
        part = normal(min(256, n - r), v, std=2.0)
        part.scatter_add_(1, ids[r:r + 256], normal(part.shape[0], kk, std=2.0, mean=7.0))
        if case["masked"]:
            part[:, real:] = -math.inf
        z[r:r + 256] = part
    pick = ids.gather(1, integers(kk, n, 1))[:, 0]
    targets = torch.where(integers(8, n) < 7, pick, integers(real, n)).to(torch.int32)
    st = {"op": case["op"], "z": z, "targets": targets, "tau": case["tau"], "k": k}
    if case["op"] == "logprobs":
        st["out"] = {"logp": torch.empty(n, device=DEV), "lse": torch.empty(n, device=DEV), "entropy": torch.empty(n, device=DEV)}
        if k:
            st["out"]["top_ids"] = torch.empty((n, k), dtype=torch.int32, device=DEV)
            st["out"]["top_logp"] = torch.empty((n, k), device=DEV)
    elif case["op"] == "logprobs_grad":
        # what the forward pass left, and the loss's gradients: a mean over the rows
        u = z.double() / case["tau"]
        lse = torch.logsumexp(u, 1)
        p = torch.exp(u - lse[:, None])
        st["lse"] = lse.float()
        st["entropy"] = (lse - (p * torch.where(p > 0, u, 0)).sum(1)).float()
        st["d_logp"] = normal(n, std=1.0 / n)
        st["d_entropy"] = normal(n, std=0.01 / n, mean=-0.01 / n)
        st["dz"] = _matrix(case, case["grad"])
    else:
        # the teacher's logits of its likely tokens; prompts shorter than the batch leave their
        # rows out of the mean
        st["ids"] = ids[:, :k].to(torch.int32).contiguous()
        st["teacher"] = normal(n, k, std=2.0, mean=9.0)
        st["weight"] = torch.rand(n, generator=gen, device=DEV).add_(0.5).div_(n)
        st["alpha"] = case["alpha"]
        st["loss"] = torch.empty(n, device=DEV)
        st["dz"] = _matrix(case, case["grad"]) if "grad" in case else None
    if case["op"] != "logprobs_grad":
        # scratch for the parts of rows, which a program keeps beside its outputs
        st["ws"] = torch.empty(4 << 20, dtype=torch.uint8, device=DEV)
    return st


# ------------------------------------------------------------------------------- plain form
def _top(x, k):
    """The k largest of each row of fp32 x, ties to the lowest index: of the value's bits in their
    order above the column's complement, no two of which are alike."""
    bits = (x + 0.0).view(torch.int32)
    bits = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).to(torch.int64)
    key = (bits << 32) | (x.shape[1] - 1 - torch.arange(x.shape[1], device=x.device))
    return x.shape[1] - 1 - (torch.topk(key, k, dim=1)[0] & 0xFFFFFFFF)


def _softmax(x):
    """max, sum of exponentials and the exponentials of each row."""
    m = x.amax(1, keepdim=True)
    e = torch.exp(x - m)
    return m, e.sum(1, keepdim=True), e


def _plain_logprobs(st):
    x = st["z"].float() / st["tau"]
    m, s, e = _softmax(x)
    log_s = torch.log(s)
    t = st["targets"].long()[:, None]
    out = {"logp": ((x.gather(1, t) - m) - log_s)[:, 0], "lse": (m + log_s)[:, 0],
           "entropy": (log_s - (e * torch.where(e > 0, x - m, 0.0)).sum(1, keepdim=True) / s)[:, 0]}
    if st["k"]:
        ids = _top(st["z"].float(), st["k"])
        out["top_ids"] = ids.to(torch.int32)
        out["top_logp"] = (x.gather(1, ids) - m) - log_s
    return out


def _plain_logprobs_grad(st):
    logp = st["z"].float() / st["tau"] - st["lse"][:, None]
    p = torch.exp(logp)
    g = -st["d_logp"][:, None] * p
    g -= st["d_entropy"][:, None] * p * (torch.where(p > 0, logp, 0.0) + st["entropy"][:, None])
    t = st["targets"].long()[:, None]
    g.scatter_add_(1, t, st["d_logp"][:, None])
    return (g / st["tau"]).to(st["dz"].dtype)


def _plain_distill(st):
    z, tau, alpha, w = st["z"].float(), st["tau"], st["alpha"], st["weight"][:, None]
    ids, t = st["ids"].long(), st["targets"].long()[:, None]
    _, sp, p = _softmax(st["teacher"] / tau)
    p = p / sp
    m, s, e = _softmax(z / tau)
    kl = (p * (torch.log(p) - ((z.gather(1, ids) / tau - m) - torch.log(s)))).sum(1, keepdim=True)
    loss = alpha * tau * tau * kl
    if alpha < 1:
        m1, s1, e1 = _softmax(z)
        loss = loss + (1 - alpha) * (torch.log(s1) - (z.gather(1, t) - m1))
    out = {"loss": (w * loss)[:, 0]}
    if st["dz"] is not None:
        g = (alpha * tau) * (e / s)
        g.scatter_add_(1, ids, (-alpha * tau) * p)
        if alpha < 1:
            g += (1 - alpha) * (e1 / s1)
            g.scatter_add_(1, t, torch.full_like(w, alpha - 1))
        out["dz"] = (w * g).to(st["dz"].dtype)
    return out


# ------------------------------------------------------------------------------- the calls
def run(st):
    if own:
        from paper_2510_03425_amd import device as D
        if st["op"] == "logprobs":
            D.token_logprobs(st["z"], st["targets"], st["k"], st["tau"], st["out"], st["ws"])
            return st["out"]
        if st["op"] == "logprobs_grad":
            D.token_logprobs_backward(st["z"], st["targets"], st["lse"], st["entropy"], st["d_logp"], st["d_entropy"],
                                      st["dz"], st["tau"])
            return st["dz"]
        D.distill_topk(st["z"], st["ids"], st["teacher"], st["loss"], st["dz"], st["tau"], st["alpha"],
                       st["targets"] if st["alpha"] < 1 else None, st["weight"], st["ws"])
        return {"loss": st["loss"]} if st["dz"] is None else {"loss": st["loss"], "dz": st["dz"]}
    if st["op"] == "logprobs":
        return _plain_logprobs(st)
    return _plain_logprobs_grad(st) if st["op"] == "logprobs_grad" else _plain_distill(st)


def work(case):
    n, v, k = case["rows"], case["vocab"], case.get("top", 0)
    size = {"f32": 4, "f16": 2, "bf16": 2}
    nbytes = n * v * size[case["dtype"]] + (n * v * size[case["grad"]] if "grad" in case else 0)
    # per row: target and the row's numbers; K ids and values
    nbytes += n * {"logprobs": 16 + 8 * k, "logprobs_grad": 20, "distill": 12 + 8 * k}[case["op"]]
    # per logit: scale and subtract, exp, add; entropy or gradient on top
    return {"bytes": nbytes, "flops": n * v * {"logprobs": 6, "logprobs_grad": 6, "distill": 8 if "grad" in case else 4}[case["op"]]}


# ------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    parts = []
    for r in range(0, case["rows"], 64):
        rows = slice(r, r + 64)
        z = st["z"][rows].double()
        at = torch.arange(z.shape[0], device=DEV)
        t = st["targets"][rows].long()
        logq = torch.log_softmax(z / case["tau"], 1)
        q = logq.exp()
        if case["op"] == "logprobs":
            o = {"logp": logq[at, t], "lse": torch.logsumexp(z / case["tau"], 1), "entropy": torch.special.entr(q).sum(1)}
            if st["k"]:
                order = torch.sort(z, dim=1, descending=True, stable=True)[1][:, :st["k"]]
                o["top_ids"] = order.to(torch.int32)
                o["top_logp"] = torch.gather(logq, 1, order)
        elif case["op"] == "logprobs_grad":
            # d logp_t / dz = (1[t] - q) / tau, dH / dz = -q (log q + H) / tau
            ent = torch.special.entr(q)
            one = torch.zeros_like(q)
            one[at, t] = 1.0
            o = {"dz": ((one - q) * st["d_logp"][rows].double()[:, None]
                        + (ent - q * ent.sum(1, keepdim=True)) * st["d_entropy"][rows].double()[:, None]) / case["tau"]}
        else:
            ids, w = st["ids"][rows].long(), st["weight"][rows].double()
            logp = torch.log_softmax(st["teacher"][rows].double() / case["tau"], 1)
            kl = (logp.exp() * (logp - logq.gather(1, ids))).sum(1)
            log1 = torch.log_softmax(z, 1)
            ce = -log1[at, t]
            a, tau = case["alpha"], case["tau"]
            o = {"loss": w * (a * tau * tau * kl + (1 - a) * ce)}
            if "grad" in case:
                p = torch.zeros_like(q).scatter_(1, ids, logp.exp())
                hard = log1.exp()
                hard[at, t] -= 1.0
                o["dz"] = w[:, None] * (a * tau * (q - p) + (1 - a) * hard)
        parts.append(o)
    whole = {k: torch.cat([p[k] for p in parts]) for k in parts[0]}
    return whole["dz"] if case["op"] == "logprobs_grad" else whole
