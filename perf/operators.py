"""Performance cases of the operators around the output head's logits.

* ``int8``     the int8 head: full-vocabulary logits of W_out's int8 rows (scales per token and per channel);
* ``lists``    the token drawn from a head's top-k lists (temperature, top-k, top-p, min-p, a given uniform number);
* ``rows``     the token drawn from full-vocabulary logit rows, by the same rule;
* ``loss``     distillation from a teacher's top-k lists: the loss of each token, forward only;
* ``grad``     its forward pass followed by its backward pass, as two calls;
* ``step``     loss and gradient in one call, as a training loop takes them.

``run`` makes the framework's calls where ``own`` is true and computes the
same in elementary torch operations where it is not.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one decoding step of a small head: launch latency and one small stream of int8 rows
        {"name": "int8-32k-d256-b1", "op": "int8", "V": 32768, "d": 256, "B": 1, "in": "f32", "out": "f32"},
        # one decoding step of a Qwen3-0.6B-shaped head: bound by the int8 rows
        {"name": "int8-qwen0.6b-b1", "op": "int8", "V": 151936, "d": 1024, "B": 1, "in": "bf16", "out": "f32"},
        # a small serving batch on a ragged vocabulary and a width that is no multiple of 16
        {"name": "int8-50257x1000-b5", "op": "int8", "V": 50257, "d": 1000, "B": 5, "in": "bf16", "out": "f32"},
        # a full serving batch, Llama-3.2-1B-shaped head
        {"name": "int8-llama1b-b64", "op": "int8", "V": 128256, "d": 2048, "B": 64, "in": "bf16", "out": "bf16"},
        # the logits of every token of a long prompt, or of a teacher's pass: bound by the matrix cores (the largest)
        {"name": "int8-llama1b-b2048", "op": "int8", "V": 128256, "d": 2048, "B": 2048, "in": "bf16", "out": "bf16"},
        # one decoding step after a top-50 head: pure latency (the smallest)
        {"name": "lists-k50-b1", "op": "lists", "k": 50, "B": 1, "pad": 0, "mixed": False},
        # a serving batch after the search with 64 forced tokens, each request with its own settings, padded tails
        {"name": "lists-k114-b256", "op": "lists", "k": 114, "B": 256, "pad": 9, "mixed": True},
        # one decoding step over the largest vocabulary's full row
        {"name": "rows-gemma270m-b1", "op": "rows", "V": 262144, "B": 1, "type": "f32", "mask": False, "mixed": False},
        # a serving batch of bf16 rows, each request with its own settings, some rows under a grammar's mask
        {"name": "rows-qwen0.6b-b64", "op": "rows", "V": 151936, "B": 64, "type": "bf16", "mask": True, "mixed": True},
        # scoring a few sequences' tokens against a teacher's lists
        {"name": "loss-32k-f32-n48", "op": "loss", "V": 32768, "N": 48, "k": 50, "type": "f32", "tau": 1.0},
        # forward and backward as an autograd loop calls them, fp32 logits of a ragged vocabulary
        {"name": "grad-50257-f32-n384", "op": "grad", "V": 50257, "N": 384, "k": 37, "type": "f32", "tau": 2.0},
        # a training step's head: loss and gradient of bf16 logits at once
        {"name": "step-llama1b-bf16-n2048", "op": "step", "V": 128256, "N": 2048, "k": 64, "type": "bf16", "tau": 2.0},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: vocabularies of 1 k to 262144 rows, widths of 64 to 2560 (odd ones too), 1 to 2048 tokens."""
    op = rng.choice(["int8", "int8", "lists", "rows", "rows", "loss", "grad", "step"])
    V = _log_int(rng, 1000, 262144)
    if op == "int8":
        d = 16 * _log_int(rng, 4, 160)
        if rng.random() < 0.2:
            d -= rng.randint(1, 15)
        B = _log_int(rng, 1, 1500)
        while B * V * d > 2048 * 128256 * 2048:
            B = (B + 1) // 2
        return {"op": op, "V": V, "d": d, "B": B, "in": rng.choice(["f32", "bf16"]), "out": rng.choice(["f32", "bf16"])}
    if op == "lists":
        k = _log_int(rng, 1, 1024)
        return {"op": op, "k": k, "B": _log_int(rng, 1, 512), "pad": rng.choice([0, 0, k // 5]), "mixed": rng.random() < 0.5}
    if op == "rows":
        return {"op": op, "V": V, "B": _log_int(rng, 1, 64), "type": rng.choice(["f32", "bf16"]),
                "mask": rng.random() < 0.3, "mixed": rng.random() < 0.5}
    N = max(1, min(_log_int(rng, 1, 2048), 2048 * 128256 // V // 2))
    return {"op": op, "V": V, "N": N, "k": min(_log_int(rng, 1, 256), V), "type": rng.choice(["f32", "bf16"]),
            "tau": rng.choice([1.0, 2.0, 4.0])}


def _settings(B, mixed, gen):
    """Sampling settings: one for all, or per request (among them greedy, unlimited and narrow ones)."""
    if not mixed:
        return {"temperature": 0.8, "top_k": 0, "top_p": 0.95, "min_p": 0.0}
    pick = lambda values, t: torch.tensor(values, dtype=t, device="cuda")[  # noqa: E731
        torch.randint(0, len(values), (B,), device="cuda", generator=gen)]
    return {"temperature": pick([0.0, 0.6, 0.8, 1.0, 1.0, 1.3], torch.float32),
            "top_k": pick([0, 0, 20, 50, 200], torch.int32),
            "top_p": pick([1.0, 0.9, 0.95, 0.98], torch.float32),
            "min_p": pick([0.0, 0.0, 0.02, 0.1], torch.float32)}


def _vocab_logits(n, V, gen):
    """Rows as a language model's head gives them: a broad bulk and a few dozen likely tokens."""
    z = 1.7 * torch.randn(n, V, device="cuda", generator=gen)
    likely = torch.randint(0, V, (n, min(V, 48)), device="cuda", generator=gen)
    z.scatter_add_(1, likely, 5.0 + 1.5 * torch.randn(likely.shape, device="cuda", generator=gen))
    return z


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1 + int(seed))
    s = {"case": case}
    if case["op"] == "int8":
        V, d, B = case["V"], case["d"], case["B"]
        W = torch.randn(V, d, device="cuda", generator=gen) / math.sqrt(d)
        W *= torch.exp(0.25 * torch.randn(V, 1, device="cuda", generator=gen))
        s["scale"] = W.abs().amax(1) / 127.0
        s["q"] = torch.round(W / s["scale"][:, None]).clamp_(-127, 127).to(torch.int8)
        pick = torch.randint(0, V, (B, 3), device="cuda", generator=gen)
        h = W[pick[:, 0]] + W[pick[:, 1]] + W[pick[:, 2]]
        h += math.sqrt(0.1 / d) * torch.randn(B, d, device="cuda", generator=gen)
        s["h"] = h.to(TYPES[case["in"]])
    elif case["op"] == "lists":
        k, B = case["k"], case["B"]
        lg = torch.sort(2.0 * torch.randn(B, 8 * k, device="cuda", generator=gen), descending=True)[0][:, :k] + 8.0
        ids = torch.argsort(torch.rand(B, 8 * k, device="cuda", generator=gen), dim=1)[:, :k].to(torch.int32)
        if case["pad"]:
            lg[:, k - case["pad"]:] = -math.inf
            ids[:, k - case["pad"]:] = -1
        s["ids"], s["logits"] = ids.contiguous(), lg.contiguous()
    elif case["op"] == "rows":
        z = _vocab_logits(case["B"], case["V"], gen)
        if case["mask"]:  # a grammar allows a tenth of the tokens in every fourth row, and none in the last
            out = torch.rand(case["B"], case["V"], device="cuda", generator=gen) < 0.9
            out[torch.arange(case["B"], device="cuda") % 4 != 0] = False
            if case["B"] > 1:
                out[-1] = True
            z.masked_fill_(out, -math.inf)
        s["logits"] = z.to(TYPES[case["type"]])
    else:
        N, V, k = case["N"], case["V"], case["k"]
        s["logits"] = torch.empty(N, V, dtype=TYPES[case["type"]], device="cuda")
        ids = torch.empty(N, k, dtype=torch.int64, device="cuda")
        for a in range(0, N, 256):  # the lists are those of a teacher that agrees with the student in part
            z = _vocab_logits(min(256, N - a), V, gen)
            s["logits"][a:a + 256] = z
            teacher = z + 1.0 * torch.randn(z.shape, device="cuda", generator=gen)
            top, at = torch.topk(teacher, k, dim=1)
            ids[a:a + 256] = at
            s.setdefault("tops", []).append(top)
        s["teacher"] = torch.cat(s.pop("tops")).contiguous()
        s["ids"] = ids.to(torch.int32)
        s["weight"] = 1.0 / N
    if case["op"] in ("lists", "rows"):
        s["u"] = torch.rand(case["B"], device="cuda", generator=gen)
        s["settings"] = _settings(case["B"], case["mixed"], gen)
    return s


def _quantized(h):
    # fp32 quotients; taken in 64 bits and rounded, which gives the same value whatever the divide in use
    scale = (h.double().abs().amax(1) / 127.0).float()
    x = (h.double() / torch.where(scale > 0, scale, 1.0).double()[:, None]).float()
    return torch.round(x).clamp(-127, 127), scale


def _int8_plain(q, scale, h, out):
    # integer sums reach 8192 * 127 * 127, above 2^24: in 64 bits
    x, xs = _quantized(h)
    z = (x.double() @ q.double().t()).float()
    return (z * scale * xs[:, None]).to(out)


def _column(v, like, t):
    return v.to(t)[:, None] if isinstance(v, torch.Tensor) else torch.full((like.shape[0], 1), v, dtype=t, device=like.device)


def _sample_plain(ids, logits, u, temperature, top_k, top_p, min_p):
    # sums and borders in 64 bits: a token is decided by comparing them
    z = logits.float()
    ok = z > -math.inf
    if ids is not None:
        ok &= ids >= 0
    z, at = torch.sort(torch.where(ok, z, -math.inf), dim=1, descending=True, stable=True)
    live = z > -math.inf
    count = live.sum(1, keepdim=True)
    t, p, m = (_column(v, z, torch.float64) for v in (temperature, top_p, min_p))
    top = _column(top_k, z, torch.int64)
    w = torch.exp((z.double() - z[:, :1].double()) / t)
    w = torch.where(live, torch.where(z == z[:, :1], 1.0, w), 0.0)
    sums = torch.cumsum(w, 1)
    limit = torch.where(top > 0, torch.minimum(top, count), count).clamp(min=1)
    kept = torch.where(p < 1, torch.minimum(limit, (sums < p * sums.gather(1, limit - 1)).sum(1, keepdim=True) + 1), limit)
    kept = torch.where(m > 0, torch.minimum(kept, ((w >= m) & live).sum(1, keepdim=True)), kept).clamp(min=1)
    kept = torch.where(t > 0, kept, 1)
    total = sums.gather(1, kept - 1)
    j = torch.where(t > 0, torch.minimum((sums <= u.double()[:, None] * total).sum(1, keepdim=True), kept - 1), 0)
    token = (at if ids is None else ids.gather(1, at)).gather(1, j).to(torch.int32)
    prob = torch.where(t > 0, w.gather(1, j) / total, 1.0).float()
    some = count > 0
    return (torch.where(some, token, -1)[:, 0], torch.where(some, prob, 0.0)[:, 0],
            torch.where(some, kept, 0)[:, 0].to(torch.int32))


def _teacher(ids, teacher, V, tau):
    ok = (ids >= 0) & (ids < V) & (teacher > -math.inf)
    t = torch.where(ok, teacher / tau, -math.inf)
    top = t.amax(1, keepdim=True)
    e = torch.where(ok, torch.exp(t - top), 0.0)
    total = e.sum(1, keepdim=True)
    return ok, e / total, t - top - torch.log(total)


def _distill_plain(logits, ids, teacher, tau, weight, backward):
    s = logits.float() / tau
    top = s.amax(1, keepdim=True)
    e = torch.exp(s - top)
    total = e.sum(1, keepdim=True)
    ok, p, logp = _teacher(ids, teacher, logits.shape[1], tau)
    at = torch.where(ok, ids, 0).long()
    logq = s.gather(1, at) - top - torch.log(total)
    loss = tau * tau * torch.where(ok & (p > 0), p * (logp - logq), 0.0).sum(1)
    if not backward:
        return loss
    some = ok.any(1, keepdim=True)
    loss = torch.where(some[:, 0], loss, 0.0)
    grad = (e / total).scatter_add_(1, at, torch.where(ok, -p, 0.0)).mul_(tau * weight)
    return loss, torch.where(some, grad, 0.0).to(logits.dtype)


def run(s):
    op, case = s["case"]["op"], s["case"]
    if own:
        from paper_2608_27460_amd import vie
        if op == "int8":
            return vie.Int8Head(s["q"], s["scale"])(s["h"], dtype=TYPES[case["out"]])
        if op == "lists":
            return vie.sample(s["ids"], s["logits"], s["u"], **s["settings"])
        if op == "rows":
            return vie.sample_rows(s["logits"], s["u"], **s["settings"])
        if op == "loss":
            return vie.distill(s["logits"], s["ids"], s["teacher"], case["tau"])[0]
        if op == "grad":
            loss, stats = vie.distill(s["logits"], s["ids"], s["teacher"], case["tau"])
            return loss, vie.distill_grad(s["logits"], s["ids"], s["teacher"], stats, case["tau"], weight=s["weight"])
        return vie.distill_step(s["logits"], s["ids"], s["teacher"], case["tau"], weight=s["weight"])
    if op == "int8":
        return _int8_plain(s["q"], s["scale"], s["h"], TYPES[case["out"]])
    if op in ("lists", "rows"):
        return _sample_plain(s.get("ids"), s["logits"], s["u"], **s["settings"])
    return _distill_plain(s["logits"], s["ids"], s["teacher"], case["tau"], s.get("weight"), op != "loss")


def work(case):
    size = lambda t: 4 if t == "f32" else 2  # noqa: E731
    if case["op"] == "int8":
        V, d, B = case["V"], case["d"], case["B"]
        return {"bytes": V * d + 4 * V + B * d * size(case["in"]) + B * V * size(case["out"]), "flops": 2 * B * V * d}
    if case["op"] in ("lists", "rows"):
        B = case["B"]
        values = case["k"] * 8 if case["op"] == "lists" else case["V"] * size(case["type"])
        n = case.get("k") or case["V"]
        # a weight: difference, quotient, exponential, sum
        return {"bytes": B * (values + 4 + 12 + (16 if case["mixed"] else 0)), "flops": 4 * B * n}
    N, V, k = case["N"], case["V"], case["k"]
    passes = {"loss": 1, "grad": 3, "step": 2}[case["op"]]  # reads, then reads and writes; at once: a read and a write
    return {"bytes": N * (V * size(case["type"]) * passes + 8 * k + 4), "flops": N * V * (4 if passes == 1 else 7)}


def _draw_exact(l, ids, u, t, k, p, m):
    """One row's token, probability and count from the definition (numpy, 64 bits)."""
    import numpy as np
    at = np.flatnonzero(l > -np.inf)
    if not at.size:
        return -1, 0.0, 0
    at = at[np.lexsort((ids[at], -l[at]))]
    if not t > 0:
        return int(ids[at[0]]), 1.0, 1
    if k > 0:
        at = at[:k]
    w = np.exp((l[at] - l[at[0]]) / t)
    part = np.add.accumulate(w)
    n = at.size
    if p < 1:
        n = min(n, int(np.searchsorted(part, p * part[-1], side="left")) + 1)
    if m > 0:
        n = min(n, int(np.count_nonzero(w >= m)))
    n = max(n, 1)
    j = min(int(np.searchsorted(part[:n], u * part[n - 1], side="right")), n - 1)
    return int(ids[at[j]]), w[j] / part[n - 1], n


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "int8":
        h = s["h"].double()
        xs = (torch.linalg.vector_norm(h, math.inf, dim=1) / 127.0).float().double()
        x = torch.clamp((h / xs.clamp(min=1e-45)[:, None]).float().round(), -127, 127).double()
        out = torch.empty(h.shape[0], case["V"], dtype=torch.float64, device="cuda")
        for a in range(0, case["V"], 16384):
            q = s["q"][a:a + 16384].double() * s["scale"][a:a + 16384].double()[:, None]
            out[:, a:a + 16384] = torch.mm(x, q.t().contiguous()) * xs[:, None]
        return out
    if case["op"] in ("lists", "rows"):
        import numpy as np
        B = case["B"]
        z = s["logits"].double().cpu().numpy()
        u = s["u"].double().cpu().numpy()
        of = {n: v.double().cpu().numpy() if isinstance(v, torch.Tensor) else np.full(B, float(v))
              for n, v in s["settings"].items()}
        every = np.arange(z.shape[1])
        got = []
        for b in range(B):
            ids = s["ids"][b].cpu().numpy() if "ids" in s else every
            row = np.where(ids >= 0, z[b], -np.inf)
            got.append(_draw_exact(row, ids, u[b], of["temperature"][b], int(of["top_k"][b]), of["top_p"][b], of["min_p"][b]))
        token, prob, kept = zip(*got)
        return (torch.tensor(token, dtype=torch.int32, device="cuda"),
                torch.tensor(prob, dtype=torch.float64, device="cuda"),
                torch.tensor(kept, dtype=torch.int32, device="cuda"))
    N, V, tau = case["N"], case["V"], case["tau"]
    loss = torch.empty(N, dtype=torch.float64, device="cuda")
    grad = None if case["op"] == "loss" else torch.empty(N, V, dtype=torch.float64, device="cuda")
    for a in range(0, N, 256):
        rows = slice(a, min(N, a + 256))
        x = s["logits"][rows].double() / tau
        lse = torch.logsumexp(x, 1, keepdim=True)
        p = torch.softmax(s["teacher"][rows].double() / tau, 1)
        at = s["ids"][rows].long()
        loss[rows] = tau * tau * (torch.special.entr(p).neg() - p * (x.gather(1, at) - lse)).sum(1)
        if grad is not None:
            g = torch.exp(x - lse)
            g.scatter_add_(1, at, -p)
            grad[rows] = g * (tau * s["weight"])
    return loss if grad is None else (loss, grad)
