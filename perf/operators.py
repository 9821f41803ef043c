"""The vocabulary head's operators as measured work: the loss through the head with its gradient
(gk_vocab_loss), distillation from a teacher's top logits through the head (gk_vocab_distill), and
the top logits of rows (gk_vocab_topk).

`run` computes a case either with elementary torch operations in 32 bits (`own` false) or through
the library's calls (`own` true); `exact` computes it from the definitions in 64 bits."""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
IGNORED = -100


def listed():
    loss = {"op": "loss", "grad": True, "left_out": 0.0}
    score = {"op": "loss", "grad": False, "left_out": 0.0}
    distill = {"op": "distill", "grad": True}
    return [
        # a unit test's or a toy model's step: latency of the whole call
        {"name": "loss_tiny", **loss, "n": 33, "D": 256, "V": 1003, "type": "f16", "left_out": 0.25},
        # the head of the LSTM workload: 20 sequences of 35 words, rows of 3000 bytes
        {"name": "loss_lstm_head", **loss, "n": 700, "D": 1500, "V": 10000, "type": "bf16"},
        # a fine-tuning step: prompts' positions carry no loss, an odd vocabulary
        {"name": "loss_train", **loss, "n": 4096, "D": 2048, "V": 50001, "type": "bf16", "left_out": 0.3},
        # a pre-training step's micro-batch on a wide head
        {"name": "loss_largest", **loss, "n": 8192, "D": 4096, "V": 128000, "type": "bf16"},
        # evaluation: log-probabilities of a prompt
        {"name": "score_prompt", **score, "n": 2000, "D": 2048, "V": 32000, "type": "f16"},
        # evaluation while decoding: one token
        {"name": "score_token", **score, "n": 1, "D": 4096, "V": 128000, "type": "bf16"},
        # a small student
        {"name": "distill_small", **distill, "n": 48, "D": 512, "V": 8000, "K": 16, "T": 2.0, "mass": False, "type": "f16"},
        # a student's step against a teacher's stored messages, with the teacher's full mass
        {"name": "distill_train", **distill, "n": 2048, "D": 2048, "V": 32000, "K": 64, "T": 1.0, "mass": True, "type": "bf16"},
        # the same on a wide head
        {"name": "distill_large", **distill, "n": 4096, "D": 4096, "V": 128000, "K": 100, "T": 1.5, "mass": True, "type": "bf16"},
        # a server's answer with the top alternatives of one token
        {"name": "topk_token", "op": "topk", "n": 1, "V": 50001, "K": 20, "T": 1.0, "type": "f32", "masked": 0.0},
        # a batch of tokens with part of the vocabulary forbidden
        {"name": "topk_batch", "op": "topk", "n": 500, "V": 32000, "K": 64, "T": 1.0, "type": "bf16", "masked": 0.4},
        # a teacher writes messages for a stretch of corpus
        {"name": "topk_corpus", "op": "topk", "n": 4096, "V": 128000, "K": 100, "T": 1.5, "type": "bf16", "masked": 0.0},
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over the logarithm, odd ones among them."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["loss", "loss", "score", "distill", "distill", "topk"])
    if op == "topk":
        V = _spread(rng, 1000, 128000)
        return {"op": "topk", "n": _spread(rng, 1, 4096), "V": V, "K": _spread(rng, 1, 128), "T": rng.choice([1.0, 1.5, 2.0]),
                "type": rng.choice(["bf16", "f16", "f32"]), "masked": rng.choice([0.0, 0.0, 0.4])}
    D = _spread(rng, 128, 4096)
    if rng.random() < 0.7:
        D = max(128, D // 64 * 64)
    case = {"n": _spread(rng, 1, 8192 if op != "distill" else 4096), "D": D, "V": _spread(rng, 1000, 128000), "type": rng.choice(["bf16", "bf16", "f16"])}
    if op == "distill":
        return {"op": "distill", "grad": True, **case, "K": _spread(rng, 1, 128), "T": rng.choice([1.0, 1.5, 2.0]), "mass": rng.random() < 0.5}
    return {"op": "loss", "grad": op == "loss", "left_out": rng.choice([0.0, 0.1, 0.3]), **case}


def prepare(case, seed):
    """Inputs on the GPU, and the buffers that a program keeps for the results."""
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(int(seed) * 1000003 + case["n"] * 31 + case["V"])
    normal = lambda *s: torch.randn(*s, generator=gen, device=dev)  # noqa: E731
    uniform = lambda *s: torch.rand(*s, generator=gen, device=dev)  # noqa: E731
    n, V, dtype = case["n"], case["V"], TYPES[case["type"]]
    s = {"case": case}
    if case["op"] == "topk":
        K = case["K"]
        z = normal(n, V) * 2.5
        z[torch.arange(n, device=dev), (uniform(n) * V).long().clamp_(max=V - 1)] += 8.0
        if case["masked"]:
            z.masked_fill_(uniform(1, V) < case["masked"], -math.inf)
        s["logits"] = z.to(dtype)
        s["idx"] = torch.empty(n, K, dtype=torch.int32, device=dev)
        s["val"] = torch.empty(n, K, dtype=torch.float32, device=dev)
        s["lse"] = torch.empty(n, dtype=torch.float32, device=dev)
        return s
    D = case["D"]
    w = normal(V, D).mul_(2.0 / math.sqrt(D)).to(dtype)
    # words as frequent as words are: the r-th about 1 / r
    word = (torch.exp(uniform(n) * math.log(V)) - 1.0).long().clamp_(0, V - 1)
    # a state that has learned something: between 0 and 12 nats for its word over the rest
    s["h"] = (normal(n, D) + w[word].float() * (uniform(n, 1) * 3.0)).to(dtype)
    s["w"] = w
    s["loss"] = torch.empty(n, dtype=torch.float32, device=dev)
    s["lse"] = torch.empty(n, dtype=torch.float32, device=dev)
    if case["grad"]:
        s["dh"] = torch.empty(n, D, dtype=dtype, device=dev)
        s["dw"] = torch.empty(V, D, dtype=dtype, device=dev)
    if case["op"] == "loss":
        out = uniform(n) < case["left_out"]
        if n > 1:
            out[0] = False
        s["target"] = torch.where(out, torch.full_like(word, IGNORED), word) if n > 1 else word
        counted = (s["target"] >= 0).float()
        s["row_grad"] = torch.ones(n, device=dev) / counted.sum()
        return s
    K = case["K"]
    # one pair in each of K stretches of the vocabulary, the word's stretch taken by the word
    at = ((torch.arange(K, device=dev) + uniform(n, K)) * (V / K)).long().clamp_(max=V - 1)
    at.scatter_(1, (word * K // V).clamp_(max=K - 1)[:, None], word[:, None])
    t = normal(n, K) * 2.0 + 4.0
    t.scatter_(1, (word * K // V).clamp_(max=K - 1)[:, None], 8.0)
    s["t_idx"], s["t_val"] = at.to(torch.int32), t
    s["t_lse"] = torch.logsumexp(t / case["T"], 1) + 0.2 * uniform(n) if case["mass"] else None
    s["row_grad"] = torch.full((n,), 1.0 / n, device=dev)
    return s


def run(s):
    case = s["case"]
    if own:
        return _own(s, case)
    if case["op"] == "topk":
        z = s["logits"].float()
        order = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :case["K"]]
        idx = torch.sort(order, dim=1).values
        zt = z / case["T"]
        top = zt.max(dim=1, keepdim=True).values
        lse = top[:, 0] + torch.log(torch.exp(zt - top).sum(dim=1))
        return {"idx": idx.to(torch.int32), "val": torch.gather(z, 1, idx), "lse": lse}
    h, w = s["h"].float(), s["w"].float()
    T = case.get("T", 1.0)
    z = (h @ w.t()) / T
    top = z.max(dim=1, keepdim=True).values
    e = torch.exp(z - top)
    total = e.sum(dim=1, keepdim=True)
    lse = top + torch.log(total)
    if case["op"] == "loss":
        keep = (s["target"] >= 0)[:, None]
        at = s["target"].clamp(min=0)[:, None]
        q = torch.ones_like(lse)
        loss = lse - torch.gather(z, 1, at)
    else:
        keep = torch.ones_like(lse, dtype=torch.bool)
        at = s["t_idx"].long()
        t = s["t_val"] / T
        if s["t_lse"] is None:
            m = t.max(dim=1, keepdim=True).values
            logq = t - m - torch.log(torch.exp(t - m).sum(dim=1, keepdim=True))
        else:
            logq = t - s["t_lse"][:, None]
        q = torch.exp(logq)
        loss = (q * (logq - torch.gather(z, 1, at) + lse)).sum(dim=1, keepdim=True)
    out = {"loss": torch.where(keep, loss, 0.0)[:, 0], "lse": torch.where(keep, lse, 0.0)[:, 0]}
    if case["grad"]:
        dz = e * (q.sum(dim=1, keepdim=True) / total)
        dz = dz.scatter_add_(1, at, -q)
        dz = torch.where(keep, dz * (s["row_grad"][:, None] / T), 0.0)
        out["dh"] = (dz @ w).to(s["h"].dtype)
        out["dw"] = (dz.t() @ h).to(s["w"].dtype)
    return out


def _own(s, case):
    from paper_1911_08772_b200 import binding as gk
    if case["op"] == "topk":
        gk.gk_vocab_topk(s["logits"], case["K"], s["idx"], s["val"], lse_out=s["lse"], temperature=case["T"])
        return {"idx": s["idx"], "val": s["val"], "lse": s["lse"]}
    grads = {"row_grad": s["row_grad"], "dh": s["dh"], "dw": s["dw"]} if case["grad"] else {}
    if case["op"] == "loss":
        gk.gk_vocab_loss(s["h"], s["w"], s["target"], s["loss"], s["lse"], ignore_index=IGNORED, **grads)
    else:
        gk.gk_vocab_distill(s["h"], s["w"], s["t_idx"], s["t_val"], s["loss"], s["lse"], t_lse=s["t_lse"],
                            temperature=case["T"], **grads)
    out = {"loss": s["loss"], "lse": s["lse"]}
    if case["grad"]:
        out["dh"], out["dw"] = s["dh"], s["dw"]
    return out


def work(case):
    n, V = case["n"], case["V"]
    if case["op"] == "topk":
        size = 4 if case["type"] == "f32" else 2
        return {"bytes": n * V * size + n * case["K"] * 8 + n * 4, "flops": 0}
    D = case["D"]
    counted = n * (1.0 - case.get("left_out", 0.0)) if n > 1 else 1.0
    target = 8 * n if case["op"] == "loss" else 8 * n * case["K"] + (4 * n if case["mass"] else 0)
    passes = 2 if case["grad"] else 1     # h and w are read, dh and dw are written
    return {"bytes": passes * 2 * (n * D + V * D) + target + 8 * n + (4 * n if case["grad"] else 0),
            "flops": (3 if case["grad"] else 1) * 2.0 * counted * D * V}


def exact(case, seed):
    s = prepare(case, seed)
    n, V = case["n"], case["V"]
    T = case.get("T", 1.0)
    rows = max(1, min(n, (1 << 27) // V))      # pieces of about 1 GB in 64 bits
    if case["op"] == "topk":
        lse = torch.cat([torch.logsumexp(s["logits"][a:a + rows].double() / T, dim=1) for a in range(0, n, rows)])
        return {"idx": None, "val": None, "lse": lse}
    w = s["w"].double()
    loss = torch.zeros(n, dtype=torch.float64, device=w.device)
    lse = torch.zeros_like(loss)
    dh = torch.zeros(n, case["D"], dtype=torch.float64, device=w.device)
    dw = torch.zeros_like(w)
    for a in range(0, n, rows):
        h = s["h"][a:a + rows].double()
        logp = h @ w.t()
        logp /= T
        part = torch.logsumexp(logp, dim=1)
        logp -= part[:, None]
        if case["op"] == "loss":
            target = s["target"][a:a + rows]
            on = (target >= 0).double()
            at = target.clamp(min=0)[:, None]
            q = on[:, None]
            loss[a:a + rows] = -on * torch.gather(logp, 1, at)[:, 0]
            lse[a:a + rows] = on * part
        else:
            at = s["t_idx"][a:a + rows].long()
            t = s["t_val"][a:a + rows].double() / T
            logq = t - (torch.logsumexp(t, 1) if s["t_lse"] is None else s["t_lse"][a:a + rows].double())[:, None]
            q = torch.exp(logq)
            loss[a:a + rows] = (q * (logq - torch.gather(logp, 1, at))).sum(1)
            lse[a:a + rows] = part
        if case["grad"]:
            dz = logp.exp_()
            dz *= q.sum(1, keepdim=True)
            dz.scatter_add_(1, at, -q)
            dz *= s["row_grad"][a:a + rows, None].double() / T
            dh[a:a + rows] = dz @ w
            dw += dz.t() @ h
    out = {"loss": loss, "lse": lse}
    if case["grad"]:
        out["dh"], out["dw"] = dh, dw
    return out
