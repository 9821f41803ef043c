"""Log probabilities of given tokens at a vocabulary head with entropy, rank and the most probable
alternatives (gk_vocab_logprob), their gradient (gk_vocab_logprob_grad), the norm over the
gradients of many tensors (gk_grad_norm) and clipping them, into the flat vector that the sparsifier
takes or into tensors of their own type (gk_grad_clip), as measured work.

`run` computes a case either with elementary torch operations in 32 bits (`own` false; sums over
many tensors in 64) or through the library's calls (`own` true); `exact` computes it from the
definitions in 64 bits."""
import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
IGNORED = -100


def listed():
    logprob = {"op": "logprob", "m": 1, "k": 0, "T": 1.0, "masked": 0.0, "left_out": 0.0}
    grad = {"op": "logprob_grad", "m": 1, "T": 1.0, "masked": 0.0, "left_out": 0.0, "entropy": True, "lse": False}
    return [
        # a server's answer: the sampled token, its rank, and the alternatives beside it
        {"name": "logprob_token", **logprob, "n": 1, "V": 50001, "k": 20, "type": "f32"},
        # a batch of tokens at a server, part of the vocabulary forbidden
        {"name": "logprob_batch", **logprob, "n": 64, "V": 32000, "k": 5, "T": 0.7, "masked": 0.4, "type": "bf16"},
        # a prompt's log probabilities with alternatives, an odd vocabulary; its last positions are padding
        {"name": "logprob_prompt", **logprob, "n": 2000, "V": 50001, "k": 20, "left_out": 0.1, "type": "f16"},
        # answers to choose from: several given tokens a row, the LSTM workload's vocabulary
        {"name": "logprob_choices", **logprob, "n": 700, "V": 10000, "m": 5, "k": 1, "type": "f32"},
        # a policy step scores its rollouts: log probability and entropy of every token
        {"name": "logprob_rollout", **logprob, "n": 4096, "V": 128000, "type": "bf16"},
        # a unit test's or a toy model's step: latency of the whole call
        {"name": "grad_tiny", **grad, "n": 33, "V": 1003, "left_out": 0.25, "type": "f16"},
        # the LSTM workload's head, fp32 logits, the log-sum-exp held near zero as well
        {"name": "grad_lstm_head", **grad, "n": 700, "V": 10000, "lse": True, "type": "f32"},
        # a policy step with an entropy bonus; prompts' positions carry no loss
        {"name": "grad_policy", **grad, "n": 4096, "V": 128000, "left_out": 0.3, "type": "bf16"},
        # the gradients of a convolutional network of 161 tensors
        {"name": "norm_161_tensors", "op": "norm", "tensors": 161, "total": 25557032, "type": "f32"},
        # a language model's gradients in 16 bits
        {"name": "norm_largest", "op": "norm", "tensors": 400, "total": 1000000007, "type": "bf16"},
        # a small network's gradients, clipped into the sparsifier's vector
        {"name": "clip_small", "op": "clip", "tensors": 65, "total": 269722, "type": "f32", "flat": True, "share": 0.3},
        # a language model's: matrices in 16 bits and vectors in fp32, clipped into the sparsifier's vector
        {"name": "clip_mixed", "op": "clip", "tensors": 290, "total": 400000003, "type": "mixed", "flat": True, "share": 0.5},
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over the logarithm, odd ones among them."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["logprob", "logprob", "logprob_grad", "norm", "clip"])
    if op in ("norm", "clip"):
        case = {"op": op, "tensors": _spread(rng, 1, 1000), "type": rng.choice(["f32", "bf16", "f16", "mixed"])}
        most = 1000000007 if op == "norm" else 400000003
        case["total"] = _spread(rng, max(5000, 20 * case["tensors"]), most // 2 if case["type"] == "f32" else most)
        if op == "clip":
            # into a vector of fp32, or into tensors of the gradients' own type; norms below the limit and above
            case["flat"] = case["type"] == "mixed" or rng.random() < 0.6
            case["share"] = rng.choice([0.1, 0.5, 0.9, 2.0])
        return case
    V = _spread(rng, 1000, 128000)
    case = {"op": op, "n": _spread(rng, 1, 4096), "V": V, "m": rng.choice([1, 1, 1, rng.randint(2, 8)]),
            "T": rng.choice([1.0, 0.7, 1.5]), "masked": rng.choice([0.0, 0.0, 0.4]), "left_out": rng.choice([0.0, 0.1, 0.3]),
            "type": rng.choice(["bf16", "bf16", "f16", "f32"])}
    if case["type"] == "f32":
        case["n"] = min(case["n"], 2048)
    if op == "logprob":
        case["k"] = rng.choice([0, _spread(rng, 1, 100)])
    else:
        case["entropy"], case["lse"] = rng.random() < 0.7, rng.random() < 0.3
    return case


def _sizes(case):
    """Sizes of the tensors, which follow from the case alone: two of five are vectors of 64 to 4096, the others
    share the rest unevenly; odd ones among them."""
    count, total = case["tensors"], case["total"]
    rng = random.Random(count * 1000003 + total)
    small = [i % 5 in (1, 3) and count > 2 for i in range(count)]
    most = max(1, total // (2 * count))
    sizes = [min(most, rng.choice([64, 128, 256, 512, 1000, 2048, 4096, 77])) if s else 0 for s in small]
    weight = [0.0 if s else math.exp(rng.uniform(-2.0, 2.0)) for s in small]
    rest, share = total - sum(sizes), sum(weight)
    sizes = [n or int(rest * w / share) for n, w in zip(sizes, weight)]
    sizes[0] += total - sum(sizes)
    return sizes


def prepare(case, seed):
    """Inputs on the GPU, and the buffers that a program keeps for the results."""
    dev = torch.device("cuda")
    if case["op"] in ("norm", "clip"):
        return _prepare_grads(case, seed, dev)
    n, V, m, dtype = case["n"], case["V"], case["m"], TYPES[case["type"]]
    gen = torch.Generator(device=dev).manual_seed(int(seed) * 1000003 + n * 31 + V)
    uniform = lambda *s: torch.rand(*s, generator=gen, device=dev)  # noqa: E731
    z = torch.randn(n, V, generator=gen, device=dev).mul_(2.5)
    z[torch.arange(n, device=dev), (uniform(n) * V).long().clamp_(max=V - 1)] += 12.0 * uniform(n)
    if case["masked"]:
        forbidden = uniform(1, V) < case["masked"]
        forbidden[:, :max(2, m)] = False
        z.masked_fill_(forbidden, -math.inf)
    z = z.to(dtype)
    rows = max(1, (1 << 28) // V)
    token, lse, entropy = [], [], []
    for a in range(0, n, rows):
        y = z[a:a + rows].float() / case["T"]
        # tokens sampled from the rows
        noise = -torch.log(-torch.log(uniform(*y.shape).clamp_(1e-20, 1 - 1e-7)))
        token.append((y + noise).argmax(1))
        y = y.double()
        lse.append(torch.logsumexp(y, 1))
        logp = y - lse[-1][:, None]
        entropy.append(-torch.where(logp > -math.inf, torch.exp(logp) * logp, 0.0).sum(1))
    token = torch.cat(token)[:, None]
    if m > 1:
        more = (uniform(n, m - 1) * V).long().clamp_(max=V - 1)
        if case["masked"]:
            more = more % max(2, m)      # allowed ones
        token = torch.cat([token, more], 1)
    if n > 1 and case["left_out"]:
        out = uniform(n) < case["left_out"]
        out[0] = False
        token = torch.where(out[:, None], torch.full_like(token, IGNORED), token)
    s = {"case": case, "logits": z, "token": token}
    empty = lambda *s, t=torch.float32: torch.empty(*s, dtype=t, device=dev)  # noqa: E731
    if case["op"] == "logprob":
        s["logp"], s["rank"] = empty(n, m), empty(n, t=torch.int32)
        s["entropy"], s["lse"] = empty(n), empty(n)
        if case["k"]:
            s["idx"], s["val"] = empty(n, case["k"], t=torch.int32), empty(n, case["k"])
        return s
    s["lse"], s["entropy"] = torch.cat(lse).float(), torch.cat(entropy).float()
    s["logp_grad"] = torch.randn(n, m, generator=gen, device=dev) / n      # advantages
    s["entropy_grad"] = torch.full((n,), -0.01 / n, device=dev) if case["entropy"] else None
    s["lse_grad"] = s["lse"] * (2e-4 / n) if case["lse"] else None
    s["dz"] = empty(n, V, t=dtype)
    return s


def _prepare_grads(case, seed, dev):
    sizes = _sizes(case)
    gen = torch.Generator(device=dev).manual_seed(int(seed) * 1000003 + case["total"])
    types = [TYPES["f32" if n <= 4096 else "bf16"] if case["type"] == "mixed" else TYPES[case["type"]] for n in sizes]
    # each layer's gradients have a scale of their own
    scale = torch.exp(torch.rand(len(sizes), generator=gen, device=dev) * 4.0 - 8.0)
    grads = [(torch.randn(n, generator=gen, device=dev) * scale[i]).to(t) for i, (n, t) in enumerate(zip(sizes, types))]
    s = {"case": case, "grads": grads, "ends": torch.tensor(sizes, device=dev).cumsum(0),
         "norm": torch.empty(1, device=dev)}
    if case["op"] == "norm":
        s["norms"] = torch.empty(len(sizes), device=dev)
    else:
        total = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
        s["limit"] = case["share"] * total
        s["out"] = torch.empty(case["total"], dtype=torch.float32 if case["flat"] else types[0], device=dev)
    if own:
        # a program whose gradients stay where they are makes this once
        from paper_1911_08772_b200 import binding as gk
        s["list"] = gk.GradList(grads, out=s.get("out"))
    return s


def run(s):
    case = s["case"]
    if own:
        return _own(s, case)
    if case["op"] in ("norm", "clip"):
        flat = torch.cat(s["grads"]).float()
        if case["op"] == "norm":
            sums = torch.cumsum(flat * flat, 0, dtype=torch.float64)[s["ends"] - 1]
            return {"norm": torch.sqrt(sums[-1:]).float(), "norms": torch.sqrt(torch.diff(sums, prepend=sums.new_zeros(1))).float()}
        norm = torch.sqrt((flat * flat).sum(dtype=torch.float64))
        return {"norm": norm.float()[None], "out": (flat * (s["limit"] / norm).clamp(max=1.0).float()).to(s["out"].dtype)}
    token = s["token"]
    keep = (token >= 0).any(1)
    at = token.clamp(min=0)
    z = s["logits"].float()
    y = z / case["T"]
    if case["op"] == "logprob":
        y = y - y.max(dim=1, keepdim=True).values
        e = torch.exp(y)
        total = e.sum(dim=1, keepdim=True)
        log_total = torch.log(total)
        entropy = log_total[:, 0] - torch.where(e > 0, e * y, 0.0).sum(dim=1) / total[:, 0]
        lse = z.max(dim=1).values / case["T"] + log_total[:, 0]
        first = torch.gather(z, 1, at[:, :1])
        place = torch.arange(case["V"], device=z.device)
        rank = ((z > first) | ((z == first) & (place < at[:, :1]))).sum(dim=1)
        out = {"logp": torch.where(token >= 0, torch.gather(y, 1, at) - log_total, 0.0), "rank": torch.where(keep, rank, -1).to(torch.int32),
               "entropy": torch.where(keep, entropy, 0.0), "lse": torch.where(keep, lse, 0.0)}
        if case["k"]:
            idx = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :case["k"]]
            out["idx"] = torch.where(keep[:, None], idx, -1).to(torch.int32)
            out["val"] = torch.where(keep[:, None], torch.gather(y, 1, idx) - log_total, 0.0)
        return out
    logp = y - s["lse"][:, None]
    p = torch.exp(logp)
    g = torch.where(token >= 0, s["logp_grad"], 0.0)
    factor = -g.sum(dim=1, keepdim=True)
    if case["lse"]:
        factor = factor + s["lse_grad"][:, None]
    if case["entropy"]:
        factor = factor - s["entropy_grad"][:, None] * (torch.where(p > 0, logp, 0.0) + s["entropy"][:, None])
    dz = (p * factor).scatter_add_(1, at, g) / case["T"]
    return {"dz": torch.where(keep[:, None], dz, 0.0).to(s["logits"].dtype)}


def _own(s, case):
    from paper_1911_08772_b200 import binding as gk
    if case["op"] == "norm":
        gk.gk_grad_norm(s["list"], s["norm"], norms_out=s["norms"])
        return {"norm": s["norm"], "norms": s["norms"]}
    if case["op"] == "clip":
        gk.gk_grad_clip(s["list"], s["limit"], norm_out=s["norm"])
        return {"norm": s["norm"], "out": s["out"]}
    if case["op"] == "logprob_grad":
        gk.gk_vocab_logprob_grad(s["logits"], s["token"], s["lse"], s["dz"], logp_grad=s["logp_grad"],
                                 entropy=s["entropy"] if case["entropy"] else None, entropy_grad=s["entropy_grad"],
                                 lse_grad=s["lse_grad"], temperature=case["T"])
        return {"dz": s["dz"]}
    names = ["logp", "rank", "entropy", "lse"] + (["idx", "val"] if case["k"] else [])
    gk.gk_vocab_logprob(s["logits"], s["token"], temperature=case["T"], **{name + "_out": s[name] for name in names})
    return {name: s[name] for name in names}


def work(case):
    if case["op"] in ("norm", "clip"):
        size = sum(n * (4 if case["type"] == "f32" or case["type"] == "mixed" and n <= 4096 else 2) for n in _sizes(case))
        if case["op"] == "norm":
            return {"bytes": size + 4 + 4 * case["tensors"], "flops": 2.0 * case["total"]}
        return {"bytes": size + (4 if case["flat"] else 2 if case["type"] != "f32" else 4) * case["total"] + 4, "flops": 3.0 * case["total"]}
    n, V, m = case["n"], case["V"], case["m"]
    counted = n * (1.0 - case["left_out"]) if n > 1 else 1.0
    size = 4 if case["type"] == "f32" else 2
    if case["op"] == "logprob":
        return {"bytes": int(counted * V * size) + n * (12 * m + 12 + 8 * case["k"]), "flops": 6.0 * counted * V}
    return {"bytes": int((counted + n) * V * size) + n * (12 * m + 16), "flops": 6.0 * counted * V}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("norm", "clip"):
        squares = torch.stack([g.double().pow(2).sum() for g in s["grads"]])
        norm = squares.sum().sqrt()
        if case["op"] == "norm":
            return {"norm": norm[None], "norms": squares.sqrt()}
        c = min(1.0, s["limit"] / float(norm))
        return {"norm": norm[None], "out": torch.cat([g.double() * c for g in s["grads"]])}
    n, V, T = case["n"], case["V"], case["T"]
    rows = max(1, min(n, (1 << 27) // V))      # pieces of about 1 GB in 64 bits
    parts = []
    for a in range(0, n, rows):
        at = slice(a, a + rows)
        token, z = s["token"][at], s["logits"][at].double() / T
        keep = (token >= 0).any(1)
        on = (token >= 0).double()
        there = token.clamp(min=0)
        if case["op"] == "logprob":
            lse = torch.logsumexp(z, 1)
            logp = z - lse[:, None]
            h = -torch.special.xlogy(torch.exp(logp), torch.exp(logp)).sum(1)
            part = {"logp": torch.gather(logp, 1, there).masked_fill(on == 0, 0.0),
                    "entropy": h.masked_fill(~keep, 0.0), "lse": lse.masked_fill(~keep, 0.0)}
            if case["k"]:
                part["val"] = torch.topk(logp, case["k"], dim=1).values.masked_fill(~keep[:, None], 0.0)
        else:
            # by the chain rule through the softmax, with the row's own log-sum-exp and entropy
            logp = torch.log_softmax(z, 1)
            p = torch.exp(logp)
            g = s["logp_grad"][at].double() * on
            dz = torch.zeros_like(p).scatter_add_(1, there, g) - p * g.sum(1, keepdim=True)
            if case["lse"]:
                dz += p * s["lse_grad"][at].double()[:, None]
            if case["entropy"]:
                surprise = -torch.special.xlogy(p, p)
                dz += s["entropy_grad"][at].double()[:, None] * (surprise - p * surprise.sum(1, keepdim=True))
            part = {"dz": (dz / T).masked_fill(~keep[:, None], 0.0)}
        parts.append(part)
    out = {name: torch.cat([p[name] for p in parts]) for name in parts[0]}
    if case["op"] == "logprob":
        out["rank"] = None
        if case["k"]:
            out["idx"] = None
    return out
