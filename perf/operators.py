"""Workloads of the fine-tuning operators: what is timed, on which inputs, and what the results have to be.

A fitted completion ranks the columns of a row: softmax(w_i H) is the model's distribution over the n columns (the
next word of a bigram table, the partner of a cell).  The operators fine-tune such factors on preferences or rewards:

  token_logprobs    log-probability of one column per row of a logits matrix
  factor_logprobs   the same from the factors, without a logits matrix
  preference_loss   paired log ratios (chosen against rejected sequences) and the gradient of the logits
  policy_loss       clipped ratio loss with a KL term and the gradient of the logits
  clip_grad_norm    global norm of a list of gradients, and the gradients scaled to a largest norm

A target below zero leaves its row out (a prompt token, padding): log-probability 0 and a zero gradient row.
"""
import math
import random

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}
COLUMNS = 139255          # columns of the connectome-shaped workload
MOST_LOGITS = 4096 * COLUMNS


# ---------------------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # the log-probability of one sampled column while a sequence is being produced: one row, latency counts
        {"name": "token_logprobs_one_row", "op": "token_logprobs", "tokens": 1, "vocab": COLUMNS, "stride": COLUMNS,
         "dtype": "bf16", "ignored": 0.0, "banned": 0.0, "temperature": 1.0},
        # old log-probabilities of a batch of rollouts: a padded vocabulary, prompts left out, a sampling temperature
        {"name": "token_logprobs_rollouts", "op": "token_logprobs", "tokens": 4001, "vocab": 50001, "stride": 50048,
         "dtype": "fp16", "ignored": 0.2, "banned": 0.05, "temperature": 0.8},
        # reference log-probabilities of a few rows of the connectome-shaped factors (r = 64): reads H once
        {"name": "factor_logprobs_few_rows", "op": "factor_logprobs", "tokens": 7, "columns": COLUMNS, "rank": 64,
         "dtype": "bf16", "ignored": 0.0, "temperature": 1.0},
        # reference log-probabilities of a whole block of 4096 rows of the same factors
        {"name": "factor_logprobs_block", "op": "factor_logprobs", "tokens": 4096, "columns": COLUMNS, "rank": 64,
         "dtype": "bf16", "ignored": 0.0, "temperature": 1.0},
        # the 32-bit factors of the planted 20,000-column workload (r = 32), an odd number of rows
        {"name": "factor_logprobs_fp32", "op": "factor_logprobs", "tokens": 2047, "columns": 20000, "rank": 32,
         "dtype": "fp32", "ignored": 0.1, "temperature": 0.7},
        # a few short sequences over a small vocabulary: launches and host work count
        {"name": "preference_small", "op": "preference_loss", "pairs": 4, "tokens": 160, "ragged": True,
         "vocab": 4096, "stride": 4096, "dtype": "fp32", "ignored": 0.25, "banned": 0.0, "temperature": 1.0,
         "smoothing": 0.0, "average": False, "grad": True},
        # a present against an absent link of each of 1024 cells: sequences of one token, odd unpadded rows
        {"name": "preference_links", "op": "preference_loss", "pairs": 1024, "tokens": 2048, "ragged": False,
         "vocab": COLUMNS, "stride": COLUMNS, "dtype": "bf16", "ignored": 0.0, "banned": 0.0, "temperature": 1.0,
         "smoothing": 0.1, "average": False, "grad": True},
        # ragged sequences of some hundred tokens, some of them empty, averaged over their length
        {"name": "preference_sequences", "op": "preference_loss", "pairs": 16, "tokens": 8191, "ragged": True,
         "vocab": 32768, "stride": 32768, "dtype": "bf16", "ignored": 0.3, "banned": 0.02, "temperature": 1.0,
         "smoothing": 0.0, "average": True, "grad": True},
        # one small rollout batch, mean over sequences of each one's mean
        {"name": "policy_small", "op": "policy_loss", "sequences": 5, "tokens": 255, "vocab": 4096, "stride": 4096,
         "dtype": "fp32", "ignored": 0.2, "banned": 0.0, "temperature": 1.0, "kl": 0.05, "grad": True},
        # a large rollout batch over every column of the connectome-shaped workload, mean over tokens
        {"name": "policy_rollouts", "op": "policy_loss", "sequences": 0, "tokens": 4096, "vocab": COLUMNS,
         "stride": COLUMNS + 9, "dtype": "bf16", "ignored": 0.1, "banned": 0.0, "temperature": 1.0, "kl": 0.02,
         "grad": True},
        # the gradients of the two connectome-shaped factors
        {"name": "clip_grad_norm_factors", "op": "clip_grad_norm", "tensors": 2, "elements": 2 * COLUMNS * 64,
         "even": True, "dtype": "fp32", "clipped": True},
        # the gradients of a model of many tensors, from a few elements to tens of millions, in two types
        {"name": "clip_grad_norm_many", "op": "clip_grad_norm", "tensors": 300, "elements": 400_000_000,
         "even": False, "dtype": "mixed", "clipped": True},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["token_logprobs", "factor_logprobs", "preference_loss", "policy_loss", "clip_grad_norm"])
    dtype = rng.choice(["fp32", "bf16", "bf16", "fp16"])
    temperature = rng.choice([1.0, 1.0, 0.7, 1.3])
    ignored = rng.choice([0.0, 0.1, 0.3, 0.6])
    if op == "clip_grad_norm":
        tensors = _log_int(rng, 1, 500)
        return {"op": op, "tensors": tensors, "elements": max(tensors, _log_int(rng, 1000, 400_000_000)),
                "even": rng.random() < 0.3, "dtype": rng.choice(["fp32", "bf16", "fp16", "mixed"]),
                "clipped": rng.random() < 0.8}
    if op == "factor_logprobs":
        rank, dtype = rng.randint(1, 256), rng.choice(["fp32", "bf16", "bf16", "fp16"])
        columns = _log_int(rng, 2, COLUMNS)
        # an fp32 product is counted as the plain one that it is: the largest listed case bounds rows x columns x rank
        most = max(1, min(4096, MOST_LOGITS * 64 // (columns * rank * (4 if dtype == "fp32" else 1))))
        return {"op": op, "tokens": _log_int(rng, 1, most), "columns": columns, "rank": rank, "dtype": dtype,
                "ignored": ignored, "temperature": temperature}
    vocab = _log_int(rng, 2, COLUMNS)
    tokens = _log_int(rng, 1, max(1, min(8192, MOST_LOGITS * 2 // (vocab * BYTES[dtype]))))
    case = {"op": op, "tokens": tokens, "vocab": vocab, "stride": vocab + rng.choice([0, 0, 0, 1, 8, -vocab % 64]),
            "dtype": dtype, "ignored": ignored, "banned": rng.choice([0.0, 0.0, 0.1]) if vocab >= 16 else 0.0,
            "temperature": temperature}
    if op == "preference_loss":
        ragged = rng.random() < 0.7
        pairs = _log_int(rng, 1, max(1, tokens // 2))
        if not ragged:
            case["tokens"] = tokens = 2 * pairs * max(1, tokens // (2 * pairs))
        case.update(pairs=pairs, ragged=ragged, smoothing=rng.choice([0.0, 0.0, 0.1]), average=rng.random() < 0.4,
                    grad=rng.random() < 0.8)
    if op == "policy_loss":
        case.update(sequences=rng.choice([0, _log_int(rng, 1, tokens)]), kl=rng.choice([0.0, 0.02, 0.1]),
                    grad=rng.random() < 0.8)
    return case


# --------------------------------------------------------------------------------------------------------- inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _offsets(sequences, tokens, ragged, g):
    """Borders of the sequences in the packed rows: equal lengths, or random cuts (some sequences come out empty)."""
    if not ragged:
        each = tokens // sequences
        return torch.arange(sequences + 1, device="cuda", dtype=torch.int64) * each
    cuts = torch.randint(0, tokens + 1, (sequences - 1,), device="cuda", generator=g).sort().values
    ends = torch.tensor([0, tokens], device="cuda", dtype=torch.int64)
    return torch.cat([ends[:1], cuts, ends[1:]])


def _targets(case, columns, g):
    T = case["tokens"]
    y = torch.randint(0, columns, (T,), device="cuda", generator=g)
    return y, _mask(case, y, g)


def _mask(case, y, g):
    """`y` with the case's share of rows left out: a fixed number of them, at random places."""
    out = int(case["ignored"] * case["tokens"])
    y = y.clone()
    if out:
        y[torch.randperm(case["tokens"], device="cuda", generator=g)[:out]] = -100
    return y


def _logits(case, g):
    """Logits of a trained model: broad, the target's raised, some columns banned (-inf) for all rows."""
    T, V = case["tokens"], case["vocab"]
    dtype = DTYPES[case["dtype"]]
    x = torch.empty((T, case["stride"]), device="cuda", dtype=dtype)
    for at in range(0, T, 512):
        rows = x[at:at + 512]
        rows.copy_(2.5 * torch.randn(rows.shape, device="cuda", generator=g, dtype=torch.float32))
    x = x[:, :V]
    all_targets, targets = _targets(case, V, g)
    if case["banned"]:
        x[:, torch.randperm(V, device="cuda", generator=g)[:int(case["banned"] * V)]] = float("-inf")
    rows = torch.arange(T, device="cuda")
    x[rows, all_targets] = (6.0 + 2.0 * torch.randn(T, device="cuda", generator=g)).to(dtype)
    return x, targets, all_targets


def _true_logprobs(x, y, temperature):
    got = torch.empty(x.shape[0], device="cuda", dtype=torch.float32)
    for at in range(0, x.shape[0], 512):
        z = x[at:at + 512].float() / temperature
        got[at:at + 512] = z.gather(1, y[at:at + 512, None])[:, 0] - z.logsumexp(1)
    return got


def _left_out(v, y):
    """Values of rows that are left out were never computed: nothing may depend on them."""
    return torch.where(y >= 0, v, float("nan"))


def _sizes(case):
    """Elements of each gradient: equal, or spread over the logarithm with the case's sum."""
    n, total = case["tensors"], case["elements"]
    if case["even"]:
        weights = [1.0] * n
    else:
        r = random.Random(1000003 * n + total)
        weights = [math.exp(r.uniform(0.0, math.log(1e5))) for _ in range(n)]
    left, scale = total - n, sum(weights)
    sizes = [1 + int(left * w / scale) for w in weights]
    sizes[sizes.index(max(sizes))] += total - sum(sizes)
    kinds = ["fp32", "bf16"] if case["dtype"] == "mixed" else [case["dtype"]]
    return [(s, kinds[k % len(kinds)]) for k, s in enumerate(sizes)]


def prepare(case, seed):
    g = _generator(seed)
    op = case["op"]
    if op == "clip_grad_norm":
        sizes = _sizes(case)
        grads, views, flat = [], [], {}
        for kind in sorted({k for _, k in sizes}):
            flat[kind] = torch.empty(sum((s + 15) // 16 * 16 for s, k in sizes if k == kind), device="cuda",
                                     dtype=DTYPES[kind])
            flat[kind].zero_()
        at = dict.fromkeys(flat, 0)
        for s, kind in sizes:
            x = torch.randn(s, device="cuda", generator=g, dtype=DTYPES[kind])
            grads.append(x.mul_(0.01))
            views.append(flat[kind][at[kind]:at[kind] + s])
            at[kind] += (s + 15) // 16 * 16
        norm = 0.01 * math.sqrt(case["elements"])
        return {"op": op, "grads": grads, "out": views, "flat": [flat[k] for k in sorted(flat)],
                "max_norm": (0.1 if case["clipped"] else 10.0) * norm}
    if op == "factor_logprobs":
        T, n, r = case["tokens"], case["columns"], case["rank"]
        scale = math.sqrt(2.5 / math.sqrt(r))     # logits of deviation 2.5, as below
        A = (scale * torch.randn((T, r), device="cuda", generator=g)).to(DTYPES[case["dtype"]])
        B = (scale * torch.randn((n, r), device="cuda", generator=g)).to(DTYPES[case["dtype"]])
        _, y = _targets(case, n, g)
        return {"op": op, "A": A, "B": B, "targets": y, "temperature": case["temperature"]}
    x, y, every = _logits(case, g)
    s = {"op": op, "logits": x, "targets": y, "temperature": case["temperature"]}
    T = case["tokens"]
    if op == "preference_loss":
        true = _true_logprobs(x, every, case["temperature"])
        s["offsets"] = _offsets(2 * case["pairs"], T, case["ragged"], g)
        s["reference"] = _left_out(true + 0.3 * torch.randn(T, device="cuda", generator=g), y)
        s.update(beta=0.1, smoothing=case["smoothing"], average=case["average"], grad=case["grad"])
    if op == "policy_loss":
        true = _true_logprobs(x, every, case["temperature"])
        s["offsets"] = _offsets(case["sequences"], T, True, g) if case["sequences"] else None
        s["old"] = _left_out(true + 0.15 * torch.randn(T, device="cuda", generator=g), y)
        s["reference"] = _left_out(true + 0.3 * torch.randn(T, device="cuda", generator=g), y)
        s["advantages"] = _left_out(torch.randn(T, device="cuda", generator=g) + 0.25, y)
        s.update(clip=(0.2, 0.28), kl=case["kl"], grad=case["grad"])
    return s


# ----------------------------------------------------------------------------------------------------------- runs

def _log_softmax(x, temperature):
    """(z - max, sum of exp(z - max)) of z = x / temperature in 32 bits."""
    z = x.float() / temperature
    z = z - z.max(1, keepdim=True).values
    return z, z.exp().sum(1, keepdim=True)


def _chosen(z, total, y):
    live = y >= 0
    lp = z.gather(1, y.clamp(min=0)[:, None])[:, 0] - total[:, 0].log()
    return torch.where(live, lp, 0.0), live


def _logits_gradient(z, total, y, live, coef, s):
    """coef_t (1[v = y_t] - p_tv) / temperature in the logits' type, zero rows where a row is left out."""
    coef = torch.where(live, coef, 0.0) / s["temperature"]
    d = z.exp() * (-coef[:, None] / total)
    d.scatter_add_(1, y.clamp(min=0)[:, None], coef[:, None])
    return torch.where(live[:, None], d, 0.0).to(s["logits"].dtype)


def _of_sequence(offsets, tokens):
    """The sequence of each packed row."""
    return torch.searchsorted(offsets, torch.arange(tokens, device=offsets.device), right=True) - 1


def _plain_preference(s):
    x, y = s["logits"], s["targets"]
    z, total = _log_softmax(x, s["temperature"])
    lp, live = _chosen(z, total, y)
    count = s["offsets"].numel() - 1
    seq = _of_sequence(s["offsets"], y.numel())
    ratio = torch.zeros(count, device=x.device).index_add_(0, seq, torch.where(live, lp - s["reference"], 0.0))
    share = torch.ones(count, device=x.device)
    if s["average"]:
        share = 1.0 / torch.zeros(count, device=x.device).index_add_(0, seq, live.float()).clamp(min=1.0)
        ratio = ratio * share
    margin = s["beta"] * (ratio[0::2] - ratio[1::2])
    down, up = torch.log1p(torch.exp(-margin.abs())) + (-margin).clamp(min=0), \
        torch.log1p(torch.exp(-margin.abs())) + margin.clamp(min=0)
    e = s["smoothing"]
    loss = ((1 - e) * down + e * up).mean()
    out = {"loss": loss, "logps": lp, "ratios": ratio, "margins": margin}
    if s["grad"]:
        slope = s["beta"] * (e - 1.0 / (1.0 + margin.exp())) / margin.numel()
        coef = (torch.stack([slope, -slope], 1).reshape(-1) * share)[seq]
        out["grad"] = _logits_gradient(z, total, y, live, coef, s)
    return out


def _plain_policy(s):
    x, y = s["logits"], s["targets"]
    z, total = _log_softmax(x, s["temperature"])
    lp, live = _chosen(z, total, y)
    if s["offsets"] is None:
        w = live.float() / live.float().sum().clamp(min=1.0)
    else:
        count = s["offsets"].numel() - 1
        seq = _of_sequence(s["offsets"], y.numel())
        per = torch.zeros(count, device=x.device).index_add_(0, seq, live.float()).clamp(min=1.0)
        w = torch.where(live, 1.0 / (count * per)[seq], 0.0)
    zero = torch.zeros((), device=x.device)
    lo, hi = 1.0 - s["clip"][0], 1.0 + s["clip"][1]
    ratio = torch.where(live, lp - s["old"], zero).exp()
    adv = torch.where(live, s["advantages"], zero)
    gap = torch.where(live, s["reference"] - lp, zero)
    cut = ((adv > 0) & (ratio > hi)) | ((adv < 0) & (ratio < lo))
    term = -torch.minimum(ratio * adv, ratio.clamp(lo, hi) * adv)
    kl = gap.exp() - gap - 1.0
    out = {"loss": (w * (term + s["kl"] * kl)).sum(), "logps": lp, "kl": (w * kl).sum(), "clipped": (w * cut).sum()}
    if s["grad"]:
        coef = w * (torch.where(cut, zero, -ratio * adv) + s["kl"] * (1.0 - gap.exp()))
        out["grad"] = _logits_gradient(z, total, y, live, coef, s)
    return out


def run(state):
    s = state
    op = s["op"]
    if own:
        from paper_2608_21607_gb300 import tuning

        if op == "token_logprobs":
            return tuning.token_logprobs(s["logits"], s["targets"], temperature=s["temperature"])
        if op == "factor_logprobs":
            return tuning.factor_logprobs(s["A"], s["B"], s["targets"], temperature=s["temperature"])
        if op == "preference_loss":
            r = tuning.preference_loss(s["logits"], s["targets"], s["offsets"], s["reference"], beta=s["beta"],
                                       label_smoothing=s["smoothing"], average=s["average"],
                                       temperature=s["temperature"], grad=s["grad"])
            out = {"loss": r.loss, "logps": r.logps, "ratios": r.ratios, "margins": r.margins}
        elif op == "policy_loss":
            r = tuning.policy_loss(s["logits"], s["targets"], s["old"], s["reference"], s["advantages"],
                                   offsets=s["offsets"], clip_low=s["clip"][0], clip_high=s["clip"][1],
                                   kl_coef=s["kl"], temperature=s["temperature"], grad=s["grad"])
            out = {"loss": r.loss, "logps": r.logps, "kl": r.kl, "clipped": r.clipped}
        else:
            return [tuning.clip_grad_norm(s["grads"], s["max_norm"], out=s["out"])] + s["flat"]
        if s["grad"]:
            out["grad"] = r.grad
        return out
    if op == "token_logprobs":
        z, total = _log_softmax(s["logits"], s["temperature"])
        return _chosen(z, total, s["targets"])[0]
    if op == "factor_logprobs":
        z, total = _log_softmax(s["A"].float() @ s["B"].float().t(), s["temperature"])
        return _chosen(z, total, s["targets"])[0]
    if op == "preference_loss":
        return _plain_preference(s)
    if op == "policy_loss":
        return _plain_policy(s)
    norm = torch.stack([g.float().square().sum() for g in s["grads"]]).sum().sqrt()
    scale = (s["max_norm"] / norm).clamp(max=1.0)
    for g, o in zip(s["grads"], s["out"]):
        o.copy_(g.float() * scale)
    return [norm] + s["flat"]


# --------------------------------------------------------------------------------------------- definitions in 64 bits

def _exact_logprobs(z, y):
    """Log-probabilities by the library's log-softmax in 64 bits, with a graph for the gradient."""
    rows = torch.nonzero(y >= 0)[:, 0]
    lp = torch.zeros(y.numel(), device=z.device, dtype=torch.float64)
    if rows.numel() == 0:
        return lp + 0.0 * z.nan_to_num(0.0, 0.0, 0.0).sum()
    chosen = torch.log_softmax(z[rows], 1)[torch.arange(rows.numel(), device=z.device), y[rows]]
    return lp.index_put((rows,), chosen)


def exact(case, seed):
    s = prepare(case, seed)
    op = s["op"]
    if op == "clip_grad_norm":
        norm = math.sqrt(math.fsum(float((g.double() ** 2).sum()) for g in s["grads"]))
        scale = min(1.0, s["max_norm"] / norm)
        flat = []
        for buffer in s["flat"]:
            whole = torch.zeros(buffer.numel(), device="cuda", dtype=torch.float64)
            for g, o in zip(s["grads"], s["out"]):
                if o.dtype == buffer.dtype:
                    at = o.storage_offset()
                    whole[at:at + o.numel()] = scale * g.double()
            flat.append(whole)
        return [torch.tensor(norm, dtype=torch.float64)] + flat
    y = s["targets"]
    if op in ("token_logprobs", "factor_logprobs"):
        got = []
        for at in range(0, y.numel(), 256):
            rows = slice(at, at + 256)
            x = s["logits"][rows].double() if op == "token_logprobs" else s["A"][rows].double() @ s["B"].double().t()
            got.append(_exact_logprobs(x / s["temperature"], y[rows]))
        return torch.cat(got)
    x = s["logits"].double().requires_grad_(s["grad"])
    lp = _exact_logprobs(x / s["temperature"], y)
    live = y >= 0
    ref = s["reference"].double()
    borders = s["offsets"].tolist() if s["offsets"] is not None else None
    if op == "preference_loss":
        per = []
        for a, b in zip(borders, borders[1:]):
            here = live[a:b]
            total = (lp[a:b] - ref[a:b])[here].sum()
            per.append(total / max(1, int(here.sum())) if s["average"] else total)
        ratios = torch.stack(per)
        margins = s["beta"] * (ratios[0::2] - ratios[1::2])
        logsig = torch.nn.functional.logsigmoid
        loss = -((1 - s["smoothing"]) * logsig(margins) + s["smoothing"] * logsig(-margins)).mean()
        out = {"loss": loss, "logps": lp, "ratios": ratios, "margins": margins}
    else:
        old, adv = s["old"].double(), s["advantages"].double()
        lo, hi = 1.0 - s["clip"][0], 1.0 + s["clip"][1]
        ratio = torch.exp(lp - old)
        kl = torch.exp(ref - lp) - (ref - lp) - 1.0
        surrogate = torch.minimum(ratio * adv, torch.clamp(ratio, lo, hi) * adv)
        cut = (((adv > 0) & (ratio > hi)) | ((adv < 0) & (ratio < lo))).double()

        def mean(v):
            if borders is None:
                return v[live].sum() / max(1, int(live.sum()))
            per = [v[a:b][live[a:b]].sum() / max(1, int(live[a:b].sum())) for a, b in zip(borders, borders[1:])]
            return torch.stack(per).mean()

        loss = mean(s["kl"] * kl - surrogate)
        out = {"loss": loss, "logps": lp, "kl": mean(kl), "clipped": mean(cut)}
    if s["grad"]:
        out["grad"] = torch.autograd.grad(loss, x, allow_unused=True)[0]
        if out["grad"] is None:
            out["grad"] = torch.zeros_like(x)
    return {k: v.detach() for k, v in out.items()}


# ----------------------------------------------------------------------------------------------------------- work

def work(case):
    """Bytes read once and written once, and the operations of the sums: rows that are left out are not read."""
    op = case["op"]
    if op == "clip_grad_norm":
        sizes = _sizes(case)
        moved = sum(2 * n * BYTES[k] for n, k in sizes)
        return {"bytes": moved + 4, "flops": 3 * case["elements"]}
    T = case["tokens"]
    live = T - int(case["ignored"] * T)
    if op == "factor_logprobs":
        n, r, b = case["columns"], case["rank"], BYTES[case["dtype"]]
        return {"bytes": (live + n) * r * b + 12 * T, "flops": 2 * live * n * r + 4 * live * n}
    V, b = case["vocab"], BYTES[case["dtype"]]
    if op == "token_logprobs":
        return {"bytes": live * V * b + 12 * T, "flops": 4 * live * V}
    side = {"preference_loss": 16 * T, "policy_loss": 24 * T}[op]
    written = T * V * b if case["grad"] else 0
    return {"bytes": live * V * b + written + side, "flops": (6 if case["grad"] else 4) * live * V}
