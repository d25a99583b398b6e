"""Workloads of the two ends of a fine-tuning loop: what is timed, on which inputs, and what the results have to be.

A fitted completion is a chain over its columns: row i scores what follows i (the next word of a bigram table).  The
losses of the framework train it on sequences; these operators make the sequences and take the training step:

  beam_select     the best continuations of each group's beams: log-softmax of every beam's row, added to the beam's
                  score, the largest of beams x columns
  beam_reorder    the beams' states (histories, caches) put in the order of the selected parents, in place
  orthogonalize   an update replaced by its orthogonal factor, by Newton-Schulz products
  muon_step       momentum, the orthogonalised update and weight decay, applied to the weights in place
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16, "int64": torch.int64,
          "int32": torch.int32}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2, "int64": 8, "int32": 4}
COLUMNS = 139255                    # columns of the connectome-shaped workload
MOST_LOGITS = 512 * COLUMNS
MOST_STATE = 2 ** 30                # bytes of all states
MOST_PRODUCT = 4096 ** 3            # smaller side squared times the larger one
MOST_MATRIX = 256 * COLUMNS
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
EPS = 1e-7


# ---------------------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # the next column of one chain with four beams over every column of the connectome-shaped workload: latency
        {"name": "beam_select_one_group", "op": "beam_select", "groups": 1, "beams": 4, "width": 4, "vocab": COLUMNS,
         "stride": COLUMNS, "dtype": "bf16", "finished": 0.0, "unused": 0.0, "banned": 0.0, "temperature": 1.0},
        # a served batch over a padded vocabulary, some beams finished, some columns banned, a temperature
        {"name": "beam_select_batch", "op": "beam_select", "groups": 64, "beams": 8, "width": 8, "vocab": 50001,
         "stride": 50048, "dtype": "fp16", "finished": 0.2, "unused": 0.0, "banned": 0.05, "temperature": 0.8},
        # twice as many candidates as beams, as a caller keeps that sets finished ones aside; 32-bit logits
        {"name": "beam_select_wide", "op": "beam_select", "groups": 255, "beams": 5, "width": 10, "vocab": 32768,
         "stride": 32768, "dtype": "fp32", "finished": 0.0, "unused": 0.1, "banned": 0.0, "temperature": 1.0},
        # candidate sequences for a block of preferences over every column, odd unpadded rows
        {"name": "beam_select_columns", "op": "beam_select", "groups": 128, "beams": 4, "width": 4, "vocab": COLUMNS,
         "stride": COLUMNS, "dtype": "bf16", "finished": 0.1, "unused": 0.0, "banned": 0.0, "temperature": 1.0},
        # the histories of one group's four beams, the used part of longer rows: latency
        {"name": "beam_reorder_histories", "op": "beam_reorder", "groups": 1, "beams": 4, "outer": 1, "tensors": 1,
         "inner": 201, "stride": 512, "dtype": "int64"},
        # the states of a served batch: sixteen tensors of 512 rows of 64 KB
        {"name": "beam_reorder_states", "op": "beam_reorder", "groups": 64, "beams": 8, "outer": 1, "tensors": 16,
         "inner": 32768, "stride": 32768, "dtype": "bf16"},
        # the update of a small square core
        {"name": "orthogonalize_core", "op": "orthogonalize", "rows": 64, "cols": 64, "dtype": "fp32", "by": "rows",
         "steps": 5},
        # the gradient of a connectome-shaped factor (r = 64)
        {"name": "orthogonalize_factor", "op": "orthogonalize", "rows": COLUMNS, "cols": 64, "dtype": "fp32",
         "by": "rows", "steps": 5},
        # the gradient of the other factor at r = 256, 16 bits, wide
        {"name": "orthogonalize_wide", "op": "orthogonalize", "rows": 256, "cols": COLUMNS, "dtype": "bf16",
         "by": "rows", "steps": 5},
        # a large square layer
        {"name": "orthogonalize_square", "op": "orthogonalize", "rows": 4096, "cols": 4096, "dtype": "bf16",
         "by": "rows", "steps": 5},
        # a training step of the planted 20,000-column workload's factor (r = 32), 32-bit throughout
        {"name": "muon_step_factor", "op": "muon_step", "rows": 32, "cols": 20000, "dtype": "fp32", "grad": "fp32",
         "by": "rows", "nesterov": True, "decay": 0.0, "steps": 5},
        # a training step of an odd-sized layer: 16-bit weights and gradients, 32-bit momentum
        {"name": "muon_step_layer", "op": "muon_step", "rows": 2047, "cols": 1001, "dtype": "bf16", "grad": "bf16",
         "by": "rows", "nesterov": True, "decay": 0.1, "steps": 5},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["beam_select", "beam_select", "beam_reorder", "orthogonalize", "orthogonalize", "muon_step"])
    if op == "beam_select":
        vocab = _log_int(rng, 2, COLUMNS)
        beams = _log_int(rng, 1, 32)
        groups = _log_int(rng, 1, max(1, min(512, MOST_LOGITS // (vocab * beams))))
        return {"op": op, "groups": groups, "beams": beams, "width": rng.choice([beams, beams, 2 * beams]),
                "vocab": vocab, "stride": vocab + rng.choice([0, 0, 0, 1, 8, -vocab % 64]),
                "dtype": rng.choice(["fp32", "bf16", "bf16", "fp16"]) if groups * beams * vocab < MOST_LOGITS // 2
                else rng.choice(["bf16", "fp16"]),
                "finished": rng.choice([0.0, 0.2, 0.5]), "unused": rng.choice([0.0, 0.0, 0.3]),
                "banned": rng.choice([0.0, 0.0, 0.1]) if vocab >= 16 else 0.0,
                "temperature": rng.choice([1.0, 1.0, 0.7, 1.3])}
    if op == "beam_reorder":
        beams, dtype, tensors = _log_int(rng, 2, 32), rng.choice(["fp32", "bf16", "fp16", "int64", "int32"]), \
            _log_int(rng, 1, 48)
        groups, outer = _log_int(rng, 1, 128), rng.choice([1, 1, 3, 4])
        inner = _log_int(rng, 1, max(1, MOST_STATE // (tensors * groups * beams * outer * BYTES[dtype] * 2)))
        return {"op": op, "groups": groups, "beams": beams, "outer": outer, "tensors": tensors, "inner": inner,
                "stride": inner + rng.choice([0, 0, 0, 3, 64]), "dtype": dtype}
    small = _log_int(rng, 1, 4096)
    large = _log_int(rng, small, max(small, min(COLUMNS, MOST_MATRIX // small, MOST_PRODUCT // small ** 2)))
    rows, cols = rng.choice([(small, large), (large, small)])
    dtype, by = rng.choice(["fp32", "bf16", "bf16", "fp16"]), rng.choice(["rows", "rows", "columns"])
    case = {"op": op, "rows": rows, "cols": cols, "dtype": dtype, "by": by, "steps": 5}
    if op == "muon_step":
        case.update(grad=rng.choice([dtype, dtype, "fp32"]), nesterov=rng.random() < 0.7, decay=rng.choice([0.0, 0.1]))
    else:
        case["steps"] = rng.choice([5, 5, 5, 3, 6])
    return case


# --------------------------------------------------------------------------------------------------------- inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(shape, g, dtype):
    return torch.randn(shape, device="cuda", generator=g, dtype=dtype)


def _gradient(case, g, dtype):
    """A gradient in earnest: a few strong directions over a floor of noise, small values; rows or columns adjacent."""
    rows, cols = case["rows"], case["cols"]
    k = max(1, min(8, rows, cols))
    x = _randn((rows, k), g, torch.float32) @ _randn((k, cols), g, torch.float32) / math.sqrt(k)
    x = (1e-3 * (x + 0.2 * _randn((rows, cols), g, torch.float32))).to(DTYPES[dtype])
    return x if case["by"] == "rows" else x.t().contiguous().t()


def prepare(case, seed):
    g = _generator(seed)
    op = case["op"]
    if op == "beam_select":
        B, K, V = case["groups"], case["beams"], case["vocab"]
        x = torch.empty((B * K, case["stride"]), device="cuda", dtype=DTYPES[case["dtype"]])
        for at in range(0, B * K, 512):
            rows = x[at:at + 512]
            rows.copy_(2.5 * _randn(rows.shape, g, torch.float32))
        x = x[:, :V]
        if case["banned"]:
            x[:, torch.randperm(V, device="cuda", generator=g)[:int(case["banned"] * V)]] = float("-inf")
        # a trained model prefers a few columns to the rest
        likely = torch.randint(0, V, (B * K, 4), device="cuda", generator=g)
        x.scatter_(1, likely, (7.0 + 2.0 * _randn((B * K, 4), g, torch.float32)).to(x.dtype))
        scores = -20.0 + 3.0 * _randn((B, K), g, torch.float32)
        scores = scores.sort(1, descending=True).values
        end = V // 2
        done = torch.rand((B, K), device="cuda", generator=g) < case["finished"]
        unused = torch.rand((B, K), device="cuda", generator=g) < case["unused"]
        scores = torch.where(unused, float("-inf"), scores)
        return {"op": op, "logits": x, "scores": scores, "finished": done if case["finished"] else None, "end": end,
                "width": case["width"], "temperature": case["temperature"]}
    if op == "beam_reorder":
        B, K, L = case["groups"], case["beams"], case["outer"]
        parents = torch.randint(0, K, (B, K), device="cuda", generator=g)
        states = []
        for _ in range(case["tensors"]):
            shape = (L, B * K, case["stride"])
            if case["dtype"].startswith("int"):
                x = torch.randint(0, COLUMNS, shape, device="cuda", generator=g, dtype=DTYPES[case["dtype"]])
            else:
                x = _randn(shape, g, DTYPES[case["dtype"]])
            states.append(x[:, :, :case["inner"]])
        return {"op": op, "states": states, "parents": parents}
    s = {"op": op, "steps": case["steps"]}
    if op == "orthogonalize":
        s["update"] = _gradient(case, g, case["dtype"])
        return s
    weight = _gradient(case, g, "fp32") * 30.0
    s["weight"] = weight.to(DTYPES[case["dtype"]])
    s["grad"] = _gradient(case, g, case["grad"])
    s["momentum"] = _gradient(case, g, "fp32")
    s.update(lr=0.02, beta=0.95, nesterov=case["nesterov"], decay=case["decay"])
    return s


# ----------------------------------------------------------------------------------------------------------- runs

def _order(x):
    """Whole numbers in the order of (value, lower column first): the value's bits, then the column from the end."""
    bits = (x.float() + 0.0).view(torch.int32)
    bits = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).to(torch.int64)
    return bits * 2 ** 32 + (2 ** 31 - 1 - torch.arange(x.shape[1], device=x.device))


def _plain_select(s):
    x, w = s["logits"], s["width"]
    B, K = s["scores"].shape
    n = min(w, x.shape[1])
    z = x.float() / s["temperature"]
    top = z.max(1, keepdim=True).values
    total = torch.exp(z - top).sum(1, dtype=torch.float64)
    at = 2 ** 31 - 1 - (torch.topk(_order(x), n, 1).values & (2 ** 32 - 1))   # each row's best, of equal ones the first
    # in 64 bits: candidates of two beams may lie next to each other
    value = (x.gather(1, at).double() - x.double().gather(1, at[:, :1])) / s["temperature"] - total.log()[:, None]
    value = s["scores"].double()[:, :, None] + value.view(B, K, n)
    at = at.view(B, K, n)
    done = s["finished"]
    if done is not None:   # a finished beam goes on as it is
        first = torch.arange(n, device=x.device) == 0
        value = torch.where(done[:, :, None], torch.where(first, s["scores"].double()[:, :, None], float("-inf")), value)
        at = torch.where(done[:, :, None], s["end"], at)
    value = torch.where(value.isfinite(), value, float("-inf"))
    pad = max(0, w - K * n)
    value = torch.cat([value.view(B, K * n), torch.full((B, pad), float("-inf"), device=x.device)], 1)
    at = torch.cat([at.view(B, K * n), torch.zeros((B, pad), device=x.device, dtype=torch.int64)], 1)
    value, index = torch.sort(value, dim=1, descending=True, stable=True)
    value, index = value[:, :w], index[:, :w]
    offered = value > float("-inf")
    parents = torch.where(offered, index // n, 0)
    tokens = torch.where(offered, at.gather(1, index), -1)
    out = {"scores": value.float(), "parents": parents, "tokens": tokens}
    if done is not None:
        out["finished"] = (offered & done.gather(1, parents)) | (tokens == s["end"])
    return out


def _plain_newton_schulz(x, steps):
    a, b, c = COEFFICIENTS
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    x = x / (x.square().sum().sqrt() + EPS)
    for _ in range(steps):
        gram = x @ x.t()
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.t() if tall else x


def _scale(weight):
    return math.sqrt(max(1.0, weight.shape[0] / weight.shape[1]))


def run(state):
    s = state
    op = s["op"]
    if own:
        from paper_2608_21607_gb300 import tuning

        if op == "beam_select":
            r = tuning.beam_select(s["logits"], s["scores"], width=s["width"], finished=s["finished"],
                                   end=None if s["finished"] is None else s["end"], temperature=s["temperature"])
            out = {"scores": r.scores, "parents": r.parents, "tokens": r.tokens}
            if s["finished"] is not None:
                out["finished"] = r.finished
            return out
        if op == "beam_reorder":
            tuning.beam_reorder(s["states"], s["parents"], dim=1)
            return s["states"]
        if op == "orthogonalize":
            return tuning.orthogonalize(s["update"], steps=s["steps"])
        tuning.muon_step(s["weight"], s["grad"], s["momentum"], lr=s["lr"], beta=s["beta"], nesterov=s["nesterov"],
                         weight_decay=s["decay"], steps=s["steps"])
        return [s["weight"], s["momentum"]]
    if op == "beam_select":
        return _plain_select(s)
    if op == "beam_reorder":
        B, K = s["parents"].shape
        rows = (s["parents"] + K * torch.arange(B, device="cuda")[:, None]).view(-1)
        for x in s["states"]:
            x.copy_(x[:, rows])
        return s["states"]
    if op == "orthogonalize":
        return _plain_newton_schulz(s["update"].float(), s["steps"]).to(s["update"].dtype)
    w, m, g = s["weight"], s["momentum"], s["grad"].float()
    m.copy_(s["beta"] * m + (1 - s["beta"]) * g)
    update = s["beta"] * m + (1 - s["beta"]) * g if s["nesterov"] else m
    step = _plain_newton_schulz(update, s["steps"])
    w.copy_((1 - s["lr"] * s["decay"]) * w.float() - s["lr"] * _scale(w) * step)
    return [w, m]


# --------------------------------------------------------------------------------------------- definitions in 64 bits

def _exact_polar(x, steps):
    """The Newton-Schulz map on the singular values: x V p(L) V^T with the eigenvalues L of the smaller Gram matrix."""
    a, b, c = COEFFICIENTS
    if x.shape[0] < x.shape[1]:
        return _exact_polar(x.t(), steps).t()
    x = x / (torch.linalg.vector_norm(x) + EPS)
    lam, v = torch.linalg.eigh(x.t() @ x)
    lam = lam.clamp(min=0.0)
    factor = torch.ones_like(lam)
    for _ in range(steps):
        q = a + lam * (b + lam * c)
        factor, lam = factor * q, lam * q * q
    return x @ ((v * factor) @ v.t())


def exact(case, seed):
    s = prepare(case, seed)
    op = s["op"]
    if op == "beam_select":
        B, K = s["scores"].shape
        V, w = s["logits"].shape[1], s["width"]
        out = {"scores": [], "parents": [], "tokens": [], "finished": []}
        for b in range(B):
            lp = torch.log_softmax(s["logits"][b * K:(b + 1) * K].double() / s["temperature"], 1)
            value = s["scores"][b].double()[:, None] + lp
            done = s["finished"][b] if s["finished"] is not None else torch.zeros(K, dtype=torch.bool, device="cuda")
            value[done] = float("-inf")
            value[done, s["end"]] = s["scores"][b].double()[done]
            value = value.nan_to_num(nan=float("-inf"), posinf=float("-inf"), neginf=float("-inf")).view(-1)
            border = torch.topk(value, min(w, K * V)).values[-1]
            near = torch.nonzero(value >= border)[:, 0]          # ascending: equal values in the order of their index
            near = near[torch.sort(value[near], dim=0, descending=True, stable=True).indices][:w]
            near = near[value[near] > float("-inf")]
            row = torch.full((w,), float("-inf"), device="cuda", dtype=torch.float64)
            parent, token = torch.zeros(w, device="cuda", dtype=torch.int64), torch.full((w,), -1, device="cuda")
            n = near.numel()
            row[:n], parent[:n], token[:n] = value[near], near // V, near % V
            end = token == s["end"]
            for name, v in zip(("scores", "parents", "tokens", "finished"), (row, parent, token, end)):
                out[name].append(v)
        out = {k: torch.stack(v) for k, v in out.items()}
        if s["finished"] is None:
            del out["finished"]
        return out
    if op == "beam_reorder":
        K = s["parents"].shape[1]
        moved = []
        for x in s["states"]:
            y = x.unflatten(1, (-1, K))
            at = s["parents"].view(1, -1, K, 1).expand(y.shape)
            moved.append(torch.gather(y, 2, at).flatten(1, 2))
        return moved
    if op == "orthogonalize":
        return _exact_polar(s["update"].double(), s["steps"])
    w, m, g = s["weight"].double(), s["momentum"].double(), s["grad"].double()
    m = torch.lerp(m, g, 1 - s["beta"])
    step = _exact_polar(torch.lerp(g, m, s["beta"]) if s["nesterov"] else m, s["steps"])
    return [w - s["lr"] * (s["decay"] * w + _scale(w) * step), m]


# ----------------------------------------------------------------------------------------------------------- work

def _products(case):
    """Operations of the cheaper of two ways: the steps as they stand, symmetric products by half; or, for a long
    matrix, one Gram matrix, the steps on it, and one product."""
    small, large = sorted((case["rows"], case["cols"]))
    square = small * small
    return min(case["steps"] * square * (3 * large + small), square * (3 * large + 4 * case["steps"] * small))


def work(case):
    """Bytes read once and written once, and the operations of sums and products."""
    op = case["op"]
    if op == "beam_select":
        rows = case["groups"] * case["beams"]
        live = rows * (1.0 - case["finished"]) * (1.0 - case["unused"])
        return {"bytes": live * case["vocab"] * BYTES[case["dtype"]] + 4 * rows + 20 * case["groups"] * case["width"],
                "flops": 4 * live * case["vocab"]}
    if op == "beam_reorder":
        rows = case["groups"] * case["beams"]
        moved = case["tensors"] * case["outer"] * rows * case["inner"] * BYTES[case["dtype"]]
        return {"bytes": 2 * moved + 8 * rows, "flops": 0}
    n = case["rows"] * case["cols"]
    if op == "orthogonalize":
        return {"bytes": 2 * n * BYTES[case["dtype"]], "flops": _products(case)}
    return {"bytes": n * (2 * BYTES[case["dtype"]] + BYTES[case["grad"]] + 8), "flops": _products(case)}
