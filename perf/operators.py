"""Timing cases of the operators on logits: what a program does with the rows that a query leaves on the device, or that a
training step gets from a model of its own.

  sample   draws one class per row from given random numbers, under temperature, top-k, top-p and min-p of each row
  top      the leading logits of each row, in order, and the probability mass outside them
  distill  the loss of each row against a teacher's leading logits, and (grad) its gradient by the row

A row has as many logits as there are classes: 10 and 1000 are this repository's SuperNets, more are label sets and
vocabularies of ordinary sizes.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
ELEM_BYTES = {"fp32": 4, "bf16": 2}
MOST_ELEMENTS = 1 << 27  # rows * classes of the largest case


def _sample(name, dtype, rows, classes, temperature=True, top_k=True, top_p=True, min_p=True, masked=False):
    return {"name": name, "kind": "sample", "dtype": dtype, "rows": rows, "classes": classes, "temperature": temperature,
            "top_k": top_k, "top_p": top_p, "min_p": min_p, "masked": masked}


def _top(name, dtype, rows, classes, k, temperature=1.0):
    return {"name": name, "kind": "top", "dtype": dtype, "rows": rows, "classes": classes, "k": k, "temperature": temperature}


def _distill(name, dtype, rows, classes, k, grad, rest=True, temperature=1.0, masked=False):
    return {"name": name, "kind": "distill", "dtype": dtype, "rows": rows, "classes": classes, "k": k, "grad": grad,
            "rest": rest, "temperature": temperature, "masked": masked}


def listed():
    return [
        # the answer to a lone query, every filter on: latency alone
        _sample("sample_1x1000", "fp32", 1, 1000),
        # a batch of 16 queries, plain draws from the softmax at a temperature
        _sample("sample_16x1000_plain", "fp32", 16, 1000, top_k=False, top_p=False, min_p=False),
        # one token of one sequence over a long vocabulary: a row that one compute unit would be long at
        _sample("sample_1x131071", "bf16", 1, 131071),
        # an odd batch of sequences, a fifth of the vocabulary masked
        _sample("sample_61x50001", "bf16", 61, 50001, masked=True),
        # many sequences over a long vocabulary
        _sample("sample_512x100003", "fp32", 512, 100003, top_k=False),
        # the five best classes of a batch of answers
        _top("top5_16x1000", "fp32", 16, 1000, 5),
        # what a teacher stores for a few long rows, and for a training set
        _top("top100_3x200003", "fp32", 3, 200003, 100, 2.0),
        _top("top64_2048x32001", "bf16", 2048, 32001, 64),
        # how far the answers of a SubNet lie from the largest SubNet's: forward only
        _distill("distill_loss_64x1000", "fp32", 64, 1000, 20, False),
        _distill("distill_loss_5x250007", "bf16", 5, 250007, 100, False, temperature=2.0),
        # training steps: a classifier's batch, tokens over a vocabulary with its padding masked and no mass outside the list
        _distill("distill_grad_256x1000", "fp32", 256, 1000, 20, True, temperature=2.0),
        _distill("distill_grad_4096x32000", "bf16", 4096, 32000, 64, True, rest=False, masked=True),
    ]


def draw(rng):
    def log_int(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))

    kind, dtype = rng.choice(["sample", "sample", "top", "distill", "distill"]), rng.choice(["fp32", "bf16"])
    classes = log_int(10, 250007)
    rows = log_int(1, max(1, min(4096, (MOST_ELEMENTS >> (1 if kind != "distill" else 0)) // classes)))
    if kind == "sample":
        on = [rng.random() < 0.7 for _ in range(4)]
        case = _sample("", dtype, rows, classes, *on, rng.random() < 0.3)
    elif kind == "top":
        case = _top("", dtype, rows, classes, log_int(1, min(256, classes)), rng.choice([0.5, 1.0, 2.0]))
    else:
        case = _distill("", dtype, rows, classes, log_int(1, min(256, classes)), rng.random() < 0.7, rng.random() < 0.6,
                        rng.choice([1.0, 2.0, 4.0]), rng.random() < 0.3)
    del case["name"]
    return case


# ---------------------------------------------------------------- what a case consists of

def _logits(gen, rows, classes, masked):
    """float32 rows as classifiers and language models give them: a bell of unlikely classes and a few that stand out."""
    z = torch.randn(rows, classes, generator=gen, device="cuda")
    z *= 1.5 + torch.rand(rows, 1, generator=gen, device="cuda")
    n = min(classes, 12)
    first = torch.randint(0, classes, (rows, 1), generator=gen, device="cuda")
    at = (first + classes // n * torch.arange(n, device="cuda")) % classes
    up = 5.0 + 6.0 * torch.rand(rows, n, generator=gen, device="cuda")
    z.scatter_(1, at, up)
    if masked:  # classes that may not be answered with, and a tail that pads the row
        allowed = torch.rand(classes, generator=gen, device="cuda") >= 0.2
        allowed[0] = True
        allowed[max(1, classes - classes // 64):] = False
        z.masked_fill_(~allowed, float("-inf"))
    return z


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rows, classes, dtype = case["rows"], case["classes"], DTYPES[case["dtype"]]
    z = _logits(gen, rows, classes, case.get("masked", False))
    state = dict(case=case)
    if case["kind"] == "distill":
        T = case["temperature"]
        teacher = z + 0.7 * torch.randn(rows, classes, generator=gen, device="cuda")
        values, index = torch.topk(teacher, case["k"], dim=1)
        out = teacher.scatter_(1, index, float("-inf")) / T
        # (a padded list: rows may hold fewer classes than it has places)
        index = torch.where(values == float("-inf"), -1, index)
        state.update(values=values, index=index.to(torch.int32), rest=None,
                     weight=torch.full((rows,), 1.0 / rows, device="cuda"))
        if case["rest"]:
            top = torch.logsumexp(values.double() / T, 1)
            state["rest"] = torch.sigmoid(torch.logsumexp(out.double(), 1) - top).float()
        del teacher, out
    state["logits"] = z.to(dtype)
    if case["kind"] == "sample":
        def uniform(lo, hi):
            return lo + (hi - lo) * torch.rand(rows, generator=gen, device="cuda")

        state["uniform"] = torch.rand(rows, generator=gen, device="cuda")
        state["temperature"] = uniform(0.5, 1.3) if case["temperature"] else None
        state["top_k"] = torch.randint(1, 200, (rows,), generator=gen, device="cuda", dtype=torch.int32) if case["top_k"] else None
        state["top_p"] = uniform(0.8, 0.99) if case["top_p"] else None
        state["min_p"] = uniform(0.001, 0.05) if case["min_p"] else None
    if own:
        import paper_2306_17266_amd as S
        n = S.sushi_logits_workspace(rows, classes)
        state.update(ctx=S.Sushi(0), workspace=torch.empty(n, dtype=torch.uint8, device="cuda"))
        state["out_class"] = torch.empty(rows, device="cuda", dtype=torch.int32)
        state["out_row"] = torch.empty(rows, device="cuda")
        if case["kind"] == "top":
            state["out_values"] = torch.empty(rows, case["k"], device="cuda")
            state["out_classes"] = torch.empty(rows, case["k"], device="cuda", dtype=torch.int32)
        if case.get("grad"):
            state["out_grad"] = torch.empty_like(state["logits"])
    torch.cuda.synchronize()
    return state


# ---------------------------------------------------------------- the operators in their plain form

def _plain_sample(s):
    """In 64 bits: where a sum passes a border decides which class comes out."""
    z = s["logits"].double()
    if s["temperature"] is not None:
        z = z / s["temperature"].double()[:, None]
    w = torch.exp(z - z.amax(1, keepdim=True))
    order = torch.sort(s["logits"].float(), dim=1, descending=True, stable=True).indices
    ws = w.gather(1, order)
    keep = torch.ones_like(ws, dtype=torch.bool)
    if s["top_k"] is not None:
        keep &= torch.arange(z.shape[1], device=z.device)[None, :] < s["top_k"][:, None]
    if s["top_p"] is not None:
        before = torch.cumsum(ws, 1) - ws
        keep &= before < s["top_p"].double()[:, None] * ws.sum(1, keepdim=True)
    if s["min_p"] is not None:
        keep &= ws >= s["min_p"].double()[:, None]
    kept = torch.zeros_like(w).scatter_(1, order, torch.where(keep, ws, 0.0))
    upto = torch.cumsum(kept, 1)
    total = upto[:, -1:]
    drawn = (upto > s["uniform"].double()[:, None] * total).to(torch.uint8).argmax(1, keepdim=True)
    return drawn[:, 0].to(torch.int32), torch.log(kept.gather(1, drawn) / total)[:, 0].float()


def _plain_top(s):
    z, k = s["logits"].float(), s["case"]["k"]
    values, order = torch.sort(z, dim=1, descending=True, stable=True)
    w = torch.exp((values - values[:, :1]) / s["case"]["temperature"])
    rest = w[:, k:].sum(1) / w.sum(1)
    return values[:, :k].contiguous(), order[:, :k].to(torch.int32), rest


def _plain_distill(s):
    """What belongs to a row in 64 bits: its loss is a small difference of large terms."""
    z, T = s["logits"].float(), s["case"]["temperature"]
    listed_ = s["index"] >= 0
    index = s["index"].clamp_min(0).long()
    t = torch.where(listed_, s["values"].double(), float("-inf")) / T
    p = torch.exp(t - t.amax(1, keepdim=True))
    rest = torch.zeros_like(p[:, 0]) if s["rest"] is None else s["rest"].double()
    p = p / p.sum(1, keepdim=True) * (1.0 - rest)[:, None]
    best = z.amax(1, keepdim=True)
    e = torch.exp((z - best) / T)
    outside = torch.ones_like(z, dtype=torch.bool)
    rows = torch.arange(z.shape[0], device=z.device)[:, None].expand_as(index)
    outside[rows[listed_], index[listed_]] = False
    e_rest = torch.where(outside, e, 0.0).sum(1, dtype=torch.float64)
    e_top = torch.where(listed_, torch.exp((z.gather(1, index).double() - best.double()) / T), 0.0)
    total = e_rest + e_top.sum(1)
    loss = torch.where(p > 0, p * torch.log(p * total[:, None] / e_top), 0.0).sum(1)
    loss = loss + torch.where(rest > 0, rest * torch.log(rest * total / e_rest), 0.0)
    if not s["case"]["grad"]:
        return loss.float()
    share = torch.where(rest > 0, 1.0 - rest * total / e_rest, 1.0)
    scale = s["weight"].double() / (T * total)
    grad = torch.where(outside, e * (scale * share).float()[:, None], 0.0)
    grad.scatter_add_(1, index, (torch.where(listed_, e_top - p * total[:, None], 0.0) * scale[:, None]).float())
    return loss.float(), grad.to(s["logits"].dtype)


def run(s):
    kind = s["case"]["kind"]
    if not own:
        return {"sample": _plain_sample, "top": _plain_top, "distill": _plain_distill}[kind](s)
    ctx, work = s["ctx"], s["workspace"]
    if kind == "sample":
        ctx.sushi_sample(s["logits"], s["uniform"], s["out_class"], s["out_row"], temperature=s["temperature"], top_k=s["top_k"],
                         top_p=s["top_p"], min_p=s["min_p"], workspace=work)
        return s["out_class"], s["out_row"]
    if kind == "top":
        ctx.sushi_top_logits(s["logits"], s["out_values"], s["out_classes"], s["out_row"], temperature=s["case"]["temperature"],
                             workspace=work)
        return s["out_values"], s["out_classes"], s["out_row"]
    grad = s["out_grad"] if s["case"]["grad"] else None
    ctx.sushi_distill(s["logits"], s["values"], s["index"], s["out_row"], rest=s["rest"], temperature=s["case"]["temperature"],
                      weight=s["weight"], grad=grad, workspace=work)
    return s["out_row"] if grad is None else (s["out_row"], grad)


def work(case):
    """The logits read once, the row's parameters or the teacher's list read once, the outputs written once; an exponential
    counts as one operation beside the subtraction, the scaling and the sum of every logit."""
    rows, n = case["rows"], case["rows"] * case["classes"]
    byts = n * ELEM_BYTES[case["dtype"]]
    if case["kind"] == "sample":
        return {"bytes": byts + rows * 4.0 * (3 + sum(case[f] for f in ("temperature", "top_k", "top_p", "min_p"))), "flops": 4.0 * n}
    if case["kind"] == "top":
        return {"bytes": byts + rows * (8.0 * case["k"] + 4.0), "flops": 4.0 * n}
    byts += rows * (8.0 * case["k"] + 4.0 + 4.0 * case["rest"])
    if case["grad"]:
        byts += n * ELEM_BYTES[case["dtype"]] + rows * 4.0
    return {"bytes": byts, "flops": (6.0 if case["grad"] else 4.0) * n}


# ---------------------------------------------------------------- the definitions in 64 bits, row by row on the host

def _exact_sample(s):
    def column(name):
        return None if s[name] is None else s[name].double().cpu().numpy()

    T, top_k, top_p, min_p, u = (column(n) for n in ("temperature", "top_k", "top_p", "min_p", "uniform"))
    logits = s["logits"].cpu()
    classes, logs = [], []
    for r in range(logits.shape[0]):
        z = logits[r].double().numpy()
        best = z.max()
        w = np.exp((z - best) / (1.0 if T is None else T[r]))
        kept = np.ones(len(z), dtype=bool)
        if min_p is not None:
            kept &= w >= min_p[r]
        if top_k is not None or top_p is not None:
            order = np.argsort(-z, kind="stable")
            last = len(z) if top_k is None else min(len(z), int(top_k[r]))
            if top_p is not None:
                upto = np.cumsum(w[order])
                last = min(last, 1 + int(np.searchsorted(upto, top_p[r] * w.sum(), side="left")))
            kept[order[last:]] = False
        members = np.flatnonzero(kept)
        upto = np.cumsum(w[members])
        n = min(len(members) - 1, int(np.searchsorted(upto, u[r] * upto[-1], side="right")))
        classes.append(members[n])
        logs.append((z[members[n]] - best) / (1.0 if T is None else T[r]) - math.log(upto[-1]))
    return np.array(classes, dtype=np.int32), np.array(logs)


def _exact_top(s):
    k, T = s["case"]["k"], s["case"]["temperature"]
    logits = s["logits"].cpu()
    values, classes, rest = [], [], []
    for r in range(logits.shape[0]):
        z = logits[r].double().numpy()
        # (only what reaches the k-th largest value is sorted)
        members = np.flatnonzero(z >= np.partition(z, len(z) - k)[len(z) - k])
        first = members[np.argsort(-z[members], kind="stable")][:k]
        w = np.exp((z - z.max()) / T)
        total = w.sum()
        w[first] = 0.0
        values.append(z[first])
        classes.append(first)
        rest.append(w.sum() / total)
    return np.array(values), np.array(classes, dtype=np.int32), np.array(rest)


def _exact_distill(s):
    T, logits = s["case"]["temperature"], s["logits"].cpu()
    t_all, index_all, weight = s["values"].double().cpu().numpy(), s["index"].cpu().numpy(), s["weight"].double().cpu().numpy()
    rest = None if s["rest"] is None else s["rest"].double().cpu().numpy()
    losses, grads = [], np.empty(logits.shape if s["case"]["grad"] else (0,))
    for r in range(logits.shape[0]):
        z = logits[r].double().numpy() / T
        at = index_all[r][index_all[r] >= 0]
        t = t_all[r][index_all[r] >= 0] / T
        mass = 1.0 if rest is None else 1.0 - rest[r]
        log_p = t - t.max()
        log_p += math.log(mass) - math.log(np.exp(log_p).sum()) if mass > 0 else -math.inf
        best = z.max()
        e = np.exp(z - best)
        log_total = math.log(e.sum())
        e_top = e[at].copy()
        e[at] = 0.0
        outside = e.sum()
        p = np.exp(log_p)
        some = p > 0
        loss = float((p[some] * (log_p[some] - (z[at][some] - best - log_total))).sum())
        share = 1.0
        if mass < 1.0:
            loss += (1.0 - mass) * (math.log(1.0 - mass) - (math.log(outside) - log_total))
            share -= (1.0 - mass) * math.exp(log_total) / outside
        losses.append(loss)
        if s["case"]["grad"]:
            g = e * (share * math.exp(-log_total))
            g[at] = e_top * math.exp(-log_total) - p
            grads[r] = g * (weight[r] / T)
    if not s["case"]["grad"]:
        return np.array(losses)
    return np.array(losses), grads


def exact(case, seed):
    s = prepare(case, seed)
    return {"sample": _exact_sample, "top": _exact_top, "distill": _exact_distill}[case["kind"]](s)
