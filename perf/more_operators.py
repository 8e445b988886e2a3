"""The two ends of a training step, as cases that can be timed: rows looked up by id with their gradient, and what makes a loss of a model's
outputs - log probabilities of labels with entropy and top alternatives, and distillation from a teacher's top logits - with its gradient.

lookup   y[i] = scale table[ids[i]], zero where ids[i] is no row of the table.  backward: the sum of scale d_y[i] over the places of each id, as
         a gradient of the whole table, or (sparse) as the distinct ids in ascending order and a row for each.
         rows x dim: the table; n: how many are looked up; skew: how unevenly the ids fall (u^skew of a uniform u); padded: a tenth are -1
scores   z = scale x, lse = log sum exp z over a row's classes, log_prob = z[label] - lse (zero without a label), entropy = -sum p log p, and
         the `top` best classes with their log probabilities, the lowest class first where some are equal.  backward: the gradient of x from those of
         log_prob, entropy and lse.
         n x classes: the matrix; pad: columns between two rows that belong to somebody else; masked: a tenth of the values is -infinity;
         unlabelled: a third of the rows has the label -100
distill  q = softmax of scale v over a row's `entries` (class, teacher's logit) pairs, loss = sum of q (log q - log p[class]), p the student's softmax of
         scale x.  backward: the gradient of x from the loss's.
         ragged: rows have fewer entries than there are columns for, the rest names the class -1, some rows have none at all
"""
import math

import numpy as np
import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


# ---- the cases ------------------------------------------------------------------------------------------------------
def _case(name, op, **sizes):
    c = {"op": op, "backward": False, "dtype": "f32", "n": 1000, "scale": 1.0}
    c.update({"rows": 10_000, "dim": 128, "skew": 1.0, "padded": False, "sparse": False, "long_ids": True} if op == "lookup" else
             {"classes": 100, "pad": 0, "masked": False, "top": 0, "unlabelled": False, "regularised": False} if op == "scores" else
             {"classes": 100, "pad": 0, "masked": False, "entries": 16, "ragged": False})
    c.update(sizes)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # the targets of a first try's mini-batch, rows of 16: launches and waits
        _case("lookup_tiny", "lookup", n=512, rows=10_000, dim=16),
        # learned base rows for 24 mini-batches on a graph of two million nodes, popular nodes in many of them
        _case("lookup_nodes", "lookup", n=543_000, rows=2_000_000, dim=128, skew=2.0, scale=math.sqrt(128), long_ids=False),
        # their gradient for an optimiser that steps the touched rows only
        _case("lookup_nodes_backward_sparse", "lookup", backward=True, sparse=True, n=543_000, rows=2_000_000, dim=128, skew=2.0, scale=math.sqrt(128),
              long_ids=False),
        # relation embeddings of a link-prediction step's 50,000 edges: few relations have most of the edges
        _case("lookup_relations_backward", "lookup", backward=True, n=50_000, rows=14_824, dim=100, skew=4.0, long_ids=False),
        # wide half-precision rows of padded batches, the whole table's gradient
        _case("lookup_wide_half_backward", "lookup", backward=True, dtype="bf16", n=150_001, rows=300_007, dim=768, skew=3.0, padded=True),
        # answering for a few users at once: the five likeliest classes of 411 nodes
        _case("scores_serving", "scores", n=411, classes=100, top=5),
        # node classification: 128 mini-batches of 1,000 targets
        _case("scores_nodes", "scores", n=128_000, classes=172, top=5, unlabelled=True),
        # its loss's gradient at an odd number of classes, in half precision, with the entropy and the normaliser in the loss
        _case("scores_odd_half_backward", "scores", backward=True, dtype="f16", n=777_777, classes=153, unlabelled=True, regularised=True),
        # many candidates: 4,096 queries against 50,257, with twenty alternatives, at a temperature
        _case("scores_many_classes", "scores", dtype="bf16", n=4_096, classes=50_257, top=20, scale=1 / 0.7),
        # a single query against a million candidates, some not allowed
        _case("scores_one_query", "scores", n=1, classes=1_000_003, top=10, masked=True),
        # distillation from a teacher's 64 top logits at temperature two: the loss ...
        _case("distill_many_classes", "distill", dtype="bf16", n=8_192, classes=32_000, entries=64, scale=0.5),
        # ... and the gradient, the teacher's rows of uneven length, rows of logits that start anywhere
        _case("distill_many_classes_backward", "distill", backward=True, n=2_048, classes=50_257, entries=50, scale=0.5, ragged=True),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(("lookup", "scores", "distill"))
    dtype, backward = rng.choice(("f32", "f16", "bf16")), rng.random() < 0.5
    scale = rng.choice((1.0, rng.uniform(0.25, 2.0)))
    if op == "lookup":
        dim = rng.choice((16, 64, 100, 101, 128, 128, 256, 300, 512, 768, 1024))
        n = log_int(1, min(1_000_000, 69_000_000 // dim))
        return _case("", op, dtype=dtype, backward=backward, scale=scale, n=n, dim=dim, rows=log_int(1, min(4_000_000, 115_000_000 // dim)),
                     skew=rng.choice((1.0, 2.0, 3.0, 6.0)), padded=rng.random() < 0.3, sparse=backward and rng.random() < 0.5, long_ids=rng.random() < 0.5)
    classes = log_int(2, 300_000)
    c = _case("", op, dtype=dtype, backward=backward, scale=scale, classes=classes, n=log_int(1, min(800_000, (100_000_000 if backward else 200_000_000) // classes)),
              pad=rng.choice((0, 0, 0, 3, 8)), masked=classes >= 128 and rng.random() < 0.3)
    if op == "scores":
        c.update(top=0 if backward else min(classes, rng.choice((0, 1, 5, 10, 20, 32))), unlabelled=rng.random() < 0.4, regularised=backward and rng.random() < 0.4)
    else:
        c.update(entries=min(classes, 256, log_int(1, 256)), ragged=rng.random() < 0.5)
        c["n"] = max(1, min(c["n"], 20_000_000 // c["entries"]))
    return c


def _named(case):
    """How many of the places name a row, and how many different ones, which is what as many independent draws would have on average."""
    rows, valid = case["rows"], case["n"] - (case["n"] // 10 if case["padded"] else 0)
    p = np.diff((np.arange(rows + 1) / rows) ** (1 / case["skew"]))
    return valid, max(1, min(rows, valid, round(float(-np.expm1(valid * np.log1p(-np.minimum(p, 1 - 1e-12))).sum()))))


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _strided(values, pad):
    """The same values with `pad` columns of another's between the rows."""
    if pad == 0:
        return values
    wide = torch.full((values.shape[0], values.shape[1] + pad), float("nan"), dtype=values.dtype, device=values.device)
    wide[:, :values.shape[1]] = values
    return wide[:, :values.shape[1]]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, dtype = case["n"], _TYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def uniform(*shape):
        return torch.rand(shape, generator=g, device="cuda")

    s = {"case": dict(case)}
    if case["op"] == "lookup":
        rows = case["rows"]
        valid, distinct = _named(case)
        popular = (uniform(valid - distinct).double().pow(case["skew"]) * distinct).long().clamp(max=distinct - 1)
        place = torch.cat([torch.arange(distinct, device="cuda"), popular])      # each of the distinct ones once, then by popularity
        ids = torch.full((n,), -1, device="cuda")
        ids[torch.randperm(n, generator=g, device="cuda")[:valid]] = torch.randperm(rows, generator=g, device="cuda")[place]
        s["ids"] = ids if case["long_ids"] else ids.int()
        if case["backward"]:
            s["d_y"] = normal(n, case["dim"]).to(dtype)
        else:
            s["table"] = (0.1 * normal(rows, case["dim"])).to(dtype)
        return s
    classes = case["classes"]
    x = normal(n, classes) * (1 + uniform(n, 1) * 2)      # rows that are surer than others
    known = torch.randint(0, classes, (n,), generator=g, device="cuda")
    x[torch.arange(n, device="cuda"), known] += 4 * uniform(n)      # a model that has learnt something
    if case["op"] == "distill":      # the teacher's likeliest classes, as many different ones
        k = case["entries"]
        step = 1 + torch.randint(0, max(1, classes // k), (n, k), generator=g, device="cuda")
        step[:, 0] = 0
        named = (known[:, None] + step.cumsum(1)) % classes      # (k steps stay below one turn)
    else:
        named = known[:, None]
    if case["masked"]:      # what is not allowed is neither a label nor the teacher's
        allowed = x.gather(1, named)
        x.masked_fill_(uniform(n, classes) < 0.1, float("-inf"))
        x.scatter_(1, named, allowed)
    s["logits"] = _strided(x.to(dtype), case["pad"])
    if case["op"] == "scores":
        s["labels"] = torch.where(uniform(n) < 1 / 3, -100, known) if case["unlabelled"] else known
        if case["backward"]:
            s["lse"], s["entropy"] = (t.float() for t in _moments(s["logits"], case["scale"], torch.float64))
            s["d_log_prob"] = -uniform(n)      # (half-precision gradients are scaled up to their type's range)
            s["d_entropy"], s["d_lse"] = (0.1 * normal(n), 0.1 * normal(n)) if case["regularised"] else (None, None)
        return s
    s["teacher_ids"] = named.int()
    s["teacher_logits"] = (8 * uniform(n, k)).sort(1, descending=True).values
    if case["ragged"]:
        length = torch.where(uniform(n) < 0.05, 0, 1 + (uniform(n) * k).long())
        s["teacher_ids"].masked_fill_(torch.arange(k, device="cuda") >= length[:, None], -1)
    if case["backward"]:
        s["lse"] = _moments(s["logits"], case["scale"], torch.float64)[0].float()
        s["d_loss"] = uniform(n)
    return s


# ---- the operators' plain forms -------------------------------------------------------------------------------------
def _pieces(n, width):
    """Rows in pieces that leave room for what is made of them."""
    step = max(1, (1 << 25) // width)
    return [slice(lo, min(lo + step, n)) for lo in range(0, n, step)]


def _moments(x, scale, dtype):
    """Logarithm of the sum of exponentials, and entropy, of each row."""
    lse, entropy = [], []
    for at in _pieces(*x.shape):
        z = x[at].to(dtype) * scale
        m = z.max(1, keepdim=True).values
        m = torch.where(m == float("-inf"), torch.zeros_like(m), m)
        e = torch.exp(z - m)
        total = e.sum(1)
        weighted = torch.where(e > 0, e * (z - m), torch.zeros_like(e)).sum(1)
        lse.append(m[:, 0] + torch.log(total))
        entropy.append(torch.log(total) - weighted / total)
    return torch.cat(lse), torch.cat(entropy)


def _lookup(s):
    ids, table = s["ids"].long(), s["table"]
    valid = (ids >= 0) & (ids < table.shape[0])
    y = table[ids.clamp(0, table.shape[0] - 1)].float() * s["case"]["scale"]
    return {"y": torch.where(valid[:, None], y, torch.zeros_like(y)).to(table.dtype)}


def _lookup_backward(s):
    c, ids, d_y = s["case"], s["ids"].long(), s["d_y"]
    valid = (ids >= 0) & (ids < c["rows"])
    kept, at = ids[valid].sort(stable=True)
    first = torch.ones_like(kept, dtype=torch.bool)
    first[1:] = kept[1:] != kept[:-1]
    distinct, group = kept[first], first.long().cumsum(0) - 1
    sums = torch.zeros(len(distinct), c["dim"], dtype=torch.float64, device="cuda")
    sums.index_add_(0, group, d_y[valid][at].double())
    sums = (sums * c["scale"]).to(d_y.dtype)
    if c["sparse"]:
        return {"ids": distinct.to(s["ids"].dtype), "rows": sums}
    out = torch.zeros(c["rows"], c["dim"], dtype=d_y.dtype, device="cuda")
    out[distinct] = sums
    return {"d_table": out}


def _scores(s):
    c, x = s["case"], s["logits"]
    lse, entropy = _moments(x, c["scale"], torch.float32)
    label = s["labels"].clamp(0, c["classes"] - 1)
    at_label = x.gather(1, label[:, None])[:, 0].float() * c["scale"] - lse
    valid = (s["labels"] >= 0) & (s["labels"] < c["classes"])
    out = {"log_prob": torch.where(valid, at_label, torch.zeros_like(at_label)), "entropy": entropy, "lse": lse}
    if c["top"]:
        best = [x[at].float().sort(dim=1, descending=True, stable=True) for at in _pieces(*x.shape)]
        out["top_ids"] = torch.cat([b.indices[:, :c["top"]] for b in best]).int()
        out["top_log_probs"] = torch.cat([b.values[:, :c["top"]] for b in best]) * c["scale"] - lse[:, None]
    return out


def _scores_backward(s):
    c, x = s["case"], s["logits"]
    out = torch.empty(x.shape, dtype=x.dtype, device="cuda")
    valid = (s["labels"] >= 0) & (s["labels"] < c["classes"])
    g = torch.where(valid, s["d_log_prob"], torch.zeros_like(s["d_log_prob"]))
    label = s["labels"].clamp(0, c["classes"] - 1)
    for at in _pieces(*x.shape):
        log_p = x[at].float() * c["scale"] - s["lse"][at][:, None]
        p = torch.exp(log_p)
        d = -p * g[at][:, None]
        if c["regularised"]:
            d += p * s["d_lse"][at][:, None]
            d -= torch.where(p > 0, p * (log_p + s["entropy"][at][:, None]), torch.zeros_like(p)) * s["d_entropy"][at][:, None]
        d.scatter_add_(1, label[at][:, None], g[at][:, None])
        out[at] = (d * c["scale"]).to(x.dtype)
    return {"d_logits": out}


def _teacher(s):
    """The teacher's probabilities, and their logarithms, of each row's entries; zero where there is none."""
    c = s["case"]
    valid = (s["teacher_ids"] >= 0) & (s["teacher_ids"] < c["classes"])
    v = (s["teacher_logits"].float() * c["scale"]).masked_fill(~valid, float("-inf"))
    m = v.max(1, keepdim=True).values
    m = torch.where(m == float("-inf"), torch.zeros_like(m), m)
    e = torch.exp(v - m)
    total = e.sum(1, keepdim=True).clamp(min=1e-30)
    return valid, e / total, v - m - torch.log(total)


def _distill(s):
    c, x = s["case"], s["logits"]
    lse = _moments(x, c["scale"], torch.float32)[0]
    valid, q, log_q = _teacher(s)
    log_p = x.gather(1, s["teacher_ids"].long().clamp(0, c["classes"] - 1)).float() * c["scale"] - lse[:, None]
    return {"loss": torch.where(valid & (q > 0), q * (log_q - log_p), torch.zeros_like(q)).sum(1), "lse": lse}


def _distill_backward(s):
    c, x = s["case"], s["logits"]
    valid, q, _ = _teacher(s)
    out = torch.empty(x.shape, dtype=x.dtype, device="cuda")
    some = valid.any(1).float()
    for at in _pieces(*x.shape):
        d = torch.exp(x[at].float() * c["scale"] - s["lse"][at][:, None]) * some[at][:, None]
        d.scatter_add_(1, s["teacher_ids"][at].long().clamp(0, c["classes"] - 1), -q[at])
        out[at] = (d * (s["d_loss"][at] * c["scale"])[:, None]).to(x.dtype)
    return {"d_logits": out}


# ---- the same through the package -----------------------------------------------------------------------------------
_kept_context = []


def _context():
    """The program's one context on the GPU."""
    import paper_2202_02365_b200 as mg
    if not _kept_context:
        _kept_context.append(mg.Context(0))
    return _kept_context[0]


def _run_own(s):
    ctx, c = _context(), s["case"]
    if c["op"] == "lookup":
        if not c["backward"]:
            return {"y": ctx.embedding(s["table"], s["ids"], scale=c["scale"])}
        if c["sparse"]:
            ids, rows = ctx.embedding_backward_rows(s["d_y"], s["ids"], c["rows"], scale=c["scale"])
            return {"ids": ids, "rows": rows}
        return {"d_table": ctx.embedding_backward(s["d_y"], s["ids"], c["rows"], scale=c["scale"])}
    if c["op"] == "scores":
        if c["backward"]:
            return {"d_logits": ctx.log_probs_backward(s["logits"], s["lse"], s["labels"], s["d_log_prob"], entropy=s["entropy"] if c["regularised"] else None,
                                                       d_entropy=s["d_entropy"], d_lse=s["d_lse"], scale=c["scale"])}
        r = ctx.log_probs(s["logits"], s["labels"], top=c["top"], scale=c["scale"])
        out = {"log_prob": r.log_prob, "entropy": r.entropy, "lse": r.lse}
        if c["top"]:
            out["top_ids"], out["top_log_probs"] = r.top_ids, r.top_log_probs
        return out
    if c["backward"]:
        return {"d_logits": ctx.distill_backward(s["d_loss"], s["logits"], s["lse"], s["teacher_ids"], s["teacher_logits"], scale=c["scale"])}
    loss, lse = ctx.distill(s["logits"], s["teacher_ids"], s["teacher_logits"], scale=c["scale"])
    return {"loss": loss, "lse": lse}


def run(state):
    if own:
        return _run_own(state)
    c = state["case"]
    plain = {"lookup": (_lookup, _lookup_backward), "scores": (_scores, _scores_backward), "distill": (_distill, _distill_backward)}
    return plain[c["op"]][c["backward"]](state)


def work(case):
    """Each value read once and written once; of a table the rows that are named.  An exponential counts as one operation."""
    width = 4 if case["dtype"] == "f32" else 2
    n = case["n"]
    if case["op"] == "lookup":
        ids, moved, distinct = (8 if case["long_ids"] else 4), n * case["dim"] * width, _named(case)[1]
        if not case["backward"]:
            return {"bytes": n * ids + moved + distinct * case["dim"] * width, "flops": n * case["dim"]}
        made = distinct * (case["dim"] * width + ids) if case["sparse"] else case["rows"] * case["dim"] * width
        return {"bytes": n * ids + moved + made, "flops": 2 * n * case["dim"]}
    values = n * case["classes"]
    if case["op"] == "scores":
        if case["backward"]:
            return {"bytes": 2 * values * width + n * (8 + 4 + 4 + (12 if case["regularised"] else 0)), "flops": (8 if case["regularised"] else 4) * values}
        return {"bytes": values * width + n * (8 + 12 + 8 * case["top"]), "flops": 6 * values}
    if case["backward"]:
        return {"bytes": 2 * values * width + n * (8 + 8 * case["entries"]), "flops": 4 * values}
    return {"bytes": values * width + n * (8 + 8 * case["entries"]), "flops": 4 * values}


# ---- the definitions in 64 bits, apart from the forms above ---------------------------------------------------------
def _exact_lookup(case, s):
    ids = s["ids"].long()
    inside = ids.ge(0) & ids.lt(case["rows"])
    if not case["backward"]:
        y = torch.zeros(case["n"], case["dim"], dtype=torch.float64, device="cuda")
        y[inside] = s["table"].index_select(0, ids[inside]).double() * case["scale"]
        return {"y": y}
    # sums from differences of running ones, a few columns at a time
    distinct, counts = torch.unique(ids[inside], return_counts=True)
    at = torch.nonzero(inside)[:, 0]
    at = at[torch.argsort(ids[at], stable=True)]
    ends = counts.cumsum(0)
    sums = torch.empty(len(distinct), case["dim"], dtype=torch.float64, device="cuda")
    for lo in range(0, case["dim"], 64):
        run = s["d_y"][:, lo:lo + 64].index_select(0, at).double().cumsum(0)
        run = torch.cat([torch.zeros_like(run[:1]), run])
        sums[:, lo:lo + 64] = (run[ends] - run[ends - counts]) * case["scale"]
    if case["sparse"]:
        return {"ids": distinct.to(s["ids"].dtype), "rows": sums}
    out = torch.zeros(case["rows"], case["dim"], dtype=torch.float64, device="cuda")
    return {"d_table": out.index_copy_(0, distinct, sums)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "lookup":
        return _exact_lookup(case, s)
    x, scale, classes = s["logits"], case["scale"], case["classes"]
    parts = []
    step = max(1, (1 << 24) // classes)
    for lo in range(0, case["n"], step):
        at = slice(lo, lo + step)
        z = x[at].double() * scale
        lse = torch.logsumexp(z, 1)
        rows = torch.arange(z.shape[0], device="cuda")
        if case["op"] == "scores":
            label = s["labels"][at]
            has = label.ge(0) & label.lt(classes)
            if not case["backward"]:
                log_p = z - lse[:, None]
                r = {"log_prob": torch.zeros_like(lse), "entropy": torch.special.entr(log_p.exp()).sum(1), "lse": lse}
                r["log_prob"][has] = log_p[rows[has], label[has]]
                if case["top"]:      # by counting which of the two comes first, for the values that can be among the best
                    value, index = torch.topk(z, case["top"], dim=1)
                    least = value[:, -1:]
                    sure = z > least
                    order = torch.where(sure, z, torch.full_like(z, float("-inf")))
                    tied = (z == least) & ((z == least).cumsum(1) <= case["top"] - sure.sum(1, keepdim=True))
                    row, col = torch.nonzero(sure | tied, as_tuple=True)
                    col, val = col.view(-1, case["top"]), torch.where(sure, order, least)[row, col].view(-1, case["top"])
                    by = torch.argsort(val, dim=1, descending=True, stable=True)
                    r["top_ids"] = col.gather(1, by).int()
                    r["top_log_probs"] = val.gather(1, by) - lse[:, None]
            else:
                log_p = z - s["lse"][at].double()[:, None]
                weight = torch.where(has, -s["d_log_prob"][at].double(), 0.0)[:, None].expand_as(z).clone()
                if case["regularised"]:
                    weight += s["d_lse"][at].double()[:, None]
                    weight -= s["d_entropy"][at].double()[:, None] * (log_p.clamp(min=-1e4) + s["entropy"][at].double()[:, None])
                d = weight * log_p.exp()
                d[rows[has], label[has]] += s["d_log_prob"][at].double()[has]
                r = {"d_logits": d * scale}
        else:
            ids = s["teacher_ids"][at].long()
            there = ids.ge(0) & ids.lt(classes)
            v = torch.where(there, s["teacher_logits"][at].double() * scale, -math.inf)
            some = there.any(1)
            q = torch.zeros_like(v)
            q[some] = torch.softmax(v[some], 1)
            row, col = torch.nonzero(there, as_tuple=True)
            if not case["backward"]:
                log_p = z[row, ids[row, col]] - lse[row]
                r = {"loss": -torch.special.entr(q).sum(1).index_add(0, row, q[row, col] * log_p), "lse": lse}
            else:
                d = torch.exp(z - s["lse"][at].double()[:, None]) * some[:, None]
                d.index_put_((row, ids[row, col]), -q[row, col], accumulate=True)
                r = {"d_logits": d * (s["d_loss"][at].double() * scale)[:, None]}
        parts.append(r)
    return {key: torch.cat([p[key] for p in parts]) for key in parts[0]}
