"""What lies between two layers of a model, as cases that can be timed: dropout whose mask comes from a counter-based generator and is
never stored, and group norm with an activation over rows whose channels lie last, with both their gradients and the two fused.

A case is a `dropout`, or a `norm` that may have a dropout behind its activation; `backward` asks for the gradients.
  rows x channels   the matrix: a row is a node of a layer's output
  samples           what shares its statistics: every row by itself ("rows"), mini-batches of uneven sizes that lie one behind the other
                    ("ragged": one of them empty where there are four or more, and `behind` rows behind the last), or equal ones ("equal")
  pad               columns between two rows that belong to somebody else
  keyed             the dropout's mask goes by a key of each row (a node's id, and its mini-batch above it), not by the row's place
Dropout: element c of a row with key r is kept where the 16-bit half c % 8 (low half first) of the Philox4x32-10 block with counter
(r, r >> 32, c / 8, 0x64720000 + site) under the key (seed, seed >> 32) is at least t = round(65536 p); what is kept is scaled by
65536 / (65536 - t), what is dropped is zero.
"""
import math

import numpy as np
import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_EPS = 1e-5


# ---- the cases ------------------------------------------------------------------------------------------------------
def _case(name, op, **sizes):
    c = {"op": op, "backward": False, "dtype": "f32", "rows": 1000, "channels": 128, "groups": 1, "samples": "rows", "count": 1, "behind": 0,
         "act": "none", "p": 0.0, "site": 0, "keyed": False, "pad": 0}
    c.update(sizes)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # the inputs of a first try's model, 512 targets of 16 columns: launches and waits
        _case("dropout_tiny", "dropout", rows=512, channels=16, p=0.5),
        # the first layer's outputs of 24 mini-batches of 1,000 targets on a graph of two million nodes
        _case("dropout_layer", "dropout", rows=543_000, channels=256, p=0.5, site=1),
        # its gradient, the mask by node, in the type that a half-precision table has, rows as wide as that table's
        _case("dropout_wide_half_backward", "dropout", backward=True, dtype="f16", rows=150_001, channels=768, p=0.3, keyed=True),
        # an odd width, rows that start anywhere
        _case("dropout_odd", "dropout", dtype="bf16", rows=77_777, channels=101, p=0.1, site=2, pad=2),
        # answering for a few users at once: three mini-batches of some 137 rows, one layer's norm over each
        _case("norm_serving", "norm", rows=411, channels=100, groups=4, samples="ragged", count=3, act="relu"),
        # every node by itself, as layers of this kind are most often normalised: 128 mini-batches' last layer but one
        _case("norm_nodes", "norm", rows=768_000, channels=256, act="relu", p=0.5, site=1),
        # and its gradient
        _case("norm_nodes_backward", "norm", backward=True, rows=543_000, channels=256, act="relu", p=0.5, site=1),
        # statistics over a mini-batch: 24 of them, some 22,600 rows each
        _case("norm_mini_batches", "norm", rows=543_000, channels=256, groups=8, samples="ragged", count=24, act="relu", p=0.5, site=1, behind=5),
        # the gradient of the same with a smooth activation, the mask by node
        _case("norm_mini_batches_backward", "norm", backward=True, rows=543_000, channels=256, groups=8, samples="ragged", count=24, act="gelu",
              p=0.5, site=1, keyed=True),
        # one mini-batch's second layer in a training step's backward pass: latency
        _case("norm_one_mini_batch_backward", "norm", backward=True, rows=6_000, channels=128, groups=8, samples="ragged", count=1, act="silu"),
        # feature maps with their channels last, the operator's usual place
        _case("norm_maps_half", "norm", dtype="f16", rows=16 * 4096, channels=512, groups=32, samples="equal", count=16, act="silu"),
        # a whole graph in one piece: two million nodes share their statistics
        _case("norm_whole_graph_backward", "norm", backward=True, rows=2_000_003, channels=128, groups=2, samples="ragged", count=1, act="silu", p=0.2),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(("dropout", "norm", "norm"))
    backward = rng.random() < 0.5
    channels = rng.choice((16, 64, 100, 101, 128, 128, 192, 256, 256, 320, 512, 602, 768, 1024))
    most = 250_000_000 if op == "norm" and backward else 139_000_000     # values in all: less than the largest listed case of the kind
    rows = log_int(1, min(2_000_000, most // channels))
    c = _case("", op, backward=backward, dtype=rng.choice(("f32", "f32", "f16", "bf16")), rows=rows, channels=channels,
              p=rng.choice((0.1, 0.2, 0.5, rng.uniform(0.01, 0.9))), site=rng.randint(0, 7), keyed=rng.random() < 0.3, pad=rng.choice((0, 0, 0, 4, 8, 3)))
    if op == "norm":
        c["samples"] = rng.choice(("rows", "ragged", "ragged", "equal"))
        c["groups"] = rng.choice([g for g in (1, 1, 2, 4, 8, 16, 32) if channels % g == 0 and channels // g >= 8])
        c["act"] = rng.choice(("none", "relu", "silu", "gelu"))
        if rng.random() < 0.4:
            c["p"], c["keyed"] = 0.0, False
        if c["samples"] != "rows":
            c["count"] = min(rows, log_int(1, 128))
        if c["samples"] == "equal":
            c["rows"] -= rows % c["count"]
            c["pad"] = 0
        if c["samples"] == "ragged" and rows > 20:
            c["behind"] = rng.choice((0, 0, 7))
    return c


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _offsets(case, seed):
    """First rows of the samples and the end of the last, or None where every row is one."""
    n, used = case["count"], case["rows"] - case["behind"]
    if case["samples"] == "rows":
        return None
    if case["samples"] == "equal":
        return torch.arange(n + 1, dtype=torch.int64) * (used // n)
    w = 0.5 + torch.rand(n, generator=torch.Generator().manual_seed(seed))
    if n >= 4:
        w[n // 2] = 0.0
    ends = (torch.cumsum(w.double(), 0) / w.double().sum() * used).round().long()
    ends[-1] = used
    return torch.cat([torch.zeros(1, dtype=torch.int64), ends])


def _strided(values, pad):
    """The same values with `pad` columns of another's between the rows."""
    if pad == 0:
        return values
    wide = torch.full((values.shape[0], values.shape[1] + pad), float("nan"), dtype=values.dtype, device=values.device)
    wide[:, :values.shape[1]] = values
    return wide[:, :values.shape[1]]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, ch, dtype = case["rows"], case["channels"], _TYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    # a layer's outputs before its activation: columns of their own scale, about a bias of their own
    centre, scale = 0.4 + 0.5 * normal(ch), 0.5 + normal(ch).abs()
    s = {"case": dict(case), "x": _strided((normal(n, ch) * scale + centre).to(dtype), case["pad"])}
    offsets = _offsets(case, seed)
    s["offsets"] = offsets
    s["drop"] = None
    if case["p"] > 0:
        keys = None
        if case["keyed"]:      # mini-batches of nodes, any ids in them
            ids = torch.randint(0, 111_000_000, (n,), generator=g, device="cuda")
            keys = (torch.arange(n, device="cuda") // 22_600 << 32) + ids
        s["drop"] = {"p": case["p"], "seed": (seed * 0x9E3779B97F4A7C15 + 12345) % 2**64, "site": case["site"], "row_keys": keys}
    if case["op"] == "norm":
        s["weight"], s["bias"] = 1 + 0.2 * normal(ch), 0.2 * normal(ch)
    if case["backward"]:
        s["d_y"] = _strided(normal(n, ch).to(dtype), case["pad"])
        if case["op"] == "norm":      # what the forward pass left
            s["mean"], s["rstd"] = (t.float() for t in _statistics(s["x"], case["groups"], offsets, torch.float64))
    return s


# ---- the operators' plain forms -------------------------------------------------------------------------------------
def _philox(c0, c1, c2, c3, k0, k1):
    """Philox4x32-10 on tensors of 64-bit integers that hold 32 bits each."""
    low = 0xFFFFFFFF
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return c0, c1, c2, c3


def _kept(drop, rows, channels):
    """Which elements stay, and the factor of those that do."""
    t = round(drop["p"] * 65536)
    key = drop["row_keys"] if drop["row_keys"] is not None else torch.arange(rows, device="cuda")
    block = torch.arange((channels + 7) // 8, device="cuda")[None, :]
    zero = torch.zeros_like(block)
    words = _philox((key & 0xFFFFFFFF)[:, None] + zero, ((key >> 32) & 0xFFFFFFFF)[:, None] + zero, block + (key * 0)[:, None],
                    torch.full_like(block, 0x64720000 + drop["site"]) + (key * 0)[:, None], drop["seed"] & 0xFFFFFFFF, drop["seed"] >> 32)
    halves = torch.stack([h >= t for w in words for h in (w & 0xFFFF, w >> 16)], dim=2)
    return halves.reshape(rows, -1)[:, :channels], 65536.0 / (65536 - t) if t < 65536 else 0.0


def _dropped(v, drop):
    keep, factor = _kept(drop, *v.shape)
    return torch.where(keep, v * factor, torch.zeros((), dtype=v.dtype, device=v.device))


def _per_sample(by_row, offsets):
    """Sums over each sample's rows, in 64 bits: differences of running sums."""
    run = torch.cumsum(by_row.t().double().contiguous(), 1)      # (down the columns as they lie, the whole pass takes 213 ms in place of 15)
    run = torch.cat([torch.zeros_like(run[:, :1]), run], 1)
    at = offsets.cuda()
    return (run[:, at[1:]] - run[:, at[:-1]]).t()


def _statistics(x, groups, offsets, dtype):
    """Mean and reciprocal deviation of every (sample, group); zero where a sample has no rows."""
    v = x.to(dtype)
    v = v.reshape(v.shape[0], groups, -1)
    if offsets is None:
        mean = v.mean(2)
        return mean, 1 / torch.sqrt((v - mean[:, :, None]).square().mean(2) + _EPS)
    length = offsets.diff().cuda()
    n = (length * v.shape[2]).clamp(min=1)[:, None]
    mean = (_per_sample(v.sum(2), offsets) / n).to(dtype)
    sample = torch.repeat_interleave(torch.arange(len(length), device="cuda"), length)
    used = int(offsets[-1])
    var = _per_sample((v[:used] - mean[sample][:, :, None]).square().sum(2), offsets) / n
    rstd = torch.where(length[:, None] > 0, 1 / torch.sqrt(var + _EPS), torch.zeros_like(var))
    return mean, rstd.to(dtype)


def _by_row(t, offsets):
    """A value of each (sample, group) for every row of the samples."""
    if offsets is None:
        return t[:, :, None]
    return torch.repeat_interleave(t, offsets.diff().cuda(), dim=0)[:, :, None]


def _act(n, kind):
    if kind == "relu":
        return torch.where(n < 0, torch.zeros_like(n), n)
    if kind == "silu":
        return n / (1 + torch.exp(-n))
    if kind == "gelu":
        return 0.5 * n * (1 + torch.erf(n * math.sqrt(0.5)))
    return n


def _act_slope(n, kind):
    if kind == "silu":
        s = 1 / (1 + torch.exp(-n))
        return s * (1 + n * (1 - s))
    if kind == "gelu":
        return 0.5 * (1 + torch.erf(n * math.sqrt(0.5))) + n * torch.exp(-0.5 * n * n) * (1 / math.sqrt(2 * math.pi))
    return torch.ones_like(n)


def _norm(s):
    c, x, offsets, groups = s["case"], s["x"], s["offsets"], s["case"]["groups"]
    mean, rstd = _statistics(x, groups, offsets, torch.float32)
    used = c["rows"] - c["behind"]
    v = x[:used].float().reshape(used, groups, -1)
    hat = ((v - _by_row(mean, offsets)) * _by_row(rstd, offsets)).reshape(used, -1)
    y = _act(hat * s["weight"] + s["bias"], c["act"])
    if s["drop"]:
        y = _dropped(torch.cat([y, y.new_zeros(c["behind"], y.shape[1])]), s["drop"])[:used]
    out = torch.zeros(x.shape, dtype=x.dtype, device=x.device)
    out[:used] = y.to(x.dtype)
    return {"y": out, "mean": mean, "rstd": rstd}


def _norm_backward(s):
    c, offsets, groups = s["case"], s["offsets"], s["case"]["groups"]
    used = c["rows"] - c["behind"]
    g = s["d_y"].float()
    if s["drop"]:
        g = _dropped(g, s["drop"])
    g, v = g[:used], s["x"][:used].float().reshape(used, groups, -1)
    mean, rstd = _by_row(s["mean"], offsets), _by_row(s["rstd"], offsets)
    hat = ((v - mean) * rstd).reshape(used, -1)
    if c["act"] == "relu":      # which side of zero a value lies on is seen in 64 bits
        at = ((v.double() - mean) * rstd).reshape(used, -1) * s["weight"] + s["bias"]
        g = torch.where(at <= 0, torch.zeros_like(g), g)
    else:
        g = g * _act_slope(hat * s["weight"] + s["bias"], c["act"])
    d_weight, d_bias = (g * hat).sum(0, dtype=torch.float64).float(), g.sum(0, dtype=torch.float64).float()
    g, hat = (g * s["weight"]).reshape(used, groups, -1), hat.reshape(used, groups, -1)
    if offsets is None:
        a, b = g.mean(2, keepdim=True), (g * hat).mean(2, keepdim=True)
    else:
        n = (offsets.diff().cuda() * g.shape[2]).clamp(min=1)[:, None]
        a = _by_row((_per_sample(g.sum(2), offsets) / n).float(), offsets)
        b = _by_row((_per_sample((g * hat).sum(2), offsets) / n).float(), offsets)
    out = torch.zeros(s["x"].shape, dtype=s["x"].dtype, device="cuda")
    out[:used] = (rstd * (g - a - hat * b)).reshape(used, -1).to(out.dtype)
    return {"d_x": out, "d_weight": d_weight, "d_bias": d_bias}


# ---- the same through the package -----------------------------------------------------------------------------------
_kept_context = []


def _context():
    """The program's one context on the GPU."""
    import paper_2202_02365_b200 as mg
    if not _kept_context:
        _kept_context.append(mg.Context(0))
    return mg, _kept_context[0]


def _run_own(s):
    mg, ctx = _context()
    c = s["case"]
    drop = mg.Dropout(**s["drop"]) if s["drop"] else None
    if c["op"] == "dropout":
        if c["backward"]:
            return {"d_x": ctx.dropout_backward(s["d_y"], drop)}
        return {"y": ctx.dropout(s["x"], drop)}
    if c["samples"] == "equal":      # [samples, places, channels]
        shape = (c["count"], c["rows"] // c["count"], c["channels"])
        x, offsets = s["x"].view(shape), None
    else:
        x, offsets = s["x"], s["offsets"]
    how = dict(groups=c["groups"], weight=s["weight"], bias=s["bias"], sample_offsets=offsets, activation=c["act"], dropout=drop)
    if c["backward"]:
        d_x, d_weight, d_bias = ctx.group_norm_backward(s["d_y"].view(x.shape), x, s["mean"], s["rstd"], **how)
        return {"d_x": d_x.view(s["x"].shape), "d_weight": d_weight, "d_bias": d_bias}
    y, mean, rstd = ctx.group_norm(x, eps=_EPS, **how)
    return {"y": y.view(s["x"].shape), "mean": mean, "rstd": rstd}


def run(state):
    if own:
        return _run_own(state)
    c = state["case"]
    if c["op"] == "norm":
        return _norm_backward(state) if c["backward"] else _norm(state)
    given = state["d_y"] if c["backward"] else state["x"]
    return {"d_x" if c["backward"] else "y": _dropped(given.float(), state["drop"]).to(given.dtype)}


def work(case):
    """Each value read once and written once; a block of the generator counts as its 20 products, 20 pairs of exclusive ors and 20 sums for
    eight elements, a normalised value as about ten operations, its gradient as about twenty."""
    width = 4 if case["dtype"] == "f32" else 2
    values, used = case["rows"] * case["channels"], (case["rows"] - case["behind"]) * case["channels"]
    drop = 10.0 if case["p"] > 0 else 0.0
    keys = 8 * case["rows"] if case["keyed"] else 0
    if case["op"] == "dropout":
        return {"bytes": 2 * width * values + keys, "flops": drop * values}
    statistics = 8 * case["groups"] * (case["rows"] if case["samples"] == "rows" else case["count"])
    if case["backward"]:
        return {"bytes": 3 * width * used + keys + statistics + 16 * case["channels"], "flops": (drop + 20.0) * used}
    return {"bytes": 2 * width * used + keys + statistics + 8 * case["channels"], "flops": (drop + 10.0) * used}


# ---- the definitions in 64 bits, apart from the forms above ---------------------------------------------------------
def _exact_kept(case, drop):
    """The mask, from a generator on the host in whole numbers of 64 bits without sign."""
    n, blocks = case["rows"], -(-case["channels"] // 8)
    keys = np.arange(n, dtype=np.uint64) if drop["row_keys"] is None else drop["row_keys"].cpu().numpy().astype(np.uint64)
    low, shift = np.uint64(0xFFFFFFFF), np.uint64(32)
    kept = np.empty((n, blocks * 8), dtype=bool)
    limit = np.uint16(min(round(drop["p"] * 65536), 65535))
    for lo in range(0, n, 1 << 16):
        k = keys[lo:lo + (1 << 16)]
        word = [np.repeat((k & low)[:, None], blocks, 1), np.repeat((k >> shift)[:, None], blocks, 1),
                np.repeat(np.arange(blocks, dtype=np.uint64)[None, :], len(k), 0), np.full((len(k), blocks), 0x64720000 + case["site"], dtype=np.uint64)]
        key = [drop["seed"] % 2**32, drop["seed"] // 2**32]
        for _ in range(10):
            first, second = word[0] * np.uint64(0xD2511F53), word[2] * np.uint64(0xCD9E8D57)
            word = [(second >> shift) ^ word[1] ^ np.uint64(key[0]), second & low, (first >> shift) ^ word[3] ^ np.uint64(key[1]), first & low]
            key = [(key[0] + 0x9E3779B9) % 2**32, (key[1] + 0xBB67AE85) % 2**32]
        bits = np.stack(word, axis=2).astype("<u4").reshape(len(k), -1).view("<u2")      # low halves first
        kept[lo:lo + len(k)] = bits >= limit
    return torch.from_numpy(kept[:, :case["channels"]]).cuda()


def _moments(part, groups):
    """Mean, and mean square about it, of each group of one sample's rows."""
    per = part.reshape(part.shape[0], groups, -1)
    var, mean = torch.var_mean(per, dim=(0, 2), correction=0)
    return mean, var


def exact(case, seed):
    s = prepare(case, seed)
    drop, groups, used = s["drop"], case["groups"], case["rows"] - case["behind"]
    given = (s["d_y"] if case["backward"] else s["x"]).double()
    keep = _exact_kept(case, drop) if drop else None
    factor = 1 / (1 - round(drop["p"] * 65536) / 65536) if drop else 1.0
    if case["op"] == "dropout":
        return {"d_x" if case["backward"] else "y": (given * factor).masked_fill_(~keep, 0.0)}
    weight, bias = s["weight"].double(), s["bias"].double()
    each = case["channels"] // groups
    out = torch.zeros(case["rows"], case["channels"], dtype=torch.float64, device="cuda")
    if s["offsets"] is None:
        spans = [(lo, min(lo + 65536, used)) for lo in range(0, used, 65536)]
    else:
        spans = list(zip(s["offsets"][:-1].tolist(), s["offsets"][1:].tolist()))
    means, rstds = [], []
    d_weight, d_bias = torch.zeros_like(weight), torch.zeros_like(bias)
    for i, (lo, hi) in enumerate(spans):
        x = s["x"][lo:hi].double()
        if case["backward"]:
            at = slice(lo, hi) if s["offsets"] is None else slice(i, i + 1)
            mean, rstd = s["mean"][at].double(), s["rstd"][at].double()
        elif hi == lo:
            mean = rstd = torch.zeros(1, groups, dtype=torch.float64, device="cuda")
        elif s["offsets"] is None:
            var, mean = torch.var_mean(x.reshape(hi - lo, groups, each), dim=2, correction=0)
            rstd = (var + _EPS).rsqrt()
        else:
            mean, var = _moments(x, groups)
            mean, rstd = mean[None], (var + _EPS).rsqrt()[None]
        means.append(mean)
        rstds.append(rstd)
        if hi == lo:
            continue
        hat = (x - mean.repeat_interleave(each, 1)) * rstd.repeat_interleave(each, 1)
        n = torch.addcmul(bias, hat, weight)
        if not case["backward"]:
            y = {"none": lambda v: v, "relu": torch.relu, "silu": lambda v: v * torch.sigmoid(v),
                 "gelu": lambda v: v * 0.5 * torch.erfc(-v / math.sqrt(2))}[case["act"]](n)
            out[lo:hi] = y if keep is None else (y * factor).masked_fill_(~keep[lo:hi], 0.0)
            continue
        slope = {"none": torch.ones_like, "relu": lambda v: (v > 0).double(), "silu": lambda v: torch.sigmoid(v) * (1 + v * torch.sigmoid(-v)),
                 "gelu": lambda v: 0.5 * torch.erfc(-v / math.sqrt(2)) + v * torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)}[case["act"]](n)
        d = given[lo:hi] * slope
        if keep is not None:
            d = (d * factor).masked_fill_(~keep[lo:hi], 0.0)
        d_weight += (d * hat).sum(0)
        d_bias += d.sum(0)
        d, h = (d * weight).reshape(hi - lo, groups, each), hat.reshape(hi - lo, groups, each)
        over = (2,) if s["offsets"] is None else (0, 2)
        d = d - d.mean(over, keepdim=True) - h * (d * h).mean(over, keepdim=True)
        out[lo:hi] = d.reshape(hi - lo, -1) * rstd.repeat_interleave(each, 1)
    if case["backward"]:
        return {"d_x": out, "d_weight": d_weight, "d_bias": d_bias}
    return {"y": out, "mean": torch.cat(means), "rstd": torch.cat(rstds)}
