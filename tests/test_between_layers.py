"""Dropout and group norm against their definitions in 64 bits, at the sizes, strides, types and samples where their kernels are cut
differently, and in the ways a program may call them.

Tolerances.  u = 2^-24 is half a step of fp32, h half a step of the row type (0 for fp32, whose roundings are counted with the others).  A sum
of n values is off by at most (chain) u times the sum of their magnitudes, the chain being the number of additions that one value goes
through: below n / 64 + 64 in every kernel here.  The other counts stand beside the formulas."""
import math
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

import paper_2202_02365_b200 as mg
from oracle import dense_oracle
from paper_2202_02365_b200 import build

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ACTS = ("none", "relu", "silu", "gelu")


def half_step(dtype):
    return 0.0 if dtype == torch.float32 else torch.finfo(dtype).eps / 2


def smallest(dtype):      # half the distance of subnormal numbers
    return {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}[dtype]


# ---- definitions ----------------------------------------------------------------------------------------------------
def kept(keys, channels, p, seed, site):
    """The mask, from the rounds of Philox4x32-10 on arrays of whole numbers."""
    low, shift = np.uint64(0xFFFFFFFF), np.uint64(32)
    blocks = -(-channels // 8)
    keys = np.asarray(keys).astype(np.uint64)[:, None]
    c = [np.broadcast_to(keys & low, (len(keys), blocks)), np.broadcast_to(keys >> shift, (len(keys), blocks)),
         np.broadcast_to(np.arange(blocks, dtype=np.uint64), (len(keys), blocks)), np.full((len(keys), blocks), 0x64720000 + site, dtype=np.uint64)]
    k0, k1 = seed % 2**32, seed >> 32
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> shift) ^ c[1] ^ np.uint64(k0), b & low, (a >> shift) ^ c[3] ^ np.uint64(k1), a & low]
        k0, k1 = (k0 + 0x9E3779B9) % 2**32, (k1 + 0xBB67AE85) % 2**32
    halves = np.stack([h for w in c for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], axis=2).reshape(len(keys), -1)[:, :channels]
    return torch.from_numpy(halves >= np.uint64(round(p * 65536)))


def factor(p):
    t = round(p * 65536)
    return 65536 / (65536 - t) if t < 65536 else 0.0


def act(n, kind):
    return {"none": lambda: n, "relu": lambda: torch.relu(n), "silu": lambda: n * torch.sigmoid(n),
            "gelu": lambda: n * 0.5 * torch.erfc(-n / math.sqrt(2))}[kind]()


def slope(n, kind):
    return {"none": lambda: torch.ones_like(n), "relu": lambda: (n > 0).double(), "silu": lambda: torch.sigmoid(n) * (1 + n * torch.sigmoid(-n)),
            "gelu": lambda: 0.5 * torch.erfc(-n / math.sqrt(2)) + n * torch.exp(-n * n / 2) / math.sqrt(2 * math.pi)}[kind]()


def over(t, spans, groups):
    """Sum of each (sample, group), and the same for every element."""
    out = torch.zeros(len(spans), groups, dtype=torch.float64, device=t.device)
    for i, (lo, hi) in enumerate(spans):
        out[i] = t[lo:hi].reshape(hi - lo, groups, t.shape[1] // groups).sum((0, 2))
    return out


def spread(t, spans, groups, channels):
    rows = [t[i:i + 1].expand(hi - lo, groups) for i, (lo, hi) in enumerate(spans)]
    return torch.cat(rows).repeat_interleave(channels // groups, 1)


def counts(spans, groups, channels, device):
    return torch.tensor([[max(1, (hi - lo) * (channels // groups))] for lo, hi in spans], dtype=torch.float64, device=device)


def norm(x, spans, groups, w, b, eps, kind, keep=None, f=1.0):
    x, n = x.double(), counts(spans, groups, x.shape[1], x.device)
    mean = over(x, spans, groups) / n
    centred = x - spread(mean, spans, groups, x.shape[1])
    var = over(centred.square(), spans, groups) / n
    rstd = (var + eps).rsqrt()
    for i, (lo, hi) in enumerate(spans):
        if lo == hi:
            rstd[i] = 0.0
    hat = centred * spread(rstd, spans, groups, x.shape[1])
    y = act(hat * w + b, kind)
    if keep is not None:
        y = torch.where(keep, y * f, torch.zeros_like(y))
    return y, mean, rstd, hat


def norm_backward(d_y, x, mean, rstd, spans, groups, w, b, kind, keep=None, f=1.0):
    x, d, n = x.double(), d_y.double(), counts(spans, groups, x.shape[1], x.device)
    r = spread(rstd.double(), spans, groups, x.shape[1])
    hat = (x - spread(mean.double(), spans, groups, x.shape[1])) * r
    if keep is not None:
        d = torch.where(keep, d * f, torch.zeros_like(d))
    d = d * slope(hat * w + b, kind)
    g = d * w
    s1, s2 = over(g, spans, groups) / n, over(g * hat, spans, groups) / n
    d_x = r * (g - spread(s1, spans, groups, x.shape[1]) - hat * spread(s2, spans, groups, x.shape[1]))
    return d_x, (d * hat).sum(0), d.sum(0), hat


# ---- the definitions themselves -------------------------------------------------------------------------------------
def test_the_mask_is_the_generators():
    keys = [0, 5, 2**32 + 7, 2**63 - 1]
    got = kept(keys, 21, 0.3, 0x123456789ABCDEF0, 9)
    for i, key in enumerate(keys):
        for c in range(21):
            block = dense_oracle.philox4x32_10((key % 2**32, key >> 32, c // 8, 0x64720009), (0x9ABCDEF0, 0x12345678))
            half = int(block[c % 8 // 2]) >> (16 * (c % 2)) & 0xFFFF
            assert bool(got[i, c]) == (half >= round(0.3 * 65536))


@pytest.mark.parametrize("kind", ACTS)
def test_the_gradient_is_the_forward_formulas(kind):
    g = torch.Generator().manual_seed(1)
    x, d_y = (torch.randn(9, 12, generator=g, dtype=torch.float64) for _ in range(2))
    w, b = (torch.randn(12, generator=g, dtype=torch.float64) for _ in range(2))
    spans = [(0, 4), (4, 4), (4, 5), (5, 9)]
    keep = kept(range(9), 12, 0.25, 7, 0)

    def value(x, w, b):
        return float((norm(x, spans, 3, w, b, 1e-3, kind, keep, factor(0.25))[0] * d_y).sum())
    _, mean, rstd, _ = norm(x, spans, 3, w, b, 1e-3, kind)
    grads = norm_backward(d_y, x, mean, rstd, spans, 3, w, b, kind, keep, factor(0.25))[:3]
    # central differences: off by the third derivative times h^2 / 6 and by roundings over h; values here are of order one to a hundred
    h = 1e-5
    for t, grad in zip((x, w, b), grads):
        for at in range(t.numel()):
            flat, was = t.view(-1), t.view(-1)[at].item()
            flat[at] = was + h
            up = value(x, w, b)
            flat[at] = was - h
            down = value(x, w, b)
            flat[at] = was
            assert abs((up - down) / (2 * h) - float(grad.reshape(-1)[at])) < 1e-5


# ---- inputs ---------------------------------------------------------------------------------------------------------
def rows_of(rows, channels, dtype, seed, pad=0, shift=0, centre=0.5):
    """Normal values; `pad` columns of NaN between the rows, the first row `shift` elements behind an allocation's start."""
    g = torch.Generator().manual_seed(seed)
    v = (torch.randn(rows, channels, generator=g) * (0.5 + torch.rand(channels, generator=g)) + centre).to(dtype)
    flat = torch.full((shift + rows * (channels + pad) + 8,), float("nan"), dtype=dtype, device="cuda")
    at = flat[shift:shift + rows * (channels + pad)].view(rows, channels + pad)[:, :channels]
    at.copy_(v)
    return at


def spans_of(samples, rows):
    if samples == "rows":
        return [(i, i + 1) for i in range(rows)], None
    ends = np.cumsum([0] + list(samples)).tolist()
    return list(zip(ends[:-1], ends[1:])), ends


@pytest.fixture(scope="module")
def ctx():
    return mg.Context(0)


def check_dropout(got, x, keep, p):
    # the factor's rounding, the product's, and the one to the row type
    want = torch.where(keep.cuda(), x.double() * factor(p), torch.zeros((), dtype=torch.float64, device="cuda"))
    assert torch.equal(got[~keep.cuda()], torch.zeros_like(got[~keep.cuda()]))
    h = half_step(got.dtype)
    assert bool(((got.double() - want).abs() <= (2.01 * U + h * (1 + 3 * U)) * want.abs() + smallest(got.dtype)).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,channels,pad,shift", [(1, 1, 0, 0), (3, 7, 0, 0), (512, 16, 0, 0), (1000, 100, 0, 0), (77, 101, 3, 1), (300, 768, 8, 0), (130, 128, 2, 0),
                                                     (5, 2001, 0, 3), (20_011, 64, 0, 0), (33, 8, 0, 2), (70, 602, 0, 0), (41, 4, 4, 4)])
def test_dropout(ctx, dtype, rows, channels, pad, shift):
    x = rows_of(rows, channels, TYPES[dtype], 3, pad, shift)
    for p, keyed in ((0.5, False), (0.1, True), (0.99, False)):
        keys = torch.randint(0, 2**62, (rows,)) if keyed else torch.arange(rows) + 5
        drop = mg.Dropout(p, seed=2**64 - 3, site=65535, first_row=5, row_keys=keys.cuda() if keyed else None)
        y = ctx.dropout(x, drop)
        keep = kept(keys.numpy(), channels, p, 2**64 - 3, 65535)
        check_dropout(y, x, keep, p)
        assert torch.equal(y, ctx.dropout_backward(x, drop))


@pytest.mark.gpu
def test_dropout_at_its_ends(ctx):
    x = rows_of(100, 64, torch.float32, 1)
    x[3, 5], x[7, 9] = float("inf"), float("nan")
    for p in (0.0, 2.0 ** -18):
        assert torch.equal(ctx.dropout(x, mg.Dropout(p, 1)).nan_to_num(9), x.nan_to_num(9))
    assert not ctx.dropout(x, mg.Dropout(1.0, 1)).any()
    keep = kept(range(100), 64, 0.5, 1, 0).cuda()
    y = ctx.dropout(x, mg.Dropout(0.5, 1))
    assert not y[~keep].any() and bool(torch.isfinite(y[keep]).all()) == bool(torch.isfinite(x[keep]).all())


@pytest.mark.gpu
def test_dropout_cut_into_calls_and_written_in_place(ctx):
    x = rows_of(997, 100, torch.float16, 2)
    whole = ctx.dropout(x, mg.Dropout(0.3, 11, site=2))
    for lo, hi in ((0, 1), (1, 500), (500, 997)):
        assert torch.equal(ctx.dropout(x[lo:hi], mg.Dropout(0.3, 11, site=2, first_row=lo)), whole[lo:hi])
    wide = torch.zeros((997, 300), dtype=torch.float16, device="cuda")
    wide[:, :100] = x
    ctx.dropout(wide[:, :100], mg.Dropout(0.3, 11, site=2), out=wide[:, 200:])      # between the input's rows
    assert torch.equal(wide[:, 200:], whole) and torch.equal(wide[:, :100], x) and not wide[:, 100:200].any()
    ctx.dropout(x, mg.Dropout(0.3, 11, site=2), out=x)
    assert torch.equal(x, whole)
    same = torch.ones(1, 64, device="cuda").expand(50, 64)                           # one row over and over
    check_dropout(ctx.dropout(same, mg.Dropout(0.5, 3)), same, kept(range(50), 64, 0.5, 3, 0), 0.5)
    maps = torch.randn(3, 5, 7, 24, device="cuda")
    assert torch.equal(ctx.dropout(maps, mg.Dropout(0.5, 3)).view(-1, 24), ctx.dropout(maps.view(-1, 24), mg.Dropout(0.5, 3)))
    assert ctx.dropout(torch.empty((0, 8), device="cuda"), mg.Dropout(0.5, 3)).shape == (0, 8)


# ---- group norm -----------------------------------------------------------------------------------------------------
def check_norm(ctx, x, samples, groups, kind, drop=None, affine=True, eps=1e-5, out=None):
    rows, channels = x.shape
    spans, ends = spans_of(samples, rows)
    used = spans[-1][1] if spans else 0
    g = torch.Generator().manual_seed(5)
    w = (1 + 0.3 * torch.randn(channels, generator=g)).cuda() if affine else None
    b = (0.3 * torch.randn(channels, generator=g)).cuda() if affine else None
    dw, db = (w.double(), b.double()) if affine else (torch.ones(channels, dtype=torch.float64, device="cuda"), torch.zeros(channels, dtype=torch.float64, device="cuda"))
    keep, f = None, 1.0
    if drop is not None:
        keys = drop.row_keys.cpu().numpy() if drop.row_keys is not None else np.arange(rows) + drop.first_row
        keep, f = kept(keys, channels, drop.p, drop.seed, drop.site)[:used].cuda(), factor(drop.p)
    how = dict(weight=w, bias=b, sample_offsets=ends, activation=kind, dropout=drop)
    y, mean, rstd = ctx.group_norm(x, groups, eps=eps, out=out, **how)
    want, wmean, wrstd, hat = norm(x[:used], spans, groups, dw, db, eps, kind, keep, f)
    n, h = counts(spans, groups, channels, "cuda"), half_step(x.dtype)
    size = over(x[:used].double().abs(), spans, groups) / n
    chain = n / 64 + 64
    # the mean: its sum and the division.  The deviation: the squares' sum, the centring's (the mean's error enters squared: the centred values
    # sum to nothing) and five roundings more; a power of -1/2 halves it, and rsqrtf is off by two units at most
    t_mean = (chain + 2) * U * size
    # (where the variance is about the square of the mean's error or below, that square counts whole)
    t_rstd = wrstd * ((chain + 8) * U + 4 * U) + 0.5 * wrstd ** 3 * t_mean ** 2
    assert bool(((mean.double() - wmean).abs() <= t_mean + 1e-45).all())
    assert bool(((rstd.double() - wrstd).abs() <= t_rstd).all())
    # n = hat w + b: the mean's error and the deviation's, three roundings of the product, one of the sum; the activation's slope is below 1.13 and
    # its own value is off by at most 8 units of |n| (exp and erf by two each); the dropout's two roundings; the one to the row type
    C = channels
    t_n = dw.abs() * (spread(t_mean * wrstd, spans, groups, C) + hat.abs() * (spread(t_rstd / wrstd.clamp(min=1e-300), spans, groups, C) + 3 * U)) + 2 * U * ((hat * dw).abs() + db.abs())
    t_y = f * (1.13 * t_n + 8 * U * (hat * dw + db).abs()) + (2 * U + h) * want.abs() + h * f * t_n + smallest(x.dtype)
    if keep is not None:
        assert not y[:used][~keep].any()
        t_y = torch.where(keep, t_y, torch.zeros_like(t_y))
    assert bool(((y[:used].double() - want).abs() <= t_y).all()), float(((y[:used].double() - want).abs() / t_y).max())
    if out is None:
        assert not y[used:].any()

    d_y = rows_of(rows, channels, x.dtype, 8, centre=0.1)
    d_x, d_w, d_b = ctx.group_norm_backward(d_y, x, mean, rstd, groups, **how)
    wdx, wdw, wdb, hat = norm_backward(d_y[:used], x[:used], mean, rstd, spans, groups, dw, db, kind, keep, f)
    r = spread(rstd.double(), spans, groups, C)
    k = torch.ones_like(hat) if keep is None else keep.double()
    # dz = d_y f slope: two roundings of the product, the slope's own ten units and what n's roundings move it by (its own slope is below 0.8)
    z = k * d_y[:used].double().abs() * f * 1.13
    t_n = 3 * U * (hat * dw).abs() + 2 * U * ((hat * dw).abs() + db.abs())
    t_z = z * (14 * U + (0.0 if kind in ("none", "relu") else 1.0) * t_n)
    gz, t_g = z * dw.abs(), (t_z + U * z) * dw.abs()
    t_gh = t_g * hat.abs() + gz * hat.abs() * 4 * U
    s1, s2 = over(gz, spans, groups) / n, over(gz * hat.abs(), spans, groups) / n
    t1 = over(t_g, spans, groups) / n + (chain + 4) * U * s1
    t2 = over(t_gh, spans, groups) / n + (chain + 4) * U * s2
    put = lambda t: spread(t, spans, groups, C)  # noqa: E731
    t_x = r * (t_g + put(t1) + hat.abs() * put(t2) + 6 * U * (gz + put(s1) + hat.abs() * put(s2)))
    t_x = t_x * (1 + h) + h * wdx.abs() + smallest(x.dtype)
    assert bool(((d_x[:used].double() - wdx).abs() <= t_x).all()), float(((d_x[:used].double() - wdx).abs() / t_x).max())
    assert not d_x[used:].any()
    rows_chain = used / 64 + 64 + len(spans) / 64
    assert bool(((d_b.double() - wdb).abs() <= t_z.sum(0) + rows_chain * U * z.sum(0) + 1e-45).all())
    assert bool(((d_w.double() - wdw).abs() <= (t_z * hat.abs() + 4 * U * z * hat.abs()).sum(0) + rows_chain * U * (z * hat.abs()).sum(0) + 1e-45).all())
    return y, mean, rstd, d_x, d_w, d_b


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,channels,groups,pad,shift", [(1, 8, 1, 0, 0), (3, 16, 2, 0, 0), (513, 128, 1, 0, 0), (100, 100, 4, 0, 0), (37, 101, 1, 3, 1), (65, 256, 8, 0, 0),
                                                            (90, 602, 7, 0, 0), (11, 1024, 32, 8, 0), (9, 2048, 4, 0, 0), (4, 4100, 5, 0, 0), (70, 96, 3, 0, 0), (129, 64, 64, 0, 0), (133, 768, 32, 0, 0), (60, 192, 16, 0, 0),
                                                            (19, 1020, 60, 1, 1), (17, 1023, 341, 0, 0), (140, 12, 4, 0, 0), (90, 360, 10, 0, 0)])
def test_every_row_by_itself(ctx, dtype, rows, channels, groups, pad, shift):
    x = rows_of(rows, channels, TYPES[dtype], 3, pad, shift)
    for i, kind in enumerate(ACTS):
        drop = (None, mg.Dropout(0.5, 3, 1), mg.Dropout(0.2, 4, row_keys=torch.randint(0, 2**40, (rows,)).cuda()), mg.Dropout(0.9, 5, 7, 100))[(i + rows) % 4]
        check_norm(ctx, x, "rows", groups, kind, drop)


SAMPLES = [[1], [2, 0, 1], [37], [64, 1, 0, 200, 65], [0, 0], [700, 3000, 1], [13] * 70]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("samples", SAMPLES, ids=lambda s: f"{len(s)}x{max(s)}")
@pytest.mark.parametrize("channels,groups,pad", [(16, 2, 0), (100, 4, 0), (101, 1, 3), (128, 8, 8), (256, 32, 0), (602, 2, 0), (1100, 11, 0)])
def test_samples_of_uneven_rows(ctx, dtype, samples, channels, groups, pad):
    rows = sum(samples) + 3      # three behind the last
    x = rows_of(rows, channels, TYPES[dtype], 3, pad)
    x[-3:] = float("nan")
    i = (channels + len(samples)) % 4
    drop = (None, mg.Dropout(0.5, 3, 1), mg.Dropout(0.2, 4, row_keys=torch.randint(0, 2**40, (rows,)).cuda()), None)[(i + len(samples)) % 4]
    check_norm(ctx, x, samples, groups, ACTS[i], drop)


# samples larger than one multiprocessor holds, than a cluster of them, and than all of them
@pytest.mark.gpu
@pytest.mark.parametrize("samples,channels,groups,dtype", [([900, 2500], 128, 8, "f32"), ([20_000, 300, 9_000], 256, 8, "f32"), ([400_000, 5, 70_000], 128, 2, "f32"), ([90_000] * 3, 1024, 8, "f16"), ([50_001], 100, 4, "f16"), ([40_000] * 3, 192, 2, "bf16"),
                                                           ([70_000, 1], 101, 1, "f32"), ([30_000, 0, 2], 1030, 2, "f16"), ([150_000], 128, 4, "f32")])
def test_large_samples(ctx, samples, channels, groups, dtype):
    x = rows_of(sum(samples), channels, TYPES[dtype], 3)
    check_norm(ctx, x, samples, groups, "silu", mg.Dropout(0.3, 9))


# samples that several blocks share: from two to sixteen of them, shares without a row, many samples for each cluster, empty ones in between
@pytest.mark.gpu
@pytest.mark.parametrize("samples,channels,groups,dtype", [([100], 128, 8, "f32"), ([2000], 128, 8, "f32"), ([35], 1024, 32, "bf16"), ([17, 0, 16, 1], 1020, 5, "f32"), ([500] * 16, 128, 4, "f32"),
                                                           ([700, 0, 300, 512] * 16, 256, 32, "f16"), ([137, 137, 137], 100, 4, "f32"), ([3, 250, 0, 249] * 35, 64, 2, "f32"), ([130] * 148, 128, 1, "f16")])
def test_samples_of_several_blocks(ctx, samples, channels, groups, dtype):
    x = rows_of(sum(samples) + 2, channels, TYPES[dtype], 3)
    for kind, drop in (("silu", None), ("relu", mg.Dropout(0.4, 6))):
        first = check_norm(ctx, x, samples, groups, kind, drop)
        for a, b in zip(first, check_norm(ctx, x, samples, groups, kind, drop)):
            assert torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("shape,groups", [((4, 9, 48), 3), ((2, 33, 17, 64), 8), ((5, 1, 32), 2), ((300, 4, 16), 1), ((3, 2000, 96), 4), ((0, 5, 8), 2), ((4, 0, 8), 2)])
def test_equal_samples(ctx, shape, groups):
    x = torch.randn(shape, device="cuda") + 0.3
    per = math.prod(shape[1:-1])
    y, mean, rstd = ctx.group_norm(x, groups, activation="gelu")
    d_x, d_w, d_b = ctx.group_norm_backward(torch.ones_like(x), x, mean, rstd, groups, activation="gelu")
    n = shape[0] if per else 0
    assert y.shape == d_x.shape == x.shape and mean.shape == rstd.shape == (n, groups)
    if not n:
        assert not d_w.any() and not d_b.any()
        return
    flat = x.view(-1, shape[-1])
    y2, mean2, rstd2 = ctx.group_norm(flat, groups, sample_offsets=torch.arange(n + 1) * per, activation="gelu")
    want, wmean, _, _ = norm(flat, [(i * per, (i + 1) * per) for i in range(n)], groups, 1.0, 0.0, 1e-5, "gelu")
    assert float((y.view(-1, shape[-1]).double() - want).abs().max()) < 2e-5      # (1.13 (n / 64 + 80) u |hat|, |hat| below 6, n below 50,000)
    assert float((y2.double() - want).abs().max()) < 2e-5 and float((mean.double() - wmean).abs().max()) < 2e-5


@pytest.mark.gpu
@pytest.mark.parametrize("samples", ["rows", [50, 0, 350], [6000]])
def test_values_far_from_zero_and_equal_ones(ctx, samples):
    rows = 400 if samples == "rows" else sum(samples)
    x = rows_of(rows, 128, torch.float32, 3, centre=3000.0)      # a mean a thousand times the deviation
    check_norm(ctx, x, samples, 4, "none")
    x.fill_(0.7)
    y, mean, rstd = ctx.group_norm(x, 4, sample_offsets=spans_of(samples, rows)[1])
    # (equal values: their sum's rounding is what deviates, and eps keeps it small)
    assert float(y.abs().max()) < 0.7 * (rows * 32 / 64 + 70) * U / math.sqrt(1e-5)


@pytest.mark.gpu
@pytest.mark.parametrize("samples", ["rows", [3, 40, 5], [900, 800, 4000]])
def test_bad_values_stay_in_their_sample_and_group(ctx, samples):
    rows = 48 if samples == "rows" else sum(samples)
    spans, ends = spans_of(samples, rows)
    x = rows_of(rows, 96, torch.float32, 3)
    clean = x.clone()
    lo, hi = spans[1]
    x[lo, 40] = float("nan")
    x[spans[2][0], 0] = float("inf")
    drop = mg.Dropout(0.5, 3)
    got = ctx.group_norm(x, 3, sample_offsets=ends, activation="relu", dropout=drop)
    want = ctx.group_norm(clean, 3, sample_offsets=ends, activation="relu", dropout=drop)
    keep = kept(range(rows), 96, 0.5, 3, 0).cuda()
    bad = torch.zeros(rows, 96, dtype=torch.bool, device="cuda")
    bad[lo:hi, 32:64] = True
    bad[spans[2][0]:spans[2][1], :32] = True
    assert torch.equal(got[0][~bad], want[0][~bad])
    assert bool(got[0][bad & keep].isnan().all()) and not got[0][~keep].any()
    d_y = torch.ones_like(x)
    a = ctx.group_norm_backward(d_y, x, got[1], got[2], 3, sample_offsets=ends, activation="silu", dropout=drop)
    b = ctx.group_norm_backward(d_y, clean, want[1], want[2], 3, sample_offsets=ends, activation="silu", dropout=drop)
    assert torch.equal(a[0][~bad], b[0][~bad]) and bool(a[0][bad].isnan().all())


# a ReLU's side of zero does not go by how the sums are cut: values whose normalised value is a rounding away from zero
@pytest.mark.gpu
@pytest.mark.parametrize("samples", ["rows", [64, 64], [4096]])
def test_the_relu_border(ctx, samples):
    rows = 128 if samples == "rows" else sum(samples)
    spans, ends = spans_of(samples, rows)
    x = rows_of(rows, 64, torch.float32, 3)
    w, b = torch.full((64,), 0.7, device="cuda"), torch.full((64,), 0.2, device="cuda")
    _, mean, rstd = ctx.group_norm(x, 2, w, b, sample_offsets=ends)
    m, r = spread(mean.double(), spans, 2, 64), spread(rstd.double(), spans, 2, 64)
    x = torch.where(torch.rand(rows, 64, device="cuda") < 0.5, x.double(), m - 0.2 / 0.7 / r).float()
    d_y = torch.ones_like(x)
    d_x, _, d_b = ctx.group_norm_backward(d_y, x, mean, rstd, 2, w, b, sample_offsets=ends, activation="relu")
    wdx, _, wdb, hat = norm_backward(d_y, x, mean, rstd, spans, 2, w.double(), b.double(), "relu")
    assert float(((hat * w + b).abs() < 1e-6).double().mean()) > 0.3
    assert torch.equal(d_b.double(), wdb)                                            # whole numbers
    assert float((d_x.double() - wdx).abs().max()) < 1e-3 * float(r.max())           # one side mistaken moves it by 0.7 r


@pytest.mark.gpu
@pytest.mark.parametrize("samples", ["rows", [5, 600, 0, 9], [30_000, 2]])
def test_in_place_other_streams_and_runs_alike(ctx, samples):
    rows = 700 if samples == "rows" else sum(samples) + 2
    ends = spans_of(samples, rows)[1]
    x = rows_of(rows, 128, torch.float32, 3)
    how = dict(sample_offsets=ends, activation="gelu", dropout=mg.Dropout(0.4, 6))
    y, mean, rstd = ctx.group_norm(x, 8, **how)
    d_y = rows_of(rows, 128, torch.float32, 9)
    grads = ctx.group_norm_backward(d_y, x, mean, rstd, 8, **how)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        late = torch.empty_like(x)
        torch.cuda._sleep(20_000_000)
        late.copy_(x)
        again = ctx.group_norm(late, 8, **how)
        grads2 = ctx.group_norm_backward(d_y, late, again[1], again[2], 8, **how)
        torch.cuda.current_stream().synchronize()
    for a, b in zip((y, mean, rstd, *grads), (*again, *grads2)):
        assert torch.equal(a, b)
    used = rows if ends is None else ends[-1]
    inout = x.clone()
    ctx.group_norm(inout, 8, out=inout, **how)
    assert torch.equal(inout[:used], y[:used]) and torch.equal(inout[used:], x[used:])
    for given in (d_y.clone(), x.clone()):
        was = given.clone()
        got = ctx.group_norm_backward(given if torch.equal(was, d_y) else d_y, given if torch.equal(was, x) else x, mean, rstd, 8, out=given, **how)
        assert got[0] is given and torch.equal(given[:used], grads[0][:used]) and torch.equal(given[used:], was[used:])
        assert torch.equal(got[1], grads[1]) and torch.equal(got[2], grads[2])


@pytest.mark.gpu
@pytest.mark.parametrize("samples", ["rows", [5, 600, 0, 9], [20_000, 2], [10] * 100])
def test_captured_and_replayed(ctx, samples):
    rows = 700 if samples == "rows" else sum(samples)
    ends = spans_of(samples, rows)[1]
    how = dict(sample_offsets=ends, activation="silu", dropout=mg.Dropout(0.4, 6))
    x, d_y = rows_of(rows, 128, torch.float32, 3), rows_of(rows, 128, torch.float32, 4)

    def step():
        y, mean, rstd = ctx.group_norm(x, 8, **how)
        return (y, mean, rstd, *ctx.group_norm_backward(d_y, x, mean, rstd, 8, **how), ctx.dropout(x, mg.Dropout(0.5, 2)))
    first = [t.clone() for t in step()]
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = step()
        graphs.append((graph, held))
    was = x.clone()
    for fresh in (was, was * 2 + 1, was):
        x.copy_(fresh)
        eager = [t.clone() for t in step()]
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in graphs]
        for s, (graph, _) in zip(streams, graphs):      # at the same time: a workspace is a call's own
            with torch.cuda.stream(s):
                for _ in range(3):
                    graph.replay()
        torch.cuda.synchronize()
        for _, held in graphs:
            assert all(torch.equal(a, b) for a, b in zip(held, eager))
    assert all(torch.equal(a, b) for a, b in zip(first, eager))


@pytest.mark.gpu
def test_rows_far_apart(ctx):
    rows, stride = 10, 2 ** 28 - 8                                                  # the last ones start behind 2^31 elements
    flat = torch.empty((rows - 1) * stride + 2 ** 20, dtype=torch.float16, device="cuda")
    for channels in (96, 4096):
        x = flat.as_strided((rows, channels), (stride, 1))
        x.copy_(rows_of(rows, channels, torch.float16, 3))
        for samples in ("rows", [rows], [4, 0, 6]):
            check_norm(ctx, x, samples, 4, "silu", mg.Dropout(0.4, 6))
        check_norm(ctx, x, [rows], 4, "gelu", out=flat.as_strided((rows, channels), (stride, 1), 4096 * 64))
        keep = kept(range(rows), channels, 0.4, 6, 0)
        y = ctx.dropout(x, mg.Dropout(0.4, 6))
        check_dropout(y, x, keep, 0.4)
        assert torch.equal(ctx.dropout(x, mg.Dropout(0.4, 6), out=x), y)


@pytest.mark.gpu
def test_more_than_two_to_the_31_elements(ctx):
    rows, channels, groups, last, p = 4_300_000, 512, 4, 1000, 0.25
    x = torch.empty((rows, channels), dtype=torch.float16, device="cuda").normal_(0.3, 1.0, generator=torch.Generator("cuda").manual_seed(7))
    assert x.numel() > 2 ** 31
    tail, first, h = x[rows - last:], rows - last, half_step(x.dtype)
    keep = kept(range(first, rows), channels, p, 9, 1)
    y = ctx.dropout(x, mg.Dropout(p, 9, 1))
    check_dropout(y[first:], tail, keep, p)
    del y
    # rows by themselves: the last ones as in a call of their own
    y, mean, rstd = ctx.group_norm(x, groups, activation="silu", dropout=mg.Dropout(p, 9, 1))
    want = ctx.group_norm(tail, groups, activation="silu", dropout=mg.Dropout(p, 9, 1, first))
    for a, b in zip((y, mean, rstd), want):
        assert torch.equal(a[first:], b)
    d_x, _, d_b = ctx.group_norm_backward(x, x, mean, rstd, groups, dropout=mg.Dropout(p, 9, 1), out=y)
    assert torch.equal(d_x[first:], ctx.group_norm_backward(tail, tail, *want[1:], groups, dropout=mg.Dropout(p, 9, 1, first))[0])
    del y, d_x
    # one sample.  It has 592 tiles, or 444 where there is a gradient: at most 9,685 rows, four threads to a channel, so that a thread adds up at most
    # 2,422; then 4 threads, 32 tiles and 14 sets of those meet: chains of fewer than 4096 roundings
    chain = 4096
    blocks = [(lo, min(lo + 100_000, rows)) for lo in range(0, rows, 100_000)]
    n = rows * (channels // groups)
    put = lambda t: t.repeat_interleave(channels // groups)  # noqa: E731
    total = lambda f: sum(f(x[lo:hi].double()).view(hi - lo, groups, -1).sum((0, 2)) for lo, hi in blocks)  # noqa: E731
    m = total(lambda t: t) / n
    size, var = total(lambda t: t.abs()) / n, total(lambda t: (t - put(m)) ** 2) / n
    y, mean, rstd = ctx.group_norm(x, groups, sample_offsets=[0, rows])
    t_mean, w_rstd = chain * U * size, (var + 1e-5).rsqrt()
    assert bool(((mean[0].double() - m).abs() <= t_mean).all())
    assert bool(((rstd[0].double() - w_rstd).abs() <= w_rstd * (chain + 12) * U + 0.5 * w_rstd ** 3 * t_mean ** 2).all())
    m, r = put(mean[0].double()), put(rstd[0].double())
    hat = (tail.double() - m) * r
    assert bool(((y[first:].double() - hat).abs() <= (6 * U + h * (1 + 6 * U)) * (hat.abs() + m.abs() * r) + smallest(x.dtype)).all())
    s1, s2 = put(total(lambda t: t) / n), put(total(lambda t: t * (t - m) * r) / n)
    a1, a2 = put(size), put(total(lambda t: (t * (t - m) * r).abs()) / n)
    d_x = ctx.group_norm_backward(x, x, mean, rstd, groups, sample_offsets=[0, rows], out=y)[0]
    want = r * (tail.double() - s1 - hat * s2)
    t_x = r * (1 + h) * ((chain + 8) * U * (a1 + hat.abs() * a2) + 8 * U * (tail.double().abs() + a1 + hat.abs() * a2)) + h * want.abs() + smallest(x.dtype)
    assert bool(((d_x[first:].double() - want).abs() <= t_x).all())


@pytest.mark.gpu
def test_refusals(ctx):
    x = torch.randn(12, 16, device="cuda")
    ones = torch.ones(16, device="cuda")
    stats = torch.ones(12, 2, device="cuda")
    bad = [lambda: ctx.dropout(x, mg.Dropout(1.5, 1)), lambda: ctx.dropout(x, mg.Dropout(float("nan"), 1)), lambda: ctx.dropout(x, mg.Dropout(-0.1, 1)),
           lambda: ctx.dropout(x[:, :8], mg.Dropout(0.5, 1), out=x[:, 4:12]), lambda: ctx.dropout(x[:8], mg.Dropout(0.5, 1), out=x[1:9]),
           lambda: ctx.group_norm(x, 3), lambda: ctx.group_norm(x, 0), lambda: ctx.group_norm(x, 2, eps=0.0), lambda: ctx.group_norm(x, 2, eps=float("inf")),
           lambda: ctx.group_norm(x, 2, sample_offsets=[0, 5, 4, 12]), lambda: ctx.group_norm(x, 2, sample_offsets=[0, 13]),
           lambda: ctx.group_norm(x, 2, sample_offsets=[1, 12]), lambda: ctx.group_norm(x, 2, sample_offsets=[0]),
           lambda: ctx.group_norm(x, 2, sample_offsets=[0] * 4097 + [12]), lambda: ctx.group_norm(x[:8], 2, out=x[2:10]),
           lambda: ctx.group_norm_backward(x, x, stats, stats, 2, dropout=mg.Dropout(2.0, 1))]
    for call in bad:
        with pytest.raises(mg.MgError) as e:
            call()
        assert e.value.code == -1
    wrong = [lambda: ctx.dropout(x.cpu(), mg.Dropout(0.5, 1)), lambda: ctx.dropout(x.double(), mg.Dropout(0.5, 1)), lambda: ctx.dropout(x[0], mg.Dropout(0.5, 1)),
             lambda: ctx.dropout(x, mg.Dropout(0.5, 1, row_keys=torch.arange(3).cuda())), lambda: ctx.dropout(x, mg.Dropout(0.5, 1, row_keys=torch.arange(12).int().cuda())),
             lambda: ctx.dropout(x, mg.Dropout(0.5, 1, site=65536)), lambda: ctx.dropout(x, mg.Dropout(0.5, 1), out=x.half()),
             lambda: ctx.group_norm(x, 2, ones[:4], ones), lambda: ctx.group_norm(x, 2, ones.half(), ones), lambda: ctx.group_norm(x.view(3, 4, 16), 2, sample_offsets=[0, 3]),
             lambda: ctx.group_norm_backward(x, x.half(), stats, stats, 2), lambda: ctx.group_norm_backward(x, x, stats[:3], stats, 2)]
    for call in wrong:
        with pytest.raises(AssertionError):
            call()
    with pytest.raises(KeyError):
        ctx.group_norm(x, 2, activation="tanh")


# ---- refusals that need no GPU --------------------------------------------------------------------------------------
HOST = r"""
#include <cstdarg>
#include <cstdio>
#include <string>
#include <vector>
#include "mg_norm_plan.cuh"
int mg_fail(mg_ctx*, int code, const char*, ...) { return code; }
int mg_cuda_fail(mg_ctx*, cudaError_t, const char*) { return MG_ERR_CUDA; }
void mg_prof_begin(mg_ctx*, int) {}
void mg_prof_end(mg_ctx*, int, int64_t) {}

static mg_ctx context;
static int bad = 0;
#define EXPECT(code, call) do { const int got = (call); if (got != (code)) { printf("line %d: %d\n", __LINE__, got); ++bad; } } while (0)

int main() {
    char* base = reinterpret_cast<char*>(1ull << 30);   // (addresses are only compared)
    DropArgs d;
    mg_dropout_spec drop{0.5, 1, 0, 0, nullptr};
    const auto dropout = [&](const void* x, int64_t xs, const void* y, int64_t ys, int dtype, int64_t rows, int32_t ch) { return check_dropout_call(&context, x, xs, y, ys, dtype, rows, ch, &drop, &d); };
    char* far = base + (1ll << 40);
    EXPECT(MG_OK, dropout(base, 16, far, 16, MG_DTYPE_F32, 10, 16));
    EXPECT(MG_OK, dropout(base, 16, base, 16, MG_DTYPE_F32, 10, 16));
    EXPECT(MG_OK, dropout(base, 64, base + 64, 64, MG_DTYPE_F32, 10, 16));                  // between the rows
    EXPECT(MG_OK, dropout(base + 64 * 5, 64, base + 128, 64, MG_DTYPE_F32, 10, 16));        // ... the output first
    EXPECT(MG_OK, dropout(base, 0, far, 16, MG_DTYPE_F32, 10, 16));                         // one row over and over
    EXPECT(MG_OK, dropout(nullptr, 16, nullptr, 16, MG_DTYPE_F32, 0, 16));
    EXPECT(MG_OK, dropout(base, 3, base, 5, MG_DTYPE_F32, 1, 16));                          // one row has no stride
    EXPECT(MG_ERR_ARG, dropout(base, 16, far, 0, MG_DTYPE_F32, 10, 16));
    EXPECT(MG_ERR_ARG, dropout(base, 16, far, 15, MG_DTYPE_F32, 10, 16));
    EXPECT(MG_ERR_ARG, dropout(base, -16, far, 16, MG_DTYPE_F32, 10, 16));
    EXPECT(MG_ERR_ARG, dropout(base, 1ll << 60, far, 16, MG_DTYPE_F32, 10, 16));
    EXPECT(MG_ERR_ARG, dropout(base, 64, base + 32, 64, MG_DTYPE_F32, 10, 16));
    EXPECT(MG_ERR_ARG, dropout(base, 64, base + 64 * 4 - 32, 64, MG_DTYPE_F32, 10, 16));
    EXPECT(MG_ERR_ARG, dropout(base, 16, base + 64, 16, MG_DTYPE_F32, 10, 16));
    EXPECT(MG_ERR_ARG, dropout(base, 16, base, 32, MG_DTYPE_F32, 10, 16));
    EXPECT(MG_ERR_ARG, dropout(nullptr, 16, far, 16, MG_DTYPE_F32, 10, 16));
    EXPECT(MG_ERR_ARG, dropout(base, 16, nullptr, 16, MG_DTYPE_F32, 10, 16));
    EXPECT(MG_ERR_ARG, dropout(base + 2, 16, far, 16, MG_DTYPE_F32, 10, 16));
    EXPECT(MG_ERR_ARG, dropout(base + 1, 16, far, 16, MG_DTYPE_BF16, 10, 16));
    EXPECT(MG_ERR_ARG, dropout(base, 16, far, 16, 3, 10, 16));
    EXPECT(MG_ERR_ARG, dropout(base, 16, far, 16, MG_DTYPE_F32, -1, 16));
    EXPECT(MG_ERR_ARG, dropout(base, 16, far, 16, MG_DTYPE_F32, 1ll << 31, 16));
    EXPECT(MG_ERR_ARG, dropout(base, 16, far, 16, MG_DTYPE_F32, 10, 0));
    for (const double p : {-0.01, 1.01, (double)NAN}) { drop.p = p; EXPECT(MG_ERR_ARG, dropout(base, 16, far, 16, MG_DTYPE_F32, 10, 16)); }
    drop.p = 0.5; drop.site = 65536; EXPECT(MG_ERR_ARG, dropout(base, 16, far, 16, MG_DTYPE_F32, 10, 16));
    drop.site = 0; drop.row_keys = reinterpret_cast<int64_t*>(base + 4); EXPECT(MG_ERR_ARG, dropout(base, 16, far, 16, MG_DTYPE_F32, 10, 16));
    drop.row_keys = nullptr;
    EXPECT(MG_ERR_ARG, check_dropout_call(&context, base, 16, far, 16, MG_DTYPE_F32, 10, 16, nullptr, &d));
    drop.p = 1.0; dropout(base, 16, far, 16, MG_DTYPE_F32, 10, 16);
    if (!d.on || d.below != 0xFFFFFFFFu || d.factor != 0.f) { printf("all dropped\n"); ++bad; }
    drop.p = 0.0; dropout(base, 16, far, 16, MG_DTYPE_F32, 10, 16);
    if (d.on) { printf("none dropped\n"); ++bad; }

    float* stats = reinterpret_cast<float*>(far);
    const int64_t ends[4] = {0, 4, 4, 9};
    mg_norm_spec ok{};
    ok.rows = 10; ok.channels = 16; ok.groups = 2; ok.eps = 1e-5f; ok.rows_per_sample = 1;
    const auto norm = [&](const mg_norm_spec& s, const float* mean = reinterpret_cast<float*>(1ull << 41), const void* ws = nullptr) {
        return check_norm_call(&context, &s, base, 16, far, 16, true, far + 4096, 16, mean, stats, ws, &d);
    };
    EXPECT(MG_OK, norm(ok));
    const auto with = [&](auto change) { mg_norm_spec s = ok; change(s); return norm(s); };
    EXPECT(MG_OK, with([&](auto& s) { s.sample_offsets = ends; s.n_samples = 3; }));
    EXPECT(MG_OK, with([&](auto& s) { s.rows_per_sample = 5; }));
    EXPECT(MG_ERR_ARG, with([&](auto& s) { s.rows_per_sample = 3; }));
    EXPECT(MG_ERR_ARG, with([&](auto& s) { s.rows_per_sample = 0; }));
    EXPECT(MG_ERR_ARG, with([&](auto& s) { s.groups = 3; }));
    EXPECT(MG_ERR_ARG, with([&](auto& s) { s.groups = 0; }));
    EXPECT(MG_ERR_ARG, with([&](auto& s) { s.groups = -2; }));
    EXPECT(MG_ERR_ARG, with([&](auto& s) { s.activation = 4; }));
    EXPECT(MG_ERR_ARG, with([&](auto& s) { s.activation = -1; }));
    EXPECT(MG_ERR_ARG, with([&](auto& s) { s.dtype = 3; }));
    EXPECT(MG_ERR_ARG, with([&](auto& s) { s.rows = 1ll << 31; }));
    for (const float eps : {0.f, -1.f, (float)NAN, (float)INFINITY}) EXPECT(MG_ERR_ARG, with([&](auto& s) { s.eps = eps; }));
    EXPECT(MG_ERR_ARG, with([&](auto& s) { s.sample_offsets = ends; s.n_samples = 0; }));
    EXPECT(MG_ERR_ARG, with([&](auto& s) { s.sample_offsets = ends; s.n_samples = MG_MAX_BATCHES + 1; }));
    EXPECT(MG_ERR_ARG, with([&](auto& s) { s.sample_offsets = ends + 1; s.n_samples = 2; }));
    EXPECT(MG_ERR_ARG, with([&](auto& s) { s.sample_offsets = ends; s.n_samples = 3; s.rows = 8; }));
    const int64_t back[3] = {0, 5, 4};
    EXPECT(MG_ERR_ARG, with([&](auto& s) { s.sample_offsets = back; s.n_samples = 2; }));
    EXPECT(MG_ERR_ARG, with([&](auto& s) { s.weight = reinterpret_cast<float*>(base + 2); }));
    EXPECT(MG_ERR_ARG, check_norm_call(&context, &ok, base, 16, far, 16, true, far + 4096, 16, stats, stats, nullptr, &d, reinterpret_cast<float*>(base + 2)));
    EXPECT(MG_ERR_ARG, check_norm_call(&context, &ok, base, 16, far, 16, true, far + 4096, 16, stats, stats, nullptr, &d, nullptr, reinterpret_cast<float*>(base + 1)));
    drop.p = 2.0;
    EXPECT(MG_ERR_ARG, with([&](auto& s) { s.dropout = &drop; }));
    EXPECT(MG_ERR_ARG, norm(ok, nullptr));
    EXPECT(MG_ERR_ARG, norm(ok, stats, base + 8));
    EXPECT(MG_ERR_ARG, check_norm_call(&context, nullptr, base, 16, far, 16, true, far, 16, stats, stats, nullptr, &d));
    EXPECT(MG_ERR_ARG, check_norm_call(&context, &ok, base, 16, nullptr, 16, true, far, 16, stats, stats, nullptr, &d));
    EXPECT(MG_ERR_ARG, check_norm_call(&context, &ok, base, 16, far, 16, true, far + 64, 16, stats, stats, nullptr, &d));   // d_x over d_y, a row behind
    EXPECT(MG_OK, check_norm_call(&context, &ok, base, 16, far, 16, true, far, 16, stats, stats, nullptr, &d));
    return bad;
}
"""


# how calls are cut: every index that the kernels form lies in its array, whatever the shape
CUTS = HOST[:HOST.index("int main")] + r"""
#include <random>
int main() {
    std::mt19937 rng(1);
    const auto pick = [&](int64_t lo, int64_t hi) { return (int64_t)std::exp(std::uniform_real_distribution<double>(std::log((double)lo), std::log(hi + 0.99))(rng)); };
#define NEED(x) do { if (!(x)) { printf("line %d: %s (rows %lld channels %d groups %d samples %lld dtype %d backward %d vec %d)\n", __LINE__, #x, (long long)s.rows, s.channels, s.groups, (long long)n, s.dtype, backward, *v); return 1; } } while (0)
    std::vector<int64_t> ends;
    for (int i = 0; i < 20000; ++i) {
        mg_norm_spec s{};
        s.groups = (int)pick(1, 64); s.channels = s.groups * (int)pick(1, i % 50 ? 300 : 5000); s.dtype = (int)(rng() % 3); s.eps = 1.f;
        s.rows_per_sample = pick(1, i % 7 ? 3000 : 40'000'000);
        s.rows = s.rows_per_sample * pick(1, i % 9 ? 40 : 3000);
        if (s.rows >= 1ll << 31) continue;
        mg_dropout_spec drop{0.5, 1, 0, 0, reinterpret_cast<int64_t*>(4096)};
        if (rng() % 2) s.dropout = &drop;
        if (rng() % 2) {
            s.n_samples = (int)std::min<int64_t>(pick(1, MG_MAX_BATCHES), s.rows + 1);
            ends.assign(1, 0);
            for (int k = 1; k < s.n_samples; ++k) ends.push_back((int64_t)(rng() % (uint64_t)(s.rows + 1)));
            ends.push_back(rng() % 16 ? s.rows : 0);   // (all of them empty, now and then)
            for (int64_t& e : ends) e = std::min(e, ends.back());
            std::sort(ends.begin(), ends.end());
            s.sample_offsets = ends.data();
        }
        const int backward = rng() % 2;
        const int64_t n = sample_count(&s);
        const size_t have = norm_workspace(&s, 148, backward);
        for (const int* v = vec_widths(s.dtype); *v; ++v) {
            if (s.channels % *v) continue;
            NormPlan p;
            TileArgs a;
            if (norm_mode(&s) == NORM_ROWS) {
                plan_rows(&s, 148, backward, *v, &p);
                NEED(p.bytes <= have && p.nv * *v <= kRowValues && p.nv * 32 * *v >= s.channels && p.grid >= 1);
                NEED(!backward || 8ull * s.channels * (p.n_parts + kParamSlices) <= p.bytes);
                continue;
            }
            plan_tiles(&s, 148, backward, *v, &p, &a);
            NEED(p.bytes <= have);
            if (p.block_grid) {
                NEED(s.channels <= kBlockChannels && s.groups <= kBlockGroups && s.channels <= (*v << a.results.tx) && a.results.tx <= 8 && p.block_grid <= n * p.cluster && p.block_grid % p.cluster == 0 && p.cluster <= kMaxCluster);
                NEED(!backward || (p.n_parts == p.block_grid && p.at_parts + 8ull * p.n_parts * s.channels <= p.at_slices && p.at_slices + 8ull * kParamSlices * s.channels <= p.bytes));
                NEED(s.n_samples <= kInlineSamples || p.at_table + 8ull * (s.n_samples + 1) <= p.at_parts);
                continue;
            }
            const int64_t pair = 2 * 4 * (int64_t)s.groups, channels = 2 * 4 * (int64_t)s.channels;
            int64_t tile = 0, fans_end = 0;
            for (int64_t q = 0; q < n; ++q) {
                const int64_t len = s.sample_offsets ? s.sample_offsets[q + 1] - s.sample_offsets[q] : s.rows_per_sample;
                const int64_t tiles = (len + a.tile_rows - 1) / a.tile_rows, first = tile / kFan + q, fans = (tiles + kFan - 1) / kFan;
                NEED(first >= fans_end && tiles <= kFan * kFan && fans <= kFan);
                fans_end = first + std::max<int64_t>(fans, 1);
                tile += tiles;
                NEED(!a.equal || tiles == a.tiles_per_sample);
            }
            NEED(tile == a.tiles && tile * std::max(a.sums.chunks, a.results.chunks) < 1ll << 31 && a.tile_rows > 0);
            NEED(a.parts_of_tile >= 1 && (int64_t)a.parts_of_tile * a.part_rows >= a.tile_rows && (int64_t)(a.parts_of_tile - 1) * a.part_rows < a.tile_rows && tile * a.parts_of_tile * a.results.chunks < 1ll << 31);
            NEED(p.at_fan_count + 4 * fans_end <= p.at_sample_count && p.at_fan_parts + fans_end * pair <= p.at_group_parts);
            NEED(p.at_sample_count + 4 * n <= p.cleared && p.at_tile_parts + tile * a.sums.chunks * pair <= p.at_fan_parts);
            NEED(!backward || (tile == 0 && p.n_parts == 0) || (p.n_parts == tile && p.at_group_parts + n * pair <= p.at_parts && p.at_parts + tile * channels <= p.at_slices && p.at_slices + kParamSlices * channels <= p.bytes));
            NEED((int64_t)s.channels <= (int64_t)a.sums.chunks * a.run && (int64_t)a.run * (a.sums.chunks - 1) < s.channels && a.run <= p.sums_vec * 256 && a.run <= (p.sums_vec << a.sums.tx));
            NEED((int64_t)s.channels <= (int64_t)a.results.chunks * (*v << a.results.tx) && a.results.tx <= 8 && a.sums.tx <= 8);
            NEED(s.channels % p.sums_vec == 0 && (a.sums.chunks == 1 || a.run % p.sums_vec == 0));
        }
    }
    return 0;
}
"""


@pytest.mark.parametrize("what", ["refusals", "cuts"])
def test_on_the_host(tmp_path, what):
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(nvcc):
        pytest.skip("no nvcc")
    source = tmp_path / "host.cu"
    source.write_text({"refusals": HOST, "cuts": CUTS}[what])
    program = str(tmp_path / "host")
    made = subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-O0", "-Xcompiler", "-w", "-I", build.CSRC,
                           "-I", os.path.join(build.ROOT, "include"), str(source), "-o", program], capture_output=True, text=True)
    assert made.returncode == 0, made.stderr[-2000:]
    ran = subprocess.run([program], capture_output=True, text=True)
    assert ran.returncode == 0, ran.stdout
