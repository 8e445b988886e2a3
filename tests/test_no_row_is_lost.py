"""Sums over many rows, on data that drifts along them and with bounds from the additions that the code makes: a tile that is left out, taken twice or
brought in with a wrong weight moves a result by many times what it may be off.

The data: x = ramp + noise / 2, the ramp from -3/2 to 3/2 over a sample's rows; d_y = 2 + noise / 2.  A part of the rows whose mean is away from the sample's moves the
mean, one whose mean is the sample's moves the variance (which has the ramp's 3/4 in it), and every part moves the sums of d_y.

The additions.  A thread adds up the rows of its tile that are its own, the block its threads, a group its channels, then come 32 tiles and 32 of those.
Tiles are as large as 444 blocks (three to a multiprocessor, 592 where there is no gradient) with 1 / 2 to spare leave them; blocks and clusters of
blocks take up to 16 rows a thread."""
import math

import pytest
import torch

import paper_2202_02365_b200 as mg
from test_between_layers import ACTS, TYPES, U, check_norm, ctx, half_step, norm_backward, over, rows_of, smallest, spans_of, spread  # noqa: F401

CASES = [([400_000, 5, 70_000], 128, 2, "f32"), ([90_000] * 3, 1024, 8, "f16"), ([70_000, 1], 256, 1, "f32"), ([30_000, 0, 2], 1032, 2, "f16"), ([150_000], 128, 4, "f32"),
         ([20_000, 300, 9_000], 256, 8, "f32"), ([900, 2500], 128, 8, "f32"), ([2000], 128, 8, "f32"), ([600] * 40, 512, 4, "f16")]


def chain(samples, channels, groups, dtype):
    vec = 8 if dtype == "f16" else 4
    across = min(256, 1 << math.ceil(math.log2(channels // vec)))
    threads, runs = 256 // across, -(-(channels // vec) // across)
    per = min(32, 1 << int(math.log2(max(1, 256 // groups))))     # threads that share a group's channels, and meet in five steps
    return 2 * -(-sum(samples) * runs // (444 * threads)) + threads + -(-channels // groups // per) + 5 + 64 + 32


def drifting(samples, channels, dtype, seed=3):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(sum(samples), channels, generator=g) / 2
    d_y = 2 + torch.randn(sum(samples), channels, generator=g) / 2
    at = 0
    for n in samples:
        x[at:at + n] += torch.linspace(-1.5, 1.5, n)[:, None]
        at += n
    return x.to(TYPES[dtype]), d_y.to(TYPES[dtype])


def bounds(most, deviation, links):
    """Of a mean and of a reciprocal deviation, relative.  A merge rounds the mean once, and the step to it, d nb / n, by six units (a quotient of two units,
    a difference, a product); the steps fall like 1 / n, and ln of the links is below ten.  A merge rounds the squares by ten units, and a mean that is off by e
    moves their sum by 2 e sqrt(n sum) at most (Cauchy and Schwarz)."""
    t_mean = (links + 64) * U * most
    return t_mean, 0.5 * ((links + 16) * U + 2 * t_mean / deviation) + 6 * U


# the mistake: what the sums would be without some rows, or with them twice
@pytest.mark.parametrize("samples,channels,groups,dtype", [c for c in CASES if sum(c[0]) * c[1] < 100_000_000])
def test_the_bounds_see_a_lost_tile(samples, channels, groups, dtype):
    x, d_y = (t.double() for t in drifting(samples, channels, dtype))
    links = chain(samples, channels, groups, dtype)
    rows, each = samples[0], channels // groups
    x, d_y = x[:rows, :each], d_y[:rows, :each]
    size = max(16, sum(samples) // 1184)       # a tile with two turns of 592 blocks (its least is 16 rows)
    n, cuts = rows * each, rows // size
    part = x[:cuts * size].reshape(cuts, -1)
    s, q, d = part.sum(1), part.square().sum(1), d_y[:cuts * size].reshape(cuts, size, each).sum(1)
    mean, total_q = x.mean(), x.square().sum()
    deviation = float((total_q / n - mean ** 2).sqrt())
    t_mean, t_rstd = bounds(float(x.abs().max()), deviation, links)
    for sign in (-1, 1):
        m = (x.sum() + sign * s) / (n + sign * part.shape[1])
        var = (total_q + sign * q) / (n + sign * part.shape[1]) - m ** 2
        seen = torch.maximum((m - mean).abs() / t_mean, ((var.rsqrt() * deviation) - 1).abs() / t_rstd)
        assert float(seen.min()) > 2, float(seen.min())
    # sums by channel, of d_y: a tile's against their bound
    assert float((d / ((links + 96) * U * d_y.abs().sum(0))).min()) > 10


@pytest.mark.gpu
@pytest.mark.parametrize("samples,channels,groups,dtype", CASES)
def test_samples(ctx, samples, channels, groups, dtype):  # noqa: F811
    x, d_y = (t.cuda() for t in drifting(samples, channels, dtype))
    spans, ends = spans_of(samples, len(x))
    links, h, each = chain(samples, channels, groups, dtype), half_step(x.dtype), channels // groups
    y, mean, rstd = ctx.group_norm(x, groups, sample_offsets=ends, eps=1e-5)
    d_x, d_w, d_b = ctx.group_norm_backward(d_y, x, mean, rstd, groups, sample_offsets=ends)
    z, zh, z_rows = 0.0, 0.0, torch.zeros((2, channels), dtype=torch.float64, device="cuda")
    for i, (lo, hi) in enumerate(spans):
        if lo == hi:
            assert not mean[i].any() and not rstd[i].any()
            continue
        t, d = x[lo:hi].double().view(hi - lo, groups, each), d_y[lo:hi].double().view(hi - lo, groups, each)
        m, v = t.mean((0, 2)), t.var((0, 2), correction=0)
        t_mean, t_rstd = bounds(t.abs().amax((0, 2)), v.sqrt(), links)
        want = (v + 1e-5).rsqrt()
        assert bool(((mean[i].double() - m).abs() <= t_mean).all()), float(((mean[i].double() - m).abs() / t_mean).max())
        assert bool(((rstd[i].double() / want - 1).abs() <= t_rstd).all()), float(((rstd[i].double() / want - 1).abs() / t_rstd).max())
        m, r = mean[i].double()[None, :, None], rstd[i].double()[None, :, None]
        hat = (t - m) * r
        # three roundings (a difference, the factor's, a product) and the row type's
        assert bool(((y[lo:hi].double().view(t.shape) - hat).abs() <= (4 * U + h * (1 + 4 * U)) * (hat.abs() + m.abs() * r) + smallest(x.dtype)).all())
        s1, s2 = d.mean((0, 2))[None, :, None], (d * hat).mean((0, 2))[None, :, None]
        t1, t2 = (links + 4) * U * d.abs().mean((0, 2))[None, :, None], (links + 8) * U * (d * hat).abs().mean((0, 2))[None, :, None]
        want = r * (d - s1 - hat * s2)
        bound = r * (t1 + hat.abs() * t2 + 8 * U * (d.abs() + s1.abs() + (hat * s2).abs()))
        bound = bound * (1 + h) + h * want.abs() + smallest(x.dtype)
        off = (d_x[lo:hi].double().view(t.shape) - want).abs() / bound
        assert float(off.max()) <= 1, float(off.max())
        z, zh = z + d.sum(0).flatten(), zh + (d * hat).sum(0).flatten()
        z_rows += torch.stack([d.abs().sum(0).flatten(), (d * hat).abs().sum(0).flatten()])
    # (then the tiles' parts: up to 1,024 in 32 turns and as many threads; one thread's turns over samples)
    parts = links + 96 + len(samples)
    assert bool(((d_b.double() - z).abs() <= parts * U * z_rows[0]).all()), float(((d_b.double() - z).abs() / (parts * U * z_rows[0])).max())
    assert bool(((d_w.double() - zh).abs() <= (parts + 6) * U * z_rows[1]).all()), float(((d_w.double() - zh).abs() / ((parts + 6) * U * z_rows[1])).max())


# rows by themselves: the gradients of weight and bias are the only sums over rows.  148 blocks of eight warps at least, 444 parts at most
@pytest.mark.gpu
@pytest.mark.parametrize("rows,channels,groups,dtype", [(400_000, 64, 2, "f32"), (300_001, 256, 8, "f32"), (200_000, 602, 2, "f32"), (150_000, 768, 1, "f16"), (100_000, 300, 10, "f16"), (20_000, 2048, 4, "f32")])
def test_rows_by_themselves(ctx, rows, channels, groups, dtype):  # noqa: F811
    x, d_y = (t.cuda() for t in drifting([rows], channels, dtype))
    y, mean, rstd = ctx.group_norm(x, groups)
    _, d_w, d_b = ctx.group_norm_backward(d_y, x, mean, rstd, groups)
    links = rows // (148 if channels > 1024 else 148 * 8) + 8 + 32 + 32 + 32
    z = zh = 0.0
    a = torch.zeros((2, channels), dtype=torch.float64, device="cuda")
    for lo in range(0, rows, 50_000):
        d, t = d_y[lo:lo + 50_000].double(), x[lo:lo + 50_000].double().view(-1, groups, channels // groups)
        hat = ((t - mean[lo:lo + 50_000, :, None].double()) * rstd[lo:lo + 50_000, :, None].double()).view(d.shape)
        z, zh = z + d.sum(0), zh + (d * hat).sum(0)
        a += torch.stack([d.abs().sum(0), (d * hat).abs().sum(0)])
    assert bool(((d_b.double() - z).abs() <= links * U * a[0]).all())
    assert bool(((d_w.double() - zh).abs() <= (links + 6) * U * a[1]).all())
    assert links * U < 1e-4        # (a block's share is above 1 / 500)


class Equal:
    """Calls of check_norm's, of equal samples in place of offsets."""

    def __init__(self, ctx, shape):  # noqa: F811
        self.ctx, self.shape = ctx, shape

    def group_norm(self, x, groups, sample_offsets, out=None, **how):
        assert out is None
        y, mean, rstd = self.ctx.group_norm(x.view(self.shape), groups, **how)
        assert y.shape == self.shape
        return y.view(x.shape), mean, rstd

    def group_norm_backward(self, d_y, x, mean, rstd, groups, sample_offsets, **how):
        d_x, d_w, d_b = self.ctx.group_norm_backward(d_y.view(self.shape), x.view(self.shape), mean, rstd, groups, **how)
        assert d_x.shape == self.shape
        return d_x.view(x.shape), d_w, d_b


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape,groups", [((4, 9, 48), 3), ((2, 33, 17, 64), 8), ((5, 1, 32), 2), ((300, 4, 16), 1), ((3, 2000, 96), 4), ((16, 512, 512), 32), ((1, 30_000, 128), 4), ((3, 5000, 100), 4), ((1000, 5, 1100), 11)])
def test_equal_samples(ctx, shape, groups, dtype):  # noqa: F811
    rows = math.prod(shape[:-1])
    x = rows_of(rows, shape[-1], TYPES[dtype], 3)
    i = (shape[0] + groups) % 4
    for drop in (None, mg.Dropout(0.3, 9)):
        check_norm(Equal(ctx, shape), x, [rows // shape[0]] * shape[0], groups, ACTS[i], drop)
