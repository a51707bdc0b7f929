"""Sampling where the point that keys and masses are relative to matters: rows masked by finite values, tied largest
logits, small temperatures, random numbers below the normal range.

The winner is computed in 64 bits.  A key is s - log noise with s = (z - max z) / T: in 32 bits a few roundings of 2^-24
of the larger of its terms, and up to 64 of its unit for the point it is relative to, so a token within
1e-5 + 1e-6 |key| of the winner's key may take its place (rows are drawn so that there is none nearly always).  Where only
tied logits are kept no rounding is left that differs between them, and the token has to be the one."""
import numpy as np
import pytest
import torch

import paper_2609_14636_amd as P

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def call(z, vocab, noise, temp, k=0, p=1.0, low=0.0):
    n = z.shape[0]
    full = lambda x, dt: torch.full((n,), x, dtype=dt, device="cuda")  # noqa: E731
    ids = torch.full((n,), -7, dtype=torch.int32, device="cuda")
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.full((max(256, P.stride_sample_workspace_size(n, vocab)),), 255, dtype=torch.uint8, device="cuda")
    P.stride_sample(vocab, z, noise, full(temp, F32), full(k, torch.int32), full(p, F32), full(low, F32), ids, flags, ws)
    assert int(flags) == 0
    return ids.tolist()


def buffers(n, vocab, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    z = 2.0 * torch.randn(n, vocab + -vocab % 8, generator=g)
    noise = torch.empty(n, vocab + -vocab % 4).exponential_(generator=g)
    return z.to(dtype), noise, g


def check(z, vocab, noise, temp, got):
    """Against the unfiltered race in 64 bits."""
    zz, e = z[:, :vocab].double().numpy(), noise[:, :vocab].double().numpy()
    with np.errstate(divide="ignore"):
        key = (zz - zz.max(1, keepdims=True)) / float(np.float32(temp)) - np.log(e)
    for r, t in enumerate(got):
        best = key[r].max()
        assert 0 <= t < vocab and key[r, t] >= best - (1e-5 + 1e-6 * abs(best)), (r, t, int(key[r].argmax()), key[r, t], best)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,vocab", [(3, 40000), (64, 40000), (140, 40000), (2, 151936), (130, 151936)])
@pytest.mark.parametrize("mask", [-1e4, -1e9, "lowest"])
def test_unfiltered_rows_with_masked_beginnings(dtype, rows, vocab, mask):
    """Ten tokens are allowed, none of them among the first of the row: past the first 9,000, or the last of all."""
    low = torch.finfo(dtype).min if mask == "lowest" else mask
    for first, step in ((9000, 2900), (vocab - 10, 1)):
        z, noise, _ = buffers(rows, vocab, dtype, seed=vocab + rows)
        allowed = torch.arange(10) * step + first
        values = z[:, allowed].clone()
        z[:, :vocab] = low
        z[:, allowed] = values
        for temp in (1.0, 0.7, 0.02):
            got = call(z.cuda(), vocab, noise.cuda(), temp)
            assert set(got) <= set(allowed.tolist())
            check(z, vocab, noise, temp, got)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows", [5, 140])
def test_unfiltered_rows_of_large_values(dtype, rows):
    """Logits far from 0 on either side, the largest of them late in the row."""
    vocab = 40000
    for shift in (-3000.0, 3000.0):
        z, noise, g = buffers(rows, vocab, F32, seed=17)
        z += shift
        z[:, 30000:30100] += 40.0
        z = z.to(dtype)
        for temp in (1.0, 5.0, 1e-3, 1e-12):
            check(z, vocab, noise, temp, call(z.cuda(), vocab, noise.cuda(), temp))


def tied(rows, vocab, dtype, ties, seed):
    """Rows whose largest value, near 18, is at `ties` places; the others are half a unit lower and more."""
    z, noise, g = buffers(rows, vocab, dtype, seed)
    at = torch.stack([torch.randperm(vocab, generator=g)[:ties].sort().values for _ in range(rows)])
    top = (17.0 + 2.0 * torch.rand(rows, 1, generator=g)).to(dtype)
    z = torch.minimum(z, top - 0.5)
    z.scatter_(1, at, top.expand(-1, ties).contiguous())
    return z, noise, at


def smallest(noise, at, kept):
    return [int(at[r, noise[r, at[r, :kept]].argmin()]) for r in range(len(at))]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,vocab", [(5, 900), (5, 40000), (140, 40000)])
@pytest.mark.parametrize("ties", [2, 6, 600, 3000])
def test_tied_largest_values(dtype, rows, vocab, ties):
    """exp(s) is 1 for them: min-p of 1 keeps all, top-p by their number, and the smallest random number wins."""
    ties = min(ties, vocab // 2)
    z, noise, at = tied(rows, vocab, dtype, ties, seed=ties)
    zc, nc = z.cuda(), noise.cuda()
    for temp, k, p, low, kept in ((1.0, 0, 1.0, 1.0, ties), (1.0, 0, 1.0, 0.9, ties), (0.7, 0, 1.0, 1.0, ties),
                                  (1.0, 4000, 1.0, 1.0, ties), (1e-4, 0, 1.0, 0.0, ties), (1e-4, 0, 1.0, 0.9, ties),
                                  (1e-6, 0, 1.0, 1.0, ties), (1e-6, 40, 1.0, 0.0, min(40, ties)), (1e-6, 0, 0.5, 0.0, ties // 2),
                                  (1e-8, 0, 0.5, 0.9, ties // 2), (1e-8, 2, 1.0, 0.0, 2), (1e-8, 0, 1.0, 0.0, ties),
                                  (1e-20, 0, 0.5, 0.0, ties // 2), (1e-20, 0, 1.0, 0.5, ties), (1e-35, 0, 0.5, 0.0, ties // 2),
                                  (1e-35, 10 ** 6, 1.0, 0.1, ties), (1e-35, 2000, 0.5, 0.0, min(1000, ties // 2))):
        got = call(zc, vocab, nc, temp, k, p, low)
        assert got == smallest(noise, at, kept), (temp, k, p, low)


@pytest.mark.parametrize("rows,vocab", [(5, 900), (5, 40000), (140, 40000)])
def test_the_largest_temperature(rows, vocab):
    """All finite logits are one then: the smallest random number wins among those that are kept."""
    z, noise, g = buffers(rows, vocab, F32, seed=23)
    z[:, :vocab][torch.rand(rows, vocab, generator=g) < 0.5] = -torch.inf
    inside = z[:, :vocab].clone()
    for k in (0, 10):
        kept = inside > -torch.inf if k == 0 else inside >= inside.topk(k, 1).values[:, -1:]
        want = torch.where(kept, noise[:, :vocab], torch.inf).argmin(1).tolist()
        assert call(z.cuda(), vocab, noise.cuda(), 3e38, k) == want


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,vocab", [(4, 900), (4, 40000), (140, 20000)])
@pytest.mark.parametrize("k,p,low", [(0, 1.0, 0.0), (50, 1.0, 0.0), (0, 1 - 2.0 ** -24, 0.0), (0, 1.0, 1e-35), (4000, 1.0, 0.0)])
def test_random_numbers_below_the_normal_range(dtype, rows, vocab, k, p, low):
    """2^-133 and 2^-131 are random numbers like others: their logarithms count, and 0 alone always wins."""
    z, noise, _ = buffers(rows, vocab, dtype, seed=5)
    z[:, [100, 300, 700]] = torch.tensor([30.0, 30.0, 40.0], dtype=dtype)
    noise[:, 100], noise[:, 300], noise[:, 700] = 2.0 ** -131, 2.0 ** -133, 1.0
    # keys: -10 + 90.8, -10 + 92.2, 0
    assert call(z.cuda(), vocab, noise.cuda(), 1.0, k, p, low) == [300] * rows
    z[:, 700] = 130.0  # -100 + 90.8, -100 + 92.2, 0
    assert call(z.cuda(), vocab, noise.cuda(), 1.0, k, p, low) == [700] * rows
    z[:, 700] = 40.0
    noise[:, 310] = 0.0
    z[:, 310] = 30.0
    assert call(z.cuda(), vocab, noise.cuda(), 1.0, k, p, low) == [310] * rows
