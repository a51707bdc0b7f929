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
