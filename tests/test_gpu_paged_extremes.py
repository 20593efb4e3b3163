"""Attention over the paged cache where logits leave the range of 32 bits or come near its ends: every kernel, and their joins."""
import math

import numpy as np
import pytest
import torch

import paged_model as M
from test_gpu_paged import Run, f64, pages_for

pytestmark = pytest.mark.gpu

# Query heads a KV head, KV heads, lengths, new tokens, sequences without a new token (hundreds of them keep the kernel for few rows to
# sequences of at most 32 rows): one block of 16 rows without a split and with some, blocks of 32 rows, 2048 rows in a few splits, the kernel for
# many rows without a split and with some.
CALLS = {
    "one token": (4, 1, [90, 0, 33], [1, 1, 1], 0),
    "one token, splits": (4, 1, [3000, 40], [1, 1], 0),
    "few tokens, splits": (4, 1, [2500, 300], [12, 30], 0),
    "joins of many rows": (8, 2, [1500, 0, 900, 40], [32, 32, 1, 5], 0),
    "many rows": (4, 1, [700, 0, 200], [130, 257, 40], 420),
    "many rows, splits": (16, 1, [3000], [90], 99),
}


def made(call, dtype, d, bad, q0, k0, window=0, seed=0, missing=()):
    """A cache whose keys have channel 0 = k0 where bad(sequence, position), else 0, and queries whose channel 0 is q0: the logits of the one
    kind of key are q0 * k0 * scale and more, those of the other ordinary numbers.  Returns the run, the batch, queries and outputs."""
    g, hkv, lengths, new, empty = CALLS[call]
    lengths, new = lengths + [0] * empty, new + [0] * empty
    rng = np.random.default_rng(seed)
    table, n_pages = pages_for(rng, lengths, new, 32)
    for s, slot in missing:
        table[s, slot] = -1
    run = Run(dtype, d, g * hkv, hkv, 32, n_pages, len(lengths), window=window, seed=seed, fill=0xFF)
    total = [a + b for a, b in zip(lengths, new)]
    k, v = run.rows(sum(total), hkv), run.rows(sum(total), hkv)
    marks = torch.tensor([bad(s, p) for s, n in enumerate(total) for p in range(n)], device=k.device)
    k[..., 0] = torch.where(marks, torch.full((), k0, device=k.device), torch.zeros((), device=k.device))[:, None].to(run.ty)
    k[marks, :, 1:32] = 0      # (what shares its block's scale would be 0 anyway)
    run.cache.append(run.batch([0] * len(total), total, table), k, v)
    batch = run.batch(lengths, new, table)
    run.want = run.cache.pages.cpu().numpy()
    q = run.rows(sum(new), g * hkv)
    q[..., 0] = q0
    return run, batch, q, run.cache.attend(batch, q)


def check_without(run, q, out, bad):
    """Rows over the keys that are not bad; NaN for a row all of whose keys are bad, zeros for one that sees none."""
    g = run.hq // run.hkv
    q64, out64 = f64(q), f64(out)
    counted = {"nan": 0, "zero": 0, "some bad": 0}
    for s in range(len(run.lengths)):
        a, e = run.offsets[s], run.offsets[s + 1]
        if a == e:
            continue
        n = run.lengths[s] + e - a
        pos, j = run.lengths[s] + np.arange(e - a), np.arange(n)
        marked = np.array([bad(s, p) for p in range(n)])
        for h in range(run.hkv):
            k, v, there = run.values(s, h, n)
            sees = (j[None] <= pos[:, None]) & there[None]
            if run.window:
                sees &= j[None] > pos[:, None] - run.window
            good = sees & ~marked[None]
            all_bad = sees.any(1) & ~good.any(1)
            nothing = ~sees.any(1)
            counted["nan"] += int(all_bad.sum())
            counted["zero"] += int(nothing.sum())
            counted["some bad"] += int(((sees & marked).any(1) & good.any(1)).sum())
            for x in range(g):
                rows, got = q64[a:e, h * g + x].copy(), out64[a:e, h * g + x]
                rows[:, 0] = 0      # the other keys have zeros there
                want, weighted, spread = M.attend(rows, np.where(marked[:, None], 0.0, k), v, good, run.scale)
                tol = M.attend_tolerance(run.ty, want, weighted, spread, run.d, n)
                assert np.isnan(got[all_bad]).all(), (s, h, x, "NaN is the softmax of nothing but -inf")
                assert (got[nothing] == 0).all(), (s, h, x)
                assert (np.abs(got - want) <= tol)[good.any(1)].all(), (s, h, x)
    return counted


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("window", [0, 100])
def test_logits_of_minus_infinity(call, dtype, d, window):
    """Keys whose logits are below the range of 32 bits (2^100 times -2^40 times the scale) have no weight next to others, wherever they are: whole
    groups at the front, all of a split, a few in between; a row all of whose keys are such is NaN, as the softmax of nothing but -inf is."""
    def bad(s, p):
        return p < 70 or p % 64 == 5 or 256 <= p < 1400 or (s == 1 and p < 300)

    run, batch, q, out = made(call, dtype, d, bad, -(2.0 ** 40), 2.0 ** 100, window=window, seed=d)
    counted = check_without(run, q, out, bad)
    assert counted["some bad"] > 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("call", CALLS)
def test_all_logits_minus_infinity_or_no_keys(call, dtype):
    """Rows that see nothing but such keys are NaN; rows whose pages are all missing are zeros."""
    g, hkv, lengths, new, empty = CALLS[call]
    total = [a + b for a, b in zip(lengths, new)]
    run, batch, q, out = made(call, dtype, 64, lambda s, p: True, -(2.0 ** 40), 2.0 ** 100, seed=3)
    assert check_without(run, q, out, lambda s, p: True)["nan"] == sum(new) * hkv
    missing = [(0, slot) for slot in range(-(-total[0] // 32))]
    run, batch, q, out = made(call, dtype, 64, lambda s, p: True, -(2.0 ** 40), 2.0 ** 100, seed=4, missing=missing)
    counted = check_without(run, q, out, lambda s, p: True)
    assert counted["zero"] == new[0] * hkv and counted["nan"] == sum(new[1:]) * hkv


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("exponent", [20, 27, 31, 45, 100])
def test_large_finite_logits(call, dtype, d, exponent):
    """Logits of 2^20 to 2^100 in size, above and below zero: the keys with the largest share the row, whatever a product with the scale rounds to."""
    g, hkv, lengths, new, empty = CALLS[call]
    lengths, new = lengths + [0] * empty, new + [0] * empty
    rng = np.random.default_rng(exponent + d)
    table, n_pages = pages_for(rng, lengths, new, 32)
    run = Run(dtype, d, g * hkv, hkv, 32, n_pages, len(lengths), seed=exponent, fill=0xFF)
    total = [a + b for a, b in zip(lengths, new)]
    size = torch.from_numpy(rng.choice([1.0, 1.5, 2.0, 3.0, 4.0, 6.0], sum(total))).to("cuda:0")      # (no channel but one: the logits are exact)
    k, v = torch.zeros_like(run.rows(sum(total), hkv)), run.rows(sum(total), hkv)
    k[..., 0] = size[:, None].to(run.ty)
    run.cache.append(run.batch([0] * len(total), total, table), k, v)
    batch = run.batch(lengths, new, table)
    run.want = run.cache.pages.cpu().numpy()
    q = run.rows(sum(new), g * hkv)
    q[..., 0] = 1.37 * 2.0 ** exponent
    q[:, ::2, 0] *= -1      # (half of the heads: all logits far below zero)
    out = f64(run.cache.attend(batch, q))
    for s in range(len(lengths)):
        a, e = run.offsets[s], run.offsets[s + 1]
        if a == e:
            continue
        n = total[s]
        seen = np.arange(n)[None] <= (lengths[s] + np.arange(e - a))[:, None]
        for h in range(hkv):
            kv, vv, _ = run.values(s, h, n)
            for x in range(g):
                rows = f64(q)[a:e, h * g + x].copy()
                rows[:, 1:] = 0
                want, weighted, _ = M.attend(rows, kv, vv, seen, run.scale)      # differences of the logits: none, or above 2^16
                tol = M.attend_tolerance(run.ty, want, weighted, np.zeros(e - a), d, n)
                assert (np.abs(out[a:e, h * g + x] - want) <= tol).all(), (s, h, x)
