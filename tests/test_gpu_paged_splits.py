"""Attention over the paged cache in hundreds of splits, in splits of more groups than a wave has lanes, and chunks over more tiles than that."""
import math

import numpy as np
import pytest
import torch

import paged_model as M
from paper_2406_17808_amd import paged
from test_gpu_paged import DEV, Run, attend_case, f64, i32, pages_for

pytestmark = pytest.mark.gpu


def values_of(run, s, h, n):
    """Run.values for long sequences: all positions at once."""
    d, size, page = run.d, M.group_bytes(run.d), run.page
    p = np.arange(n)
    slot = p // page
    at_page = np.where(slot < run.table.shape[1], run.table[s][np.minimum(slot, run.table.shape[1] - 1)], -1)
    there = (p < run.max_length) & (at_page >= 0) & (at_page < len(run.want))
    groups = run.want.reshape(len(run.want), run.hkv, page // 32, size)[np.where(there, at_page, 0), h, p % page // 32]      # [n, bytes]
    r, c = (p % 32)[:, None], np.arange(d)[None]
    take = lambda at: np.take_along_axis(groups, at.astype(np.int64), 1)  # noqa: E731
    k_codes = take(c // 32 * 512 + r * 16 + c % 32 // 2) >> (4 * (c % 2)).astype(np.uint8) & 15
    v_codes = take(16 * d + c // 64 * 1024 + r // 4 % 4 * 256 + c % 16 * 16 + c // 32 % 2 * 8 + r // 16 * 4 + r % 4) >> (4 * (c // 16 % 2)).astype(np.uint8) & 15
    k_bytes = take(32 * d + np.arange(d // 32)[None] * 32 + r % 16 * 2 + r // 16)
    at = 33 * d + 2 * (r // 4 % 4 * 8 + r // 16 * 4 + r % 4)
    scale = (take(at).astype(np.uint32) << 16 | take(at + 1).astype(np.uint32) << 24).view(np.float32).astype(np.float64)[:, 0]
    k, v = M.k_values(k_codes, k_bytes), M.v_values(v_codes, scale)
    return np.where(there[:, None], k, 0.0), np.where(there[:, None], v, 0.0), there


def check(run, q, out, rounds, sequences=None, first=None):
    """Rows against the model, with `rounds` bounding the additions of 32 bits that follow each other in a sum: those of a lane over its
    share, those of the join.  `first`: values_of sequence 0, KV head 0."""
    g = run.hq // run.hkv
    q64, out64 = f64(q), f64(out)
    for s in range(len(run.lengths)) if sequences is None else sequences:
        a, e = run.offsets[s], run.offsets[s + 1]
        n = run.lengths[s] + e - a
        if a == e:
            continue
        pos = np.repeat(run.lengths[s] + np.arange(e - a), g)      # rows: tokens, then the heads of a group
        for h in range(run.hkv):
            k, v, there = first if first is not None and s == h == 0 else values_of(run, s, h, n)
            seen = (np.arange(n)[None] <= pos[:, None]) & there[None]
            heads = slice(h * g, h * g + g)
            want, weighted, spread = M.attend(q64[a:e, heads].reshape(-1, run.d), k, v, seen, run.scale)
            off = np.abs(out64[a:e, heads].reshape(-1, run.d) - want) - M.attend_tolerance(run.ty, want, weighted, spread, run.d, rounds)
            assert (off <= 0).all(), (s, h, float(off.max()))


def test_values_of_is_values():
    run, _, _, _ = attend_case("f32", 64, 2, 2, 96, [200, 31], [3, 1], seed=1)
    table = run.table.copy()
    table[0, 1], table[1, 0] = -1, 10 ** 9
    run.batch([200, 31], [3, 1], table, max_length=201)
    for s, n in ((0, 203), (1, 32)):
        for h in range(2):
            for x, y in zip(values_of(run, s, h, n), run.values(s, h, n)):
                np.testing.assert_array_equal(x, y)


def needles(run, k, at):
    """Queries each of which points at the key k[p] of one position: [calls] of [tokens, heads, d]."""
    for p in at:
        x = torch.from_numpy(np.array(k[p])).to(DEV)
        # its own logit is 30, those of others a small share of it
        yield (30.0 / run.scale * x / (x @ x)).to(run.ty)[None, None].expand(sum(run.new), run.hq, -1).contiguous()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("context", [9000, 33000, 131071])
def test_one_token_in_hundreds_of_splits(dtype, d, context):
    """One KV head: 71, 259 and 342 splits.  Every split counts: rows that spread over all keys, and rows that look for one key, in splits from the first
    to the last."""
    run, batch, q, out = attend_case(dtype, d, 2, 1, 256, [context], [1], seed=context % 97)
    n = context + 1
    first = values_of(run, 0, 0, n)
    check(run, q, out, 600, first=first)
    assert torch.equal(out, run.cache.attend(batch, q))
    for x in needles(run, first[0], [0, 127, n // 3, n // 2 + 7, n * 3 // 4, n - 700, n - 130, n - 1]):
        check(run, x, run.cache.attend(batch, x), 600, first=first)
    # all but one page missing: its keys alone
    table = run.table.copy()
    keep = table.shape[1] * 4 // 5
    table[0, np.arange(table.shape[1]) != keep] = -1
    alone = run.batch([context], [1], table)
    check(run, q, run.cache.attend(alone, q), 600)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq", [16, 32])
def test_splits_of_more_groups_than_a_wave_has_lanes(dtype, d, hq):
    """1024 sequences leave room for four splits of 137 groups a wave (16 heads: eight of 69); a missing page, a NaN value and a key looked for behind the 64th and
    the 128th."""
    lengths, new = [70000] + [0, 3] * 511 + [40], [1] + [0, 1, 0, 0] * 255 + [0, 1, 1]
    run, batch, q, out = attend_case(dtype, d, hq, 1, 256, lengths, new, seed=d)
    few = [0, 2, 6, 1022, 1023]
    first, whole = values_of(run, 0, 0, 70001), run.table.copy()
    check(run, q, out, 1000, few, first)
    for x in needles(run, first[0], [8100, 8191, 8192, 8300, 8800, 16400, 17500, 17600, 26000, 34000, 69999, 70000]):
        check(run, x, run.cache.attend(batch, x), 1000, [0], first)
    for gone in ([32], [31], [32, 64, 97], [68], [100, 270]):      # (pages of 256 keys; splits of 17536 or 8832 keys)
        table = whole.copy()
        table[0, gone] = -1
        again = run.batch(lengths, new, table)
        check(run, q, run.cache.attend(again, q), 1000, [0])
    before = run.cache.pages.clone()
    for at in (8200, 16500, 69000):
        k, v = run.rows(1, 1), run.rows(1, 1)
        v[0, 0, 3] = math.nan
        run.cache.append(run.batch([at], [1], whole[:1]), k, v)
        got = run.cache.attend(run.batch(lengths, new, whole), q)
        assert bool(torch.isnan(got[0]).all()) and torch.equal(got[1:], out[1:])
        run.cache.pages.copy_(before)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("gone", [[131], [3], [67, 131], [0, 64, 128], [63, 64, 127, 128], [140]])
def test_many_rows_with_missing_pages_behind_64_tiles(dtype, d, gone):
    """The kernel for many rows over 75 tiles of 64 keys and more in one go (pages of 32 keys: group 131 is of tile 65, whose place is kept where tile 1's
    was): a missing page hides its keys only, wherever the others that share its lane are."""
    lengths, new = [4700] + [0] * 420, [140] + [0] * 420
    run, batch, q, _ = attend_case(dtype, d, 4, 1, 32, lengths, new, seed=len(gone))
    table = run.table.copy()
    table[0, gone] = [-1, 10 ** 9, -7, len(run.want)][:len(gone)]
    again = run.batch(lengths, new, table)
    plain = run.cache.attend(again, q)
    check(run, q, plain, 5000)
    before = run.cache.pages.clone()
    for at in (4130, 4260):      # a NaN value, a NaN key behind the 64th tile
        for which in range(2):
            k, v = run.rows(1, 1), run.rows(1, 1)
            (k if which else v)[0, 0, 3] = math.nan
            run.cache.append(run.batch([at], [1], table[:1]), k, v)
            got = run.cache.attend(run.batch(lengths, new, table), q)
            hidden = at // 32 in gone
            assert torch.equal(got, plain) if hidden else bool(torch.isnan(got).all())
            run.cache.pages.copy_(before)
    at = 4700 + 77      # among the new tokens
    k, v = run.rows(1, 1), run.rows(1, 1)
    v[0, 0, 3] = math.nan
    run.cache.append(run.batch([at], [1], table[:1]), k, v)
    got = run.cache.attend(run.batch(lengths, new, table), q)
    assert torch.equal(got[:77], plain[:77]) and bool(torch.isnan(got[77:]).all())


@pytest.mark.parametrize("rows", [6, 60])
def test_false_lengths_and_offsets_byte_by_byte(rows):
    """What the rules leave of arrays that break their promises is written and read, and nothing else: every byte of the pool."""
    half, max_length = rows // 2, 70
    run = Run("bf16", 64, 4, 2, 32, 16, 3, seed=rows)
    table = np.array([[3, 1, 14, 9], [0, 2, 5, 7], [8, 6, 4, 10]])
    run.max_length, run.table = max_length, table
    k, v = run.rows(rows, 2), run.rows(rows, 2)

    # sequence 0: its rows as far as max_length; sequence 1: no rows; sequence 2: behind max_length
    odd = paged.PagedBatch(i32([60, -7, 2 ** 31 - 1]), i32([0, half, half, 2 ** 31 - 1]), i32(table), rows, half, max_length)
    M.append(run.want, table, [60], [0, half], 32, 2, f64(k), f64(v), max_length)
    run.cache.append(odd, k, v)
    run.check_bytes()
    got_k, got_v = run.cache.read(odd)
    for h in range(2):
        wk, wv, _ = run.values(0, h, 60 + half)      # (zeros behind max_length)
        assert torch.equal(got_k[:half, h].cpu(), torch.from_numpy(wk[60:]).to(run.ty)) and torch.equal(got_v[:half, h].cpu(), torch.from_numpy(wv[60:]).to(run.ty))
    assert bool((got_k[half:] == 0).all()) and bool((got_v[half:] == 0).all())

    # a negative length is 0; an offset below 0 is 0; no more new tokens than max_new
    below = paged.PagedBatch(i32([-7]), i32([-3, 2 ** 31 - 1]), i32(table[1:2]), rows, half, max_length)
    M.append(run.want, table[1:2], [0], [0, half], 32, 2, f64(k), f64(v), max_length)
    run.cache.append(below, k, v)
    run.check_bytes()
    got_k, got_v = run.cache.read(below)
    for h in range(2):
        wk, wv, _ = run.values(1, h, half)
        assert torch.equal(got_k[:half, h].cpu(), torch.from_numpy(wk).to(run.ty)) and torch.equal(got_v[:half, h].cpu(), torch.from_numpy(wv).to(run.ty))

    # offsets that fall, so that sequences claim each other's rows: of every slot that one of them claims a whole row, that one's or what was there
    falling = paged.PagedBatch(i32([20, 5, 40]), i32([0, half, 1, rows]), i32(table), rows, half, max_length)
    one, other = run.want.copy(), run.want.copy()
    M.append(one, table[:1], [20], [0, half], 32, 2, f64(k), f64(v), max_length)
    M.append(other, table[2:], [40], [1, 1 + half], 32, 2, f64(k), f64(v), max_length)
    run.cache.append(falling, k, v)
    got = run.cache.pages.cpu().numpy()
    assert ((got == run.want) | (got == one) | (got == other)).all()
    outside = (one == run.want) & (other == run.want)
    assert (got == run.want)[outside].all()
