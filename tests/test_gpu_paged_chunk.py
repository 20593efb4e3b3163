"""The paged cache in 4 bits on the GPU: the kernel for many rows at small sizes, and joins of many rows.

Batches with hundreds of sequences without a new token keep the kernel for few rows to sequences of at most 32 rows (its row blocks would be
nearly all empty), so that the other one is reached without long computations here."""
import math

import pytest
import torch

from paper_2406_17808_amd import paged
from test_gpu_paged import attend_case

pytestmark = pytest.mark.gpu


def with_empty(lengths, new, empty):
    return list(lengths) + [0] * empty, list(new) + [0] * empty


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv,page,lengths,new,window,empty", [
    (16, 1, 32, [5000], [40], 0, 420),
    (8, 1, 96, [2500, 0, 4300], [70, 300, 1], 0, 420),
    (4, 1, 256, [0], [600], 0, 420),
    (16, 1, 64, [4500, 90], [66, 3], 1000, 420),
    (1, 1, 128, [4200], [513], 0, 420),
    (2, 1, 32, [31, 0, 1000], [257, 1, 300], 33, 420),
    (4, 2, 64, [700, 0, 1], [130, 0, 257], 0, 420),
    (33, 3, 64, [64, 200], [40, 37], 0, 420),
    (16, 1, 32, [3000], [90], 0, 99),             # split over the keys
    (16, 1, 64, [3000, 2000, 17], [90, 1, 60], 0, 97),
    (16, 1, 64, [5000, 40], [90, 3], 2050, 98),
])
def test_many_rows(dtype, d, hq, hkv, page, lengths, new, window, empty):
    lengths, new = with_empty(lengths, new, empty)
    run, batch, q, out = attend_case(dtype, d, hq, hkv, page, lengths, new, window=window, seed=sum(new))
    run.check_attend(batch, q, out)
    assert torch.equal(out, run.cache.attend(batch, q))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new,empty", [(140, 420), (400, 98)])
def test_many_rows_with_a_missing_page_and_a_nan(dtype, d, new, empty):
    """A missing page hides its keys only; a NaN key or value reaches the rows that see it only."""
    lengths, counts = with_empty([2100, 1300], [new, new], empty)
    run, batch, q, _ = attend_case(dtype, d, 4, 1, 32, lengths, counts, seed=new)
    table = run.table.copy()
    table[0, 30], table[1, 17:20] = -1, 10 ** 9
    again = run.batch(lengths, counts, table)
    plain = run.cache.attend(again, q)
    run.check_attend(again, q, plain)
    before = run.cache.pages.clone()
    for at, which in ((801, 0), (801, 1), (1300 + new // 2, 0), (1300 + new // 2, 1)):
        k, v = run.rows(1, 1), run.rows(1, 1)
        (k if which else v)[0, 0, 3] = math.nan
        run.cache.append(run.batch([0, at], [0, 1], table[:2]), k, v)
        out = run.cache.attend(run.batch(lengths, counts, table), q)
        assert torch.equal(out[:new], plain[:new])
        sees = torch.arange(1300, 1300 + new, device=out.device) >= at
        assert bool(torch.isnan(out[new:][sees]).all()) and torch.equal(out[new:][~sees], plain[new:][~sees])
        run.cache.pages.copy_(before)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_rows_with_hidden_pages_and_rows_without_keys(dtype):
    lengths, counts = with_empty([100, 40, 0, 64], [200] * 4, 400)
    run, batch, q, _ = attend_case(dtype, 64, 4, 1, 32, lengths, counts, seed=7)
    table = run.table.copy()
    table[0, 1] = -1
    table[1, :] = len(run.want)
    table[2, :] = -5
    table[3, 0] = 2 ** 31 - 1
    again = run.batch(lengths, counts, table, max_length=150)
    out = run.cache.attend(again, q)
    run.check_attend(again, q, out)
    assert bool((out[200:600] == 0).all())
    short = run.batch(lengths, counts, run.table[:, :1])
    run.check_attend(short, q, run.cache.attend(short, q))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_rows_behind_a_window_whose_pages_are_gone(dtype):
    lengths, counts = with_empty([1500, 700], [300, 300], 420)
    run, batch, q, out = attend_case(dtype, 64, 4, 1, 32, lengths, counts, window=200, seed=5)
    run.check_attend(batch, q, out)
    table = run.table.copy()
    for s, n in enumerate((1500, 700)):
        table[s, :(n - 199) // 32] = -1
    assert torch.equal(run.cache.attend(run.batch(lengths, counts, table), q), out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_rows_sharp_and_scaled(dtype):
    for gain, scale in ((30.0, 0.0), (1.0, 0.7), (0.0, 0.0)):
        lengths, counts = with_empty([400], [150], 420)
        run, batch, q, out = attend_case(dtype, 128, 4, 1, 64, lengths, counts, q_gain=gain, scale=scale, seed=2)
        run.check_attend(batch, q, out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lengths,new,window", [
    ([1500, 0, 900, 40], [32, 32, 1, 5], 0),
    ([2500, 10, 900, 40], [30, 32, 1, 0], 700),
])
def test_joins_of_many_rows_and_few_splits(dtype, d, lengths, new, window):
    """2048 rows in a few splits, several rows to a workgroup of the join; some sequences have fewer splits, or one."""
    run, batch, q, out = attend_case(dtype, d, 16, 2, 64, lengths, new, window=window, seed=sum(new))
    run.check_attend(batch, q, out)
    assert torch.equal(out, run.cache.attend(batch, q))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_long_chunk_of_many_heads(dtype):
    """Without empty sequences: a chunk large enough for the kernel for many rows, split over the keys."""
    new = 512 if dtype == "bf16" else 250
    run, batch, q, out = attend_case(dtype, 128, 32, 8, 128, [6000 - new], [new], seed=4)
    run.check_attend(batch, q, out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [3, 70])
def test_one_sequence_under_a_large_bound(dtype, new):
    """The host names far more new tokens of a single sequence than there are: the kernel for many rows takes them, rows of no sequence stay."""
    run, batch, q, _ = attend_case(dtype, 128, 32, 8, 64, [700], [new], seed=new)
    more = torch.cat([q, q[:1].expand(2000, -1, -1)])
    wide = paged.PagedBatch(batch.lengths, batch.new_offsets, batch.page_table, new + 2000, 2000, 9000)
    got = torch.full_like(more, 3.0)
    run.cache.attend(wide, more, out=got)
    run.check_attend(batch, q, got[:new])
    assert bool((got[new:] == 3).all())


@pytest.mark.parametrize("lengths,new,empty", [([3000], [90], 99), ([700, 0, 1], [400, 0, 257], 420), ([1500, 0, 900, 40], [32, 32, 1, 5], 4)])
def test_captured_and_replayed(lengths, new, empty):
    """All forms of a call from a graph, replayed between eager calls of the same cache on other inputs and with other lengths."""
    lengths, new = with_empty(lengths, new, empty)
    run, batch, q, out = attend_case("bf16", 128, 16, 2, 64, lengths, new, seed=1)
    k, v = run.rows(sum(new), 2), run.rows(sum(new), 2)
    q2, pages = run.rows(sum(new), 16), run.cache.pages.clone()
    run.cache.append(batch, k, v)
    after, want_k, want_v = run.cache.attend(batch, q), *run.cache.read(batch)
    shorter = batch.lengths.clone()
    shorter[0] -= 40
    got, stream = torch.empty_like(q), torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        before = run.cache.attend(batch, q)
        run.cache.append(batch, k, v)
        run.cache.attend(batch, q, out=got)
        got_k, got_v = run.cache.read(batch)
    for i in range(4):
        run.cache.pages.copy_(pages)
        for x in (before, got, got_k, got_v):
            x.zero_()
        other = run.cache.attend(batch, q2)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(before, out) and torch.equal(got, after), i
        assert torch.equal(got_k, want_k) and torch.equal(got_v, want_v) and other.isfinite().all()
    # what the graph reads when it runs
    was = batch.lengths.clone()
    run.cache.pages.copy_(pages)
    batch.lengths.copy_(shorter)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(before, run_at(run, batch, q, pages)), "follows the lengths"
    batch.lengths.copy_(was)


def run_at(run, batch, q, pages):
    run.cache.pages.copy_(pages)
    return run.cache.attend(batch, q)
