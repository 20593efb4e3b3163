"""The paged cache in 4 bits on the GPU: long contexts, many rows, many sequences, missing pages and NaN far from the ends."""
import math

import numpy as np
import pytest
import torch

from paper_2406_17808_amd import binding as B
from paper_2406_17808_amd import paged
from test_gpu_paged import DEV, Run, attend_case, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv,page,lengths,new,window", [
    (16, 1, 32, [5000], [40], 0),
    (8, 2, 96, [2500, 0, 4300], [70, 300, 1], 0),
    (4, 4, 256, [0], [600], 0),
    (16, 2, 64, [4500, 90], [66, 3], 1000),
    (1, 1, 128, [4200], [513], 0),
    (2, 1, 32, [31, 0, 1000], [257, 1, 300], 33),
])
def test_many_rows_on_long_contexts(dtype, d, hq, hkv, page, lengths, new, window):
    run, batch, q, out = attend_case(dtype, d, hq, hkv, page, lengths, new, window=window, seed=sum(new))
    run.check_attend(batch, q, out)
    assert torch.equal(out, run.cache.attend(batch, q))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv,page,lengths,new,window", [
    (8, 1, 32, [5000], [12], 0),
    (16, 1, 64, [3000, 10], [32, 1], 0),
    (4, 2, 96, [100, 2000, 0], [20, 60, 9], 0),
    (33, 1, 64, [700], [1], 0),
    (64, 1, 32, [2100, 40, 0], [1, 8, 3], 0),
    (8, 2, 64, [3000, 31], [40, 17], 1025),
    (5, 1, 64, [0], [102], 0),
])
def test_blocks_of_few_rows(dtype, d, hq, hkv, page, lengths, new, window):
    run, batch, q, out = attend_case(dtype, d, hq, hkv, page, lengths, new, window=window, seed=sum(new) + 1)
    run.check_attend(batch, q, out)
    assert torch.equal(out, run.cache.attend(batch, q))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [1, 24, 140])
def test_a_missing_page_and_a_nan_far_from_the_ends(dtype, d, new):
    """A page that does not exist in the middle of a long context hides its keys only, and a NaN key or value reaches the rows of its sequence only."""
    run, batch, q, _ = attend_case(dtype, d, 4, 1, 32, [2000, 1300], [new, new], seed=new)
    table = run.table.copy()
    table[0, 30], table[1, 17:20] = -1, 10 ** 9
    again = run.batch([2000, 1300], [new, new], table)
    plain = run.cache.attend(again, q)
    run.check_attend(again, q, plain)
    before = run.cache.pages.clone()
    for which in range(2):
        k, v = run.rows(1, 1), run.rows(1, 1)
        (k if which else v)[0, 0, 3] = math.nan
        one = run.batch([0, 801], [0, 1], table)
        run.cache.append(one, k, v)
        out = run.cache.attend(run.batch([2000, 1300], [new, new], table), q)
        assert torch.equal(out[:new], plain[:new])
        assert bool(torch.isnan(out[new:]).all())
        run.cache.pages.copy_(before)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 30, 300])
def test_pages_behind_the_window_may_be_gone(dtype, new):
    """What a window has left behind may be handed out again: taking those pages from the table changes nothing."""
    run, batch, q, out = attend_case(dtype, 64, 4, 2, 32, [1500, 700], [new, new], window=200, seed=new + 5)
    run.check_attend(batch, q, out)
    table = run.table.copy()
    for s, n in enumerate((1500, 700)):
        table[s, :(n - 199) // 32] = -1
    assert torch.equal(run.cache.attend(run.batch([1500, 700], [new, new], table), q), out)


@pytest.mark.parametrize("longest", [3, 40])
def test_many_sequences(longest):
    """More sequences than a wave has lanes, many without a new token: every token at its place, every row with its own keys."""
    rng = np.random.default_rng(longest)
    seqs = 210
    lengths = rng.integers(0, 70, seqs).tolist()
    new = rng.integers(0, 3, seqs).tolist()
    new[0], new[67], new[130], new[209] = 0, longest, 0, longest
    run, batch, q, out = attend_case("bf16", 64, 2, 1, 32, lengths, new, seed=longest)
    run.check_attend(batch, q, out)
    k, v = run.rows(sum(new), 1), run.rows(sum(new), 1)
    run.append(batch, k, v)
    run.check_bytes()
    got_k, got_v = run.cache.read(batch)
    for s in (1, 63, 64, 67, 128, 209):
        wk, wv, _ = run.values(s, 0, lengths[s] + new[s])
        rows = slice(run.offsets[s], run.offsets[s + 1])
        assert torch.equal(got_k[rows, 0].cpu(), torch.from_numpy(wk[lengths[s]:]).to(run.ty))
        assert torch.equal(got_v[rows, 0].cpu(), torch.from_numpy(wv[lengths[s]:]).to(run.ty))


@pytest.mark.parametrize("new", [1, 5, 130])
def test_a_call_that_names_more_than_there_is(new):
    """Bounds above what the arrays hold choose other kernels and splits, and give the same rows within the tolerance; rows of no sequence stay."""
    run, batch, q, out = attend_case("bf16", 128, 4, 1, 64, [900, 20], [new, 2], seed=new)
    n = new + 2
    more = torch.cat([q, q[:1].expand(700, -1, -1)])
    wide = paged.PagedBatch(batch.lengths, batch.new_offsets, batch.page_table, n + 700, 600, 5000)
    got = torch.full((n + 700, 4, 128), 3.0, device=DEV, dtype=torch.bfloat16)
    run.cache.attend(wide, more, out=got)
    run.check_attend(batch, q, got[:n])
    assert bool((got[n:] == 3).all())


def test_arrays_that_break_their_promises_stay_in_bounds():
    """Lengths below 0 and above the bound, offsets that fall or pass the rows: what the host named bounds everything, rows of sound sequences are right."""
    run, batch, q, out = attend_case("bf16", 64, 4, 1, 32, [200, 100, 50], [2, 2, 2], seed=8)
    before = run.cache.pages.clone()
    n_pages = run.cache.pages.shape[0]
    odd = paged.PagedBatch(i32([200, -7, 2 ** 31 - 1]), i32([0, 2, 1, 2 ** 31 - 1]), batch.page_table, 6, 2, 202)
    got = torch.full_like(q, 9.0)
    run.cache.attend(odd, q, out=got)
    assert torch.equal(got[0], out[0])
    odd_rows = run.rows(6, 1)
    run.cache.append(odd, odd_rows, odd_rows)
    run.cache.read(odd)
    torch.cuda.synchronize()
    changed = (run.cache.pages != before).any(1).nonzero().flatten().tolist()
    assert set(changed) <= set(run.table.flatten().tolist()) and len(changed) <= n_pages


def test_two_caches_on_two_streams_and_two_graphs_of_one_cache():
    cases = [attend_case("bf16", 128, 8, 2, 64, [3000, 900], [1, 1], seed=1), attend_case("f32", 64, 4, 1, 32, [700], [200], seed=2)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for stream, (run, batch, q, out) in zip(streams, cases):
            with torch.cuda.stream(stream):
                got.append(run.cache.attend(batch, q))
        torch.cuda.synchronize()
        for x, (run, batch, q, out) in zip(got, cases):
            assert torch.equal(x, out)
    # two graphs share the cache and its workspace: they run one after the other on a stream
    run, batch, q, out = cases[0]
    q2 = run.rows(2, 8)
    want2 = run.cache.attend(batch, q2)
    outs = [torch.empty_like(q), torch.empty_like(q)]
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    torch.cuda.synchronize()
    for graph, x, o in zip(graphs, (q, q2), outs):
        with torch.cuda.graph(graph, stream=streams[0]):
            run.cache.attend(batch, x, out=o)
    for _ in range(4):
        for o in outs:
            o.zero_()
        graphs[0].replay()
        graphs[1].replay()
        run.cache.attend(batch, q2)      # eager work of the same cache between the replays
        graphs[0].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], out) and torch.equal(outs[1], want2)


def test_layers_on_one_workspace():
    """Two layers, other head counts and types, on one workspace: eager and captured, what each gives alone."""
    runs = [attend_case("bf16", 128, 8, 2, 64, [3000, 900], [1, 1], seed=1), attend_case("f32", 64, 4, 1, 32, [700, 2000], [3, 40], seed=2)]
    size = max(paged.PagedKVCache.workspace_size(run.cfg) for run, _, _, _ in runs)
    workspace = torch.empty(size, dtype=torch.uint8, device=DEV)
    layers = [paged.PagedKVCache(run.cfg, DEV, pages=run.cache.pages, workspace=workspace) for run, _, _, _ in runs]
    for _ in range(2):
        for layer, (run, batch, q, out) in zip(layers, runs):
            assert torch.equal(layer.attend(batch, q), out)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        outs = [layer.attend(batch, q) for layer, (run, batch, q, out) in zip(layers, runs)]
    for _ in range(3):
        for x in outs:
            x.zero_()
        layers[0].attend(runs[0][1], runs[0][2])
        graph.replay()
        torch.cuda.synchronize()
        for x, (run, batch, q, out) in zip(outs, runs):
            assert torch.equal(x, out)
    with pytest.raises(AssertionError):
        paged.PagedKVCache(runs[0][0].cfg, DEV, pages=runs[0][0].cache.pages, workspace=workspace[:1000])
    with pytest.raises(AssertionError):
        paged.PagedKVCache(runs[0][0].cfg, DEV, pages=runs[0][0].cache.pages, workspace=workspace.to(torch.int8))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,lengths,new,empty", [
    (300, 1, [100], [3], 0),
    (1024, 1, [40, 700], [2, 1], 0),
    (512, 2, [90, 0], [9, 3], 300),
])
def test_many_heads_of_a_group(dtype, hq, hkv, lengths, new, empty):
    """More query heads of a KV head than a workgroup has rows."""
    run, batch, q, out = attend_case(dtype, 64, hq, hkv, 32, lengths + [0] * empty, new + [0] * empty, seed=hq)
    run.check_attend(batch, q, out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new,empty", [(1, 0), (40, 0), (300, 300)])
def test_pages_behind_four_gigabytes(dtype, new, empty):
    """Pages at the end of a pool of more than 2^33 bytes hold and give what the same pages of a small pool do."""
    lengths, counts = [500] + [0] * empty, [new] + [0] * empty
    run, batch, q, out = attend_case(dtype, 128, 4, 2, 64, lengths, counts, seed=new)
    n = (1 << 33) // B.cascade_paged_page_bytes(run.cfg) + 1000
    cfg = B.make_paged_config(n_q_heads=4, n_kv_heads=2, head_dim=128, dtype=run.cfg.dtype, page_size=64, n_pages=n, max_seqs=len(lengths))
    cache = paged.PagedKVCache(cfg, DEV)
    few = run.cache.pages.shape[0]
    cache.pages[n - few:] = run.cache.pages
    table = np.where(run.table >= 0, run.table + (n - few), -1)
    there = paged.PagedBatch(batch.lengths, batch.new_offsets, i32(table), batch.n_tokens, batch.max_new, batch.max_length)
    assert torch.equal(cache.attend(there, q), out)
    k, v = run.rows(new, 2), run.rows(new, 2)
    run.cache.append(batch, k, v)
    cache.append(there, k, v)
    assert torch.equal(cache.pages[n - few:], run.cache.pages)
    for x, y in zip(cache.read(there), run.cache.read(batch)):
        assert torch.equal(x, y)
    cache.close()
