"""Handles of the paged cache on the GPU: dropped while a stream is captured or busy."""
import gc

import pytest
import torch

from paper_2406_17808_amd import paged
from test_gpu_paged import DEV, attend_case

pytestmark = pytest.mark.gpu


def test_a_cache_collected_during_a_capture():
    """Another cache ends while a step is captured: the capture goes on, and its replays give what eager calls give."""
    run, batch, q, out = attend_case("bf16", 128, 8, 2, 64, [3000, 900], [1, 1], seed=1)
    dropped, _, _, _ = attend_case("f32", 64, 4, 1, 32, [40], [1], seed=2)
    got, stream = torch.zeros_like(q), torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        del dropped
        gc.collect()
        run.cache.attend(batch, q, out=got)
    for _ in range(3):
        got.zero_()
        assert torch.equal(run.cache.attend(batch, q), out)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, out)


@pytest.mark.parametrize("own_pages", [True, False])
def test_a_cache_dropped_while_another_stream_still_uses_it(own_pages):
    """Its arrays are not handed out again before the work of that stream is done."""
    run, batch, q, out = attend_case("bf16", 128, 8, 2, 64, [700], [1], seed=3)
    pages = None if own_pages else torch.empty_like(run.cache.pages)
    cache = paged.PagedKVCache(run.cfg, DEV, pages=pages)
    cache.pages.copy_(run.cache.pages)
    rope = paged.RopeTable(1000, 128, 1e4, DEV)
    rotating = paged.PagedKVCache(run.cfg, DEV, pages=cache.pages, rope=rope, workspace=cache.workspace)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    held = {x.data_ptr(): x.numel() for x in (cache.pages, cache.workspace, rope.table)}
    with torch.cuda.stream(side):
        torch.cuda._sleep(400_000_000)      # a fifth of a second
        got = cache.attend(batch, q)
        rotating.append(batch, run.rows(1, 2), run.rows(1, 2))
    del cache, rotating, pages, rope
    others = [torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV) for n in held.values() for _ in range(2)]
    if side.query():
        pytest.skip("the stream was done before the arrays were asked for")
    assert not {x.data_ptr() for x in others} & set(held)
    side.synchronize()
    assert torch.equal(got, out)


def test_a_device_without_a_number():
    """"cuda" is the current device, for tables and caches as for tensors."""
    run, batch, q, out = attend_case("bf16", 64, 4, 2, 32, [40], [3], seed=4)
    rope = paged.RopeTable(100, 64, 1e4, "cuda")
    cache = paged.PagedKVCache(run.cfg, "cuda", rope=rope)
    assert cache.device == cache.pages.device == rope.device == torch.device("cuda", torch.cuda.current_device())
    cache.pages.copy_(run.cache.pages)
    assert torch.equal(cache.attend(batch, q), out)
    paged.qk_norm_rope(q, positions=torch.arange(3, device="cuda", dtype=torch.int32), rope=rope)
    paged.PagedKVCache(run.cfg, torch.device("cuda"), pages=run.cache.pages).append(batch, q[:, :2], q[:, 2:])


def test_inputs_that_require_gradients_are_refused():
    run, batch, q, out = attend_case("f32", 64, 4, 2, 32, [40], [3], seed=5)
    rope = paged.RopeTable(100, 64, 1e4, DEV)
    rotating = paged.PagedKVCache(run.cfg, DEV, pages=run.cache.pages, rope=rope)
    k, v, w = run.rows(3, 2), run.rows(3, 2), run.rows(1, 1)[0, 0]
    leaf = lambda x: x.clone().requires_grad_()  # noqa: E731
    calls = [lambda: paged.qk_norm_rope(leaf(q)), lambda: paged.qk_norm_rope(q, leaf(k)), lambda: paged.qk_norm_rope(q, q_weight=leaf(w)),
             lambda: paged.qk_norm_rope(q, k, k_weight=leaf(w)), lambda: rotating.append(batch, leaf(k), v), lambda: rotating.append(batch, k, leaf(v)),
             lambda: rotating.append(batch, k, v, q=leaf(q)), lambda: rotating.attend(batch, leaf(q))]
    pages = run.cache.pages.clone()
    for call in calls:
        with pytest.raises(RuntimeError, match="backward"):
            call()
    assert torch.equal(run.cache.pages, pages)
    with torch.no_grad():
        for call in calls:
            call()
    assert torch.equal(rotating.attend(batch, leaf(q).detach()), rotating.attend(batch, q))
