"""The torch layer of the norms and the paged cache without a GPU: handles, devices, bounds and gradients."""
import gc

import pytest
import torch

from paper_2406_17808_amd import binding as B
from paper_2406_17808_amd import paged


def cfg(**kw):
    base = dict(n_q_heads=8, n_kv_heads=2, head_dim=64, dtype=B.CASCADE_BF16, page_size=64, n_pages=10, max_seqs=4)
    base.update(kw)
    return B.make_paged_config(**base)


@pytest.fixture(scope="module", autouse=True)
def lib():
    import os
    if not os.path.exists(B.library_path()):
        from paper_2406_17808_amd.build import build_library
        build_library()
    return B.load_library()


@pytest.mark.parametrize("end", ["close", "delete"])
def test_ending_a_cache_does_not_wait_for_the_device(monkeypatch, end):
    """A cache may be collected while a stream is being captured, where a synchronisation is an error that ends the capture; there is nothing to
    wait for, its context is a structure of the host."""
    waits = []
    monkeypatch.setattr(torch.cuda, "synchronize", lambda *a: waits.append(a))
    monkeypatch.setattr(paged.B, "cascade_paged_destroy", lambda ctx: waits.append("destroyed") if ctx == 7 else None)
    cache = paged.PagedKVCache.__new__(paged.PagedKVCache)
    cache.ctx, cache.device = 7, torch.device("cuda", 0)
    if end == "close":
        cache.close()
        assert cache.ctx is None
    else:
        del cache
        gc.collect()
    assert waits == ["destroyed"]


def test_devices_without_a_number_are_the_current_one(monkeypatch):
    monkeypatch.setattr(paged, "_current_device", lambda: 3)
    assert paged._numbered("cuda") == torch.device("cuda", 3) == paged._numbered(torch.device("cuda"))
    assert paged._numbered("cuda:1") == torch.device("cuda", 1) and paged._numbered("cpu") == torch.device("cpu")


def test_what_would_need_a_backward_is_refused():
    """Outputs have no gradient: with inputs that require one they would be cut from the graph without a word."""
    plain, leaf = torch.zeros(3), torch.zeros(3, requires_grad=True)
    paged._serving_only(plain, None)
    for args in ((leaf,), (plain, leaf), (None, plain, leaf * 2)):
        with pytest.raises(RuntimeError, match="backward"):
            paged._serving_only(*args)
        with torch.no_grad():
            paged._serving_only(*args)
        with torch.inference_mode():
            paged._serving_only(*args)


FIELDS = dict(n_q_heads=8, n_kv_heads=2, head_dim=64, dtype=1, page_size=64, max_seqs=4, window=0)


@pytest.mark.parametrize("field", FIELDS)
def test_numbers_of_a_configuration_are_not_cut_to_32_bits(field):
    for beyond in (FIELDS[field] + 2 ** 32, FIELDS[field] - 2 ** 32, 2 ** 31):
        with pytest.raises(B.CascadeError) as e:
            cfg(**{field: beyond})
        assert e.value.code == B.CASCADE_E_INVALID_CONFIG and field in str(e.value)


@pytest.mark.parametrize("field", ["n_tokens", "max_new", "max_length"])
def test_bounds_of_a_batch_are_not_cut_to_32_bits(field):
    """2^32 + 100 must not become a bound of 100, behind which keys would not be seen."""
    bounds = dict(n_tokens=6, max_new=4, max_length=100)
    paged._batch_bounds(**bounds)
    for beyond in (bounds[field] + 2 ** 32, bounds[field] - 2 ** 32, 2 ** 31):
        with pytest.raises(B.CascadeError) as e:
            paged._batch_bounds(**dict(bounds, **{field: beyond}))
        assert e.value.code == B.CASCADE_E_BAD_ARG and field in str(e.value)
