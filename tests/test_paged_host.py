"""The norms and the paged cache without a GPU: what is refused, and the places and numbers of the pages on the host."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

import paged_model as M
from paper_2406_17808_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CLANG = "/opt/rocm/lib/llvm/bin/clang++"


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.library_path()):
        from paper_2406_17808_amd.build import build_library
        build_library()
    return B.load_library()


@pytest.mark.skipif(not os.path.exists(CLANG), reason="the ROCm clang is not installed")
def test_places_and_numbers_under_sanitizers(tmp_path):
    exe = str(tmp_path / "paged_format")
    subprocess.check_call([CLANG, "-x", "c++", "-std=c++17", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-g", "-O1", "-Wall",
                           "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", os.path.join(ROOT, "tests", "native", "paged_format.cpp"), "-o", exe, "-lm"])
    env = dict(os.environ, ASAN_OPTIONS="verify_asan_link_order=0:abort_on_error=0")
    env.pop("LD_PRELOAD", None)
    res = subprocess.run([exe], env=env, capture_output=True, text=True, timeout=300)
    assert res.returncode == 0 and "0 failed" in res.stdout, res.stdout + res.stderr


def test_struct_sizes(lib):
    assert ctypes.sizeof(B.cascade_norm_rope_args) == 8 * 4 + 4 * 8 + 4 * 8 + 5 * 8
    assert ctypes.sizeof(B.cascade_paged_config) == 6 * 4 + 8 + 2 * 4
    assert ctypes.sizeof(B.cascade_paged_batch) == 4 * 4 + 4 * 8


def _cfg(**kw):
    base = dict(n_q_heads=8, n_kv_heads=2, head_dim=64, dtype=B.CASCADE_BF16, page_size=64, n_pages=10, max_seqs=4)
    base.update(kw)
    return B.make_paged_config(**base)


@pytest.mark.parametrize("kw,code", [
    (dict(n_q_heads=0), B.CASCADE_E_INVALID_CONFIG), (dict(n_q_heads=7), B.CASCADE_E_INVALID_CONFIG), (dict(n_kv_heads=0), B.CASCADE_E_INVALID_CONFIG),
    (dict(n_kv_heads=-2), B.CASCADE_E_INVALID_CONFIG), (dict(n_q_heads=4096), B.CASCADE_E_INVALID_CONFIG),
    (dict(head_dim=96), B.CASCADE_E_UNSUPPORTED), (dict(dtype=2), B.CASCADE_E_UNSUPPORTED), (dict(page_size=0), B.CASCADE_E_INVALID_CONFIG),
    (dict(page_size=48), B.CASCADE_E_INVALID_CONFIG), (dict(page_size=65536 + 32), B.CASCADE_E_INVALID_CONFIG), (dict(n_pages=0), B.CASCADE_E_INVALID_CONFIG),
    (dict(n_pages=2 ** 31), B.CASCADE_E_INVALID_CONFIG), (dict(max_seqs=0), B.CASCADE_E_INVALID_CONFIG), (dict(window=-1), B.CASCADE_E_INVALID_CONFIG),
    (dict(softmax_scale=-1.0), B.CASCADE_E_INVALID_CONFIG), (dict(softmax_scale=float("nan")), B.CASCADE_E_INVALID_CONFIG),
])
def test_invalid_configurations(lib, kw, code):
    cfg = _cfg(**kw)
    assert B.cascade_paged_page_bytes(cfg) == 0 and B.cascade_paged_workspace_bytes(cfg) == 0
    with pytest.raises(B.CascadeError) as e:
        B.cascade_paged_init(cfg, 256, 256, 1 << 40)
    assert e.value.code == code and len(str(e.value)) > 30


def test_sizes(lib):
    assert B.cascade_paged_page_bytes(_cfg()) == 2 * 2 * M.group_bytes(64) == 2 * 2 * 2176
    assert B.cascade_paged_page_bytes(_cfg(head_dim=128, page_size=96, n_kv_heads=8)) == 8 * 3 * 4352
    assert B.cascade_paged_workspace_bytes(_cfg()) > 0
    assert B.cascade_rope_table_bytes(1, 2) == 257 * 16 and B.cascade_rope_table_bytes(1 << 20, 128) == (256 + 4096) * 64 * 16
    for n, d in ((0, 64), (-1, 64), (2 ** 31 + 1, 64), (16, 0), (16, 63), (16, 258)):
        assert B.cascade_rope_table_bytes(n, d) == 0


def _refused(code, call, *args, **kw):
    with pytest.raises(B.CascadeError) as e:
        call(*args, **kw)
    assert e.value.code == code and len(str(e.value)) > 30, str(e.value)


def test_init_and_table_refusals(lib):
    need = B.cascade_paged_workspace_bytes(_cfg())
    _refused(B.CASCADE_E_NULL_ARG, B.cascade_paged_init, _cfg(), 0, 256, need)
    _refused(B.CASCADE_E_NULL_ARG, B.cascade_paged_init, _cfg(), 256, 0, need)
    _refused(B.CASCADE_E_BAD_ARG, B.cascade_paged_init, _cfg(), 64, 256, need)
    _refused(B.CASCADE_E_BAD_ARG, B.cascade_paged_init, _cfg(), 256, 128, need)
    _refused(B.CASCADE_E_WORKSPACE_TOO_SMALL, B.cascade_paged_init, _cfg(), 256, 256, need - 1)
    _refused(B.CASCADE_E_BAD_ARG, B.cascade_paged_init, _cfg(), 256, 256, need, 8, 100)
    _refused(B.CASCADE_E_BAD_ARG, B.cascade_paged_init, _cfg(), 256, 256, need, 16, 0)
    assert lib.cascade_paged_init(None, 256, 256, need, None, 0, None) == B.CASCADE_E_NULL_ARG
    lib.cascade_paged_destroy(None)
    _refused(B.CASCADE_E_NULL_ARG, B.cascade_rope_table, 0, 1 << 30, 100, 64, 1e4)
    _refused(B.CASCADE_E_BAD_ARG, B.cascade_rope_table, 256, 1 << 30, 0, 64, 1e4)
    _refused(B.CASCADE_E_BAD_ARG, B.cascade_rope_table, 256, 1 << 30, 100, 63, 1e4)
    _refused(B.CASCADE_E_BAD_ARG, B.cascade_rope_table, 256, 1 << 30, 100, 64, 0.0)
    _refused(B.CASCADE_E_BAD_ARG, B.cascade_rope_table, 256, 1 << 30, 100, 64, float("inf"))
    _refused(B.CASCADE_E_BAD_ARG, B.cascade_rope_table, 264, 1 << 30, 100, 64, 1e4)
    _refused(B.CASCADE_E_WORKSPACE_TOO_SMALL, B.cascade_rope_table, 256, B.cascade_rope_table_bytes(100, 64) - 1, 100, 64, 1e4)


def _norm_args(**kw):
    a = B.cascade_norm_rope_args(dtype=B.CASCADE_BF16, head_dim=64, n_tokens=4, n_q_heads=4, n_k_heads=2, norm=1, eps=1e-6,
                                 dev_q=4096, dev_k=8192, dev_q_out=12288, dev_k_out=16384)
    for name, x in kw.items():
        setattr(a, name, x)
    return a


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=7), B.CASCADE_E_UNSUPPORTED), (dict(head_dim=0), B.CASCADE_E_UNSUPPORTED), (dict(head_dim=65), B.CASCADE_E_UNSUPPORTED),
    (dict(head_dim=258), B.CASCADE_E_UNSUPPORTED), (dict(n_tokens=-1), B.CASCADE_E_BAD_ARG), (dict(n_tokens=(1 << 20) + 1), B.CASCADE_E_BAD_ARG),
    (dict(n_q_heads=-1), B.CASCADE_E_BAD_ARG), (dict(n_k_heads=1025), B.CASCADE_E_BAD_ARG), (dict(norm=2), B.CASCADE_E_BAD_ARG),
    (dict(reserved=1), B.CASCADE_E_BAD_ARG), (dict(eps=-1.0), B.CASCADE_E_BAD_ARG), (dict(eps=float("nan")), B.CASCADE_E_BAD_ARG),
    (dict(dev_q=None), B.CASCADE_E_NULL_ARG), (dict(dev_k_out=None), B.CASCADE_E_NULL_ARG), (dict(dev_positions=64), B.CASCADE_E_NULL_ARG),
    (dict(dev_positions=64, dev_rope=256, rope_positions=0), B.CASCADE_E_BAD_ARG), (dict(dev_positions=66, dev_rope=256, rope_positions=9), B.CASCADE_E_BAD_ARG),
    (dict(dev_positions=64, dev_rope=264, rope_positions=9), B.CASCADE_E_BAD_ARG), (dict(q_stride=255), B.CASCADE_E_BAD_ARG),
    (dict(k_out_stride=-128), B.CASCADE_E_BAD_ARG), (dict(q_stride=1 << 41), B.CASCADE_E_BAD_ARG), (dict(dev_q=4097), B.CASCADE_E_BAD_ARG),
    (dict(dev_q_out=4096, q_out_stride=512), B.CASCADE_E_BAD_ARG), (dict(dev_k_weight=4097), B.CASCADE_E_BAD_ARG),
])
def test_norm_rope_refusals(lib, kw, code):
    _refused(code, B.cascade_norm_rope, _norm_args(**kw))


def test_norm_rope_without_work(lib):
    assert lib.cascade_norm_rope(None, None) == B.CASCADE_E_NULL_ARG
    B.cascade_norm_rope(_norm_args(n_tokens=0, dev_q=None))
    B.cascade_norm_rope(_norm_args(n_q_heads=0, n_k_heads=0, dev_q=None))


@pytest.fixture
def ctx(lib):
    if torch.cuda.is_available():
        pytest.skip("made-up pointers: without a GPU only")
    made = [B.cascade_paged_init(_cfg(), 256, 256, 1 << 40), B.cascade_paged_init(_cfg(), 256, 256, 1 << 40, 4096, 1000)]
    yield made
    for c in made:
        B.cascade_paged_destroy(c)


def _batch(**kw):
    b = B.cascade_paged_batch(n_seqs=2, n_tokens=6, max_new=4, max_length=100, dev_lengths=64, dev_new_offsets=128, dev_page_table=256, table_stride=3)
    for name, x in kw.items():
        setattr(b, name, x)
    return b


BATCH_REFUSALS = [
    (dict(n_seqs=-1), B.CASCADE_E_BAD_ARG), (dict(n_seqs=5), B.CASCADE_E_BAD_ARG), (dict(n_tokens=-1), B.CASCADE_E_BAD_ARG),
    (dict(n_tokens=(1 << 20) + 1), B.CASCADE_E_BAD_ARG), (dict(max_new=-1), B.CASCADE_E_BAD_ARG), (dict(max_length=-1), B.CASCADE_E_BAD_ARG),
    (dict(max_length=2 ** 31 - 1), B.CASCADE_E_BAD_ARG), (dict(table_stride=-1), B.CASCADE_E_BAD_ARG), (dict(dev_lengths=None), B.CASCADE_E_NULL_ARG),
    (dict(dev_new_offsets=None), B.CASCADE_E_NULL_ARG), (dict(dev_page_table=None), B.CASCADE_E_NULL_ARG), (dict(dev_lengths=66), B.CASCADE_E_BAD_ARG),
]


@pytest.mark.parametrize("kw,code", BATCH_REFUSALS)
def test_batch_refusals(ctx, kw, code):
    b = _batch(**kw)
    _refused(code, B.cascade_paged_append, ctx[0], b, 4096, 0, 4096, 0)
    _refused(code, B.cascade_paged_attend, ctx[0], b, 4096, 0, 8192)
    _refused(code, B.cascade_paged_read, ctx[0], b, 4096, 8192)


def test_call_refusals(ctx, lib):
    plain, rope = ctx
    b = _batch()
    bad, null = B.CASCADE_E_BAD_ARG, B.CASCADE_E_NULL_ARG
    _refused(null, B.cascade_paged_append, plain, b, 0, 0, 4096, 0)
    _refused(null, B.cascade_paged_append, plain, b, 4096, 0, 0, 0)
    _refused(bad, B.cascade_paged_append, plain, b, 4100, 0, 4096, 0)
    _refused(bad, B.cascade_paged_append, plain, b, 4096, 127, 4096, 0)
    _refused(bad, B.cascade_paged_append, plain, b, 4096, 0, 4096, 132)
    _refused(bad, B.cascade_paged_append, plain, b, 4096, 0, 4096, 0, 4096, 0, 8192)      # queries without a table
    _refused(null, B.cascade_paged_append, rope, b, 4096, 0, 4096, 0, 4096, 0, 0)
    _refused(bad, B.cascade_paged_append, rope, b, 4096, 0, 4096, 0, 4096, 1024, 4096)     # in place, rows apart
    _refused(bad, B.cascade_paged_append, rope, _batch(max_length=1001), 4096, 0, 4096, 0)
    _refused(null, B.cascade_paged_attend, plain, b, 0, 0, 8192)
    _refused(null, B.cascade_paged_attend, plain, b, 4096, 0, 0)
    _refused(bad, B.cascade_paged_attend, plain, b, 4096, 0, 4096)
    _refused(bad, B.cascade_paged_attend, plain, b, 4096, 500, 8192)
    _refused(bad, B.cascade_paged_attend, plain, b, 4096, 0, 8200)
    _refused(bad, B.cascade_paged_read, plain, b, 4100, 8192)
    for call, args in ((lib.cascade_paged_append, (None, 1, 0, 1, 0, None, 0, None, None)), (lib.cascade_paged_attend, (None, 1, 0, 1, None)),
                       (lib.cascade_paged_read, (None, 1, 1, None))):
        assert call(None, *args) == null and call(plain, *args) == null
    # nothing to do is no error, whatever the arrays
    for empty in (_batch(n_tokens=0), _batch(n_seqs=0, dev_lengths=None), _batch(max_new=0)):
        B.cascade_paged_append(plain, empty, 0, 0, 0, 0)
        B.cascade_paged_attend(plain, empty, 0, 0, 0)
        B.cascade_paged_read(plain, empty)
    # everything in order, and no device: an error and no launch
    _refused(B.CASCADE_E_HIP, B.cascade_paged_attend, plain, b, 4096, 0, 8192)


def test_model_rounds_to_the_nearest_code():
    """The tests' own oracle against a search over all codes."""
    rng = np.random.default_rng(0)
    y = np.concatenate([rng.uniform(-8, 8, 4000), np.round(rng.uniform(-8, 8, 1000) * 8) / 8])
    dist = np.abs(y[:, None] - M.VALUES[None])
    assert (np.abs(y - M.VALUES[M.nearest_codes(y)]) == dist.min(1)).all()
    codes, byte = M.quantise_k(y.reshape(-1, 1, 8).repeat(4, 1).reshape(-1, 32))
    assert byte.shape == (625, 1)
    assert (np.abs(M.k_values(codes, byte) - y.reshape(-1, 1, 8).repeat(4, 1).reshape(-1, 32)) <= 2.0 ** (byte.astype(float) - 127) * 1.0).all()


def test_arrays_whose_tokens_share_memory_are_refused():
    """An expanded array has stride 0, which the calls take for contiguous: it must not get that far."""
    import torch
    from paper_2406_17808_amd import paged
    one = torch.zeros((1, 2, 64))
    assert paged._rows(one, one.device, one.dtype, 1, 2, 64) == 0
    assert paged._rows(torch.zeros((3, 5, 64))[:, 1:3], one.device, one.dtype, 3, 2, 64) == 5 * 64
    with pytest.raises(AssertionError):
        paged._rows(one.expand(5, -1, -1), one.device, one.dtype, 5, 2, 64)
    with pytest.raises(AssertionError):
        paged._rows(torch.zeros(2 * 64 + 64 * 4).as_strided((5, 2, 64), (64, 64, 1)), one.device, one.dtype, 5, 2, 64)
