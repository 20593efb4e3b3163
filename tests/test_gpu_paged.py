"""The paged cache in 4 bits and the per-head norms on the GPU against plain implementations in 64 bits."""
import math

import numpy as np
import pytest
import torch

import paged_model as M
from paper_2406_17808_amd import binding as B
from paper_2406_17808_amd import paged

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
CODE = {"bf16": B.CASCADE_BF16, "f32": B.CASCADE_F32}


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def f64(x):
    return x.double().cpu().numpy()


# ---------------------------------------------------------------- norms

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,hq,hk,d", [(1, 32, 8, 128), (5, 16, 2, 64), (3, 3, 1, 80), (33, 4, 4, 256), (2, 5, 0, 96), (7, 1, 1, 16),
                                            (4, 2, 3, 6), (3, 1, 1, 2), (2, 3, 2, 250), (40, 40, 8, 128), (2, 200, 100, 64), (300, 2, 1, 32)])
@pytest.mark.parametrize("norm,rotated,weights,fused", [(True, True, True, True), (True, False, True, False), (False, True, False, True),
                                                        (True, True, False, False), (False, False, False, False)])
def test_norm_rope(dtype, tokens, hq, hk, d, norm, rotated, weights, fused):
    ty = TYPES[dtype]
    gen = torch.Generator(device=DEV).manual_seed(tokens * 1000 + d)
    x = (torch.randn((tokens, hq + 2 * hk, d), generator=gen, device=DEV) * 3).to(ty)
    q, k = x[:, :hq], x[:, hq:hq + hk]
    if not fused:
        q, k = q.contiguous(), k.contiguous()
    w = (1 + 0.3 * torch.randn((2, d), generator=gen, device=DEV)).to(ty)
    base, n_pos = 500000.0, 1 << 20
    rope = paged.RopeTable(n_pos, d, base, DEV) if rotated else None
    pos = torch.randint(0, n_pos, (tokens,), generator=gen, device=DEV, dtype=torch.int32) if rotated else None
    if rotated:
        pos[0] = n_pos - 1
    before = x.clone()
    got_q, got_k = paged.qk_norm_rope(q, k if hk else None, w[0] if weights else None, w[1].contiguous() if weights and hk else None, eps=1e-5, norm=norm,
                                      positions=pos, rope=rope) if norm or not weights else (None, None)
    assert torch.equal(x, before)
    for got, src, wt in ((got_q, q, w[0]), (got_k, k, w[1])):
        if src.shape[1] == 0:
            continue
        y = M.norm_rope(f64(src), f64(wt) if weights else None, 1e-5, norm, None, None)
        want = M.rotate(y, pos.cpu().numpy(), base) if rotated else y
        half = d // 2
        size = np.abs(y[..., :half]) + np.abs(y[..., half:])
        size = np.concatenate([size, size], -1)
        # at most 20 additions in a thread and between threads (half of their relative error reaches the root), mean, eps, root, division, weight,
        # product, cosine and sine, two products and a sum of the rotation: below 24 roundings of 2^-24 of the pair's size
        tol = M.HALF_STEP[ty] * np.abs(want) + 24 * 2.0 ** -24 * size
        if not norm and not rotated:
            tol = 0.0
        assert (np.abs(f64(got) - want) <= tol).all()


def test_norm_rope_in_place_and_strided_outputs():
    gen = torch.Generator(device=DEV).manual_seed(3)
    x = torch.randn((9, 40, 128), generator=gen, device=DEV).bfloat16()
    want_q, want_k = paged.qk_norm_rope(x[:, :32], x[:, 32:])
    wide = torch.full((9, 44, 128), 7.0, device=DEV, dtype=torch.bfloat16)
    got_q, got_k = paged.qk_norm_rope(x[:, :32], x[:, 32:], q_out=wide[:, 2:34], k_out=wide[:, 34:42])
    assert torch.equal(got_q, want_q) and torch.equal(got_k, want_k)
    assert bool((wide[:, :2] == 7).all()) and bool((wide[:, 42:] == 7).all())
    paged.qk_norm_rope(x[:, :32], x[:, 32:], q_out=x[:, :32], k_out=x[:, 32:])
    assert torch.equal(x[:, :32], want_q) and torch.equal(x[:, 32:], want_k)


def test_norm_rope_unaligned_rows_and_outside_positions():
    """Rows off the 16-byte grid give what aligned ones give; a position behind the table, or below 0, gives NaN in its token alone."""
    gen = torch.Generator(device=DEV).manual_seed(4)
    flat = torch.randn(6 * 4 * 64 + 1, generator=gen, device=DEV)
    x = flat[1:].view(6, 4, 64)
    rope = paged.RopeTable(1000, 64, 10000.0, DEV)
    pos = i32([0, 999, 1000, -1, 2 ** 31 - 1, 5])
    got, _ = paged.qk_norm_rope(x, positions=pos, rope=rope)
    same, _ = paged.qk_norm_rope(x.clone(), positions=pos, rope=rope)
    bad = torch.tensor([False, False, True, True, True, False])
    assert torch.equal(torch.isnan(got).all(-1).all(-1).cpu(), bad) and torch.equal(torch.isnan(got).any(-1).any(-1).cpu(), bad)
    y = M.norm_rope(f64(x), None, 1e-6, True, None, None)
    size = np.concatenate([np.abs(y[..., :32]) + np.abs(y[..., 32:])] * 2, -1)
    want = M.rotate(y, np.where(bad.numpy(), 0, pos.cpu().numpy()), 10000.0)
    for z in (got, same):
        assert (np.abs(f64(z) - want) <= 25 * 2.0 ** -24 * size)[~bad.numpy()].all()


def test_norm_of_zero_rows():
    x = torch.zeros((3, 2, 128), device=DEV, dtype=torch.bfloat16)
    x[1, 0, 5] = 2.0
    got, _ = paged.qk_norm_rope(x, eps=1e-6)
    assert bool((got[0] == 0).all()) and bool((got[2] == 0).all()) and bool((got[1, 1] == 0).all())
    assert abs(float(got[1, 0, 5]) - 2.0 / math.sqrt(4.0 / 128 + 1e-6)) < 2.0 ** -8 * 12


# ---------------------------------------------------------------- a cache and its model

class Run:
    """A paged cache on the GPU, and the bytes its pages should hold."""

    def __init__(self, dtype, d, hq, hkv, page, n_pages, seqs, window=0, rope_base=None, scale=0.0, fill=None, seed=0, rope_positions=4096):
        self.ty, self.d, self.hq, self.hkv, self.page, self.window, self.base = TYPES[dtype], d, hq, hkv, page, window, rope_base
        self.scale = scale or 1.0 / math.sqrt(d)
        cfg = B.make_paged_config(n_q_heads=hq, n_kv_heads=hkv, head_dim=d, dtype=CODE[dtype], page_size=page, n_pages=n_pages, max_seqs=max(seqs, 1),
                                  window=window, softmax_scale=scale)
        self.cfg = cfg
        nbytes = B.cascade_paged_page_bytes(cfg)
        assert nbytes == hkv * (page // 32) * M.group_bytes(d)
        self.gen = torch.Generator(device=DEV).manual_seed(seed)
        pages = torch.randint(0, 256, (n_pages, nbytes), generator=self.gen, device=DEV, dtype=torch.int32).to(torch.uint8)
        if fill is not None:
            pages.fill_(fill)
        self.want = pages.cpu().numpy().copy()
        self.cache = paged.PagedKVCache(cfg, DEV, pages=pages, rope=paged.RopeTable(rope_positions, d, rope_base, DEV) if rope_base else None)

    def rows(self, n, heads, gain=1.0):
        return (torch.randn((n, heads, self.d), generator=self.gen, device=DEV) * gain).to(self.ty)

    def batch(self, lengths, new, table, max_length=None, n_tokens=None, max_new=None):
        offsets = np.concatenate([[0], np.cumsum(new)]).tolist()
        self.offsets, self.lengths, self.new, self.table = offsets, list(lengths), list(new), np.asarray(table)
        self.max_length = max([a + b for a, b in zip(lengths, new)], default=0) if max_length is None else max_length
        return paged.PagedBatch(i32(lengths), i32(offsets), i32(table), offsets[-1] if n_tokens is None else n_tokens,
                                max(new, default=0) if max_new is None else max_new, self.max_length)

    def append(self, batch, k, v, **kw):
        M.append(self.want, self.table, self.lengths, self.offsets, self.page, self.hkv, f64(k), f64(v), self.max_length, self.base)
        return self.cache.append(batch, k, v, **kw)

    def check_bytes(self):
        got = self.cache.pages.cpu().numpy()
        bad = np.argwhere(got != self.want)
        assert not len(bad), (len(bad), bad[:5].tolist())

    def values(self, s, h, n):
        """K, V [n, d] of sequence s that its pages hold, and which of the positions exist."""
        d, size = self.d, M.group_bytes(self.d)
        k, v, there = np.zeros((n, d)), np.zeros((n, d)), np.zeros(n, bool)
        for p in range(n):
            slot = p // self.page
            if p >= self.max_length or slot >= self.table.shape[1] or not 0 <= self.table[s, slot] < len(self.want):
                continue
            there[p] = True
            at = (h * (self.page // 32) + p % self.page // 32) * size
            g, r = self.want[self.table[s, slot], at:at + size], p % 32
            c = np.arange(d)
            kc = g[c // 32 * 512 + r * 16 + c % 32 // 2] >> (4 * (c % 2)) & 15
            kb = g[32 * d + np.arange(d // 32) * 32 + r % 16 * 2 + r // 16]
            vc = g[16 * d + c // 64 * 1024 + r // 4 % 4 * 256 + c % 16 * 16 + c // 32 % 2 * 8 + r // 16 * 4 + r % 4] >> (4 * (c // 16 % 2)) & 15
            at = 33 * d + 2 * (r // 4 % 4 * 8 + r // 16 * 4 + r % 4)
            vs = float(np.array([int(g[at]) << 16 | int(g[at + 1]) << 24], np.uint32).view(np.float32)[0])
            k[p], v[p] = M.k_values(kc, kb), M.v_values(vc, np.float64(vs))
        return k, v, there

    def check_attend(self, batch, q, out):
        """All rows of all sequences against the model; returns nothing."""
        g = self.hq // self.hkv
        q64, out64 = f64(q), f64(out)
        for s in range(len(self.lengths)):
            a, e = self.offsets[s], self.offsets[s + 1]
            if a == e:
                continue
            n = self.lengths[s] + e - a
            pos = self.lengths[s] + np.arange(e - a)
            for h in range(self.hkv):
                k, v, there = self.values(s, h, n)
                j = np.arange(n)
                seen = (j[None] <= pos[:, None]) & there[None]
                if self.window:
                    seen &= j[None] > pos[:, None] - self.window
                for x in range(g):
                    rows = q64[a:e, h * g + x]
                    with np.errstate(invalid="ignore"):
                        want, weighted, spread = M.attend(rows, k, v, seen, self.scale)
                    tol = M.attend_tolerance(self.ty, want, weighted, spread, self.d, n)
                    got = out64[a:e, h * g + x]
                    off = np.abs(got - want) - tol
                    assert np.isfinite(got).all() and (off <= 0).all(), (s, h, x, float(off.max()), np.argwhere(off > 0)[:4].tolist())


def pages_for(rng, lengths, new, page, extra=2):
    """A page table with pages in any order, and the number of pages of the pool."""
    need = [-(-(a + b) // page) for a, b in zip(lengths, new)]
    order = rng.permutation(sum(need) + extra)
    table = np.full((len(need), max(max(need, default=0), 1)), -1)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    return table, sum(need) + extra


# ---------------------------------------------------------------- append and read

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("base", [None, 10000.0])
@pytest.mark.parametrize("hq,hkv,page,lengths,new", [
    (4, 2, 32, [0], [1]),
    (4, 2, 64, [31, 0, 63], [2, 0, 1]),
    (8, 8, 96, [5, 100, 0, 191], [40, 1, 33, 2]),
    (5, 1, 32, [17], [75]),
    (2, 2, 256, [250, 3], [20, 300]),
    (3, 3, 64, [0, 64, 1], [64, 64, 31]),
])
def test_append_writes_these_bytes_and_no_others(dtype, d, base, hq, hkv, page, lengths, new):
    rng = np.random.default_rng(sum(lengths) + sum(new))
    table, n_pages = pages_for(rng, lengths, new, page)
    run = Run(dtype, d, hq, hkv, page, n_pages, len(lengths), rope_base=base, seed=d + len(new))
    batch = run.batch(lengths, new, table)
    n = sum(new)
    qkv = run.rows(n, hq + 2 * hkv)      # a fused projection: rows of q, k and v lie apart
    q, k, v = qkv.split([hq, hkv, hkv], 1)
    q_out = run.append(batch, k, v, q=q if base else None)
    run.check_bytes()
    got_k, got_v = run.cache.read(batch)
    t = 0
    for s in range(len(lengths)):
        for h in range(hkv):
            wk, wv, _ = run.values(s, h, lengths[s] + new[s])
            rows = slice(run.offsets[s], run.offsets[s + 1])
            assert torch.equal(got_k[rows, h].cpu(), torch.from_numpy(wk[lengths[s]:]).to(run.ty))
            assert torch.equal(got_v[rows, h].cpu(), torch.from_numpy(wv[lengths[s]:]).to(run.ty))
    if base:
        pos = np.concatenate([np.arange(a, a + b) for a, b in zip(lengths, new)])
        x = f64(q)
        want = M.rotate(x, pos, base)
        size = np.concatenate([np.abs(x[..., :d // 2]) + np.abs(x[..., d // 2:])] * 2, -1)
        # cosine and sine, two products and their sum in 32 bits, then the type's rounding
        assert (np.abs(f64(q_out) - want) <= M.HALF_STEP[run.ty] * np.abs(want) + 4 * 2.0 ** -24 * size).all()


@pytest.mark.parametrize("new", [3, 64])
def test_append_borders_zeros_and_extremes(new):
    """Rows on the borders between codes, of zeros, with infinities and NaN, of the smallest and largest numbers."""
    for dtype in ("bf16", "f32"):
        run = Run(dtype, 64, 1, 1, 64, 3, 1, seed=1)
        batch = run.batch([9], [new], [[2, 0]])
        k, v = run.rows(new, 1), run.rows(new, 1)
        borders = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0], device=DEV).repeat(8)
        sign = torch.tensor([1.0, -1.0], device=DEV).repeat_interleave(8).repeat(4)
        k[0, 0], v[0, 0] = (borders * sign).to(run.ty), (torch.where(borders == 7, 6.0, borders) * sign).to(run.ty)
        k[1], v[1] = 0, 0
        k[2, 0, 3], v[2, 0, 40] = math.inf, -math.inf
        if new > 8:
            k[3, 0, 33], v[3, 0, 0] = math.nan, math.nan
            k[4], v[4] = 1e-38, 1e-38
            k[5, 0, :32], v[5] = 3e38, 3e38
            k[6, 0, 32:], v[6] = 0, 2.0 ** -97
            k[7], v[7] = -1e-40, -1e-40
            k[8] = (borders * 1.0078125).to(run.ty)
        run.append(batch, k, v)
        run.check_bytes()
        got_k, got_v = (f64(x) for x in run.cache.read(batch))
        wk, wv, _ = run.values(0, 0, 9 + new)
        np.testing.assert_array_equal(got_k[:, 0], torch.from_numpy(wk[9:]).to(run.ty).double().numpy())
        np.testing.assert_array_equal(got_v[:, 0], torch.from_numpy(wv[9:]).to(run.ty).double().numpy())


@pytest.mark.parametrize("new", [1, 70])
def test_append_leaves_out_what_has_no_place(new):
    """Pages that do not exist, positions behind the table or max_length, rows of no sequence: nothing else is written."""
    run = Run("bf16", 64, 2, 2, 32, 6, 4, seed=2)
    lengths, counts = [0, 30, 60, 5], [new, new, new, 2]
    table = [[-1, 4, 0], [1, 6, 2], [7, 7, 3], [5, -9, 2 ** 30]]
    batch = run.batch(lengths, counts, table, max_length=98, n_tokens=3 * new + 5, max_new=new + 1)
    k, v = run.rows(3 * new + 5, 2), run.rows(3 * new + 5, 2)
    run.append(batch, k, v)
    run.check_bytes()
    got_k, got_v = run.cache.read(batch)
    for s in range(4):
        for h in range(2):
            wk, wv, _ = run.values(s, h, lengths[s] + counts[s])
            rows = slice(run.offsets[s], run.offsets[s + 1])
            assert torch.equal(got_k[rows, h].cpu(), torch.from_numpy(wk[lengths[s]:]).to(run.ty))
            assert torch.equal(got_v[rows, h].cpu(), torch.from_numpy(wv[lengths[s]:]).to(run.ty))


def test_append_far_positions():
    """Angles of positions above 10^8 keep the codes of the definition in 64 bits."""
    run = Run("bf16", 128, 1, 1, 65536, 1, 1, rope_base=500000.0, rope_positions=(1 << 28), seed=5)
    table = np.full((1, 4096), -1)
    table[0, 4095] = 0
    batch = run.batch([(1 << 28) - 40], [40], table)
    run.append(batch, run.rows(40, 1), run.rows(40, 1))
    run.check_bytes()


# ---------------------------------------------------------------- attention

def attend_case(dtype, d, hq, hkv, page, lengths, new, window=0, q_gain=1.0, seed=0, fill=0xFF, scale=0.0):
    """Caches filled by append in a few calls, then one call of the new tokens."""
    rng = np.random.default_rng(seed)
    table, n_pages = pages_for(rng, lengths, new, page)
    run = Run(dtype, d, hq, hkv, page, n_pages, len(lengths), window=window, seed=seed, fill=fill, scale=scale)
    if sum(lengths):
        old = run.batch([0] * len(lengths), lengths, table)
        run.cache.append(old, run.rows(sum(lengths), hkv), run.rows(sum(lengths), hkv))
    batch = run.batch(lengths, new, table)
    run.cache.append(batch, run.rows(sum(new), hkv), run.rows(sum(new), hkv))
    run.want = run.cache.pages.cpu().numpy()      # what append writes has tests of its own
    q = run.rows(sum(new), hq, q_gain)
    out = run.cache.attend(batch, q)
    return run, batch, q, out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv,page,lengths,new", [
    (4, 1, 32, [0], [1]),
    (8, 2, 64, [1, 30, 31, 32, 33, 63], [1, 1, 1, 1, 1, 1]),
    (1, 1, 96, [500], [1]),
    (10, 2, 64, [100, 0, 257], [1, 0, 1]),
    (16, 1, 32, [333], [1]),
    (32, 1, 32, [129], [1]),
    (40, 1, 32, [70], [1]),
    (8, 2, 64, [40, 7], [3, 4]),
    (6, 2, 64, [0, 61, 200], [9, 2, 11]),
    (4, 4, 128, [3, 0, 90], [33, 64, 1]),
    (8, 1, 32, [31], [70]),
    (3, 1, 64, [0], [300]),
    (2, 1, 64, [1500], [1]),
    (4, 2, 64, [700, 0, 1], [130, 0, 257]),
])
def test_attend(dtype, d, hq, hkv, page, lengths, new):
    run, batch, q, out = attend_case(dtype, d, hq, hkv, page, lengths, new, seed=sum(new) + d)
    run.check_attend(batch, q, out)
    assert torch.equal(out, run.cache.attend(batch, q))      # the same bits again


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [1, 2, 31, 32, 33, 100])
@pytest.mark.parametrize("lengths,new", [([0, 200], [1, 1]), ([0, 77], [150, 70]), ([65, 3, 0], [5, 1, 0])])
def test_attend_window(dtype, window, lengths, new):
    run, batch, q, out = attend_case(dtype, 64, 8, 2, 32, lengths, new, window=window, seed=window)
    run.check_attend(batch, q, out)


@pytest.mark.parametrize("new", [1, 20, 90])
def test_attend_sharp_and_scaled(new):
    """Large logits (one key takes nearly all), and a scale of its own."""
    for gain, scale in ((30.0, 0.0), (1.0, 0.7), (0.0, 0.0)):
        for dtype in ("bf16", "f32"):
            run, batch, q, out = attend_case(dtype, 128, 4, 1, 64, [400], [new], q_gain=gain, scale=scale, seed=new)
            run.check_attend(batch, q, out)


@pytest.mark.parametrize("new", [1, 12, 80])
def test_attend_hidden_pages_and_rows_without_keys(new):
    """Keys on pages that do not exist, behind the table or behind max_length are not seen; a row that sees nothing gives zeros."""
    run, batch, q, _ = attend_case("bf16", 64, 4, 2, 32, [100, 40, 0, 64], [new] * 4, seed=7)
    table = run.table.copy()
    table[0, 1] = -1
    table[1, :] = len(run.want)
    table[2, :] = -5
    table[3, 0] = 2 ** 31 - 1
    again = run.batch([100, 40, 0, 64], [new] * 4, table, max_length=150)
    out = run.cache.attend(again, q)
    run.check_attend(again, q, out)
    assert bool((out[new:3 * new] == 0).all())
    short = run.batch([100, 40, 0, 64], [new] * 4, run.table[:, :1])
    run.check_attend(short, q, run.cache.attend(short, q))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 6, 90])
@pytest.mark.parametrize("window", [0, 40])
def test_nan_and_infinite_rows_reach_only_who_sees_them(dtype, new, window):
    run = Run(dtype, 64, 2, 1, 32, 12, 1, window=window, fill=0xFF, seed=new)
    table = [list(range(11, 0, -1))]
    n = 120 + new
    k, v, q = run.rows(n, 1), run.rows(n, 1), run.rows(new, 2)
    k[50, 0, 5], v[n - 2, 0, 7] = math.nan, math.inf
    old = run.batch([0], [n], table)
    run.cache.append(old, k, v)
    run.want = run.cache.pages.cpu().numpy()
    batch = run.batch([120], [new], table)
    out = run.cache.attend(batch, q)
    pos = torch.arange(120, n)
    sees = (pos >= n - 2) if window else torch.ones(new, dtype=torch.bool)      # key 50 is behind the window of every row
    assert torch.equal(torch.isnan(out).all(-1).all(-1).cpu(), sees) and torch.equal(torch.isnan(out).any(-1).any(-1).cpu(), sees)
    k[50], v[n - 2] = 0, 0
    run.cache.append(old, k, v)
    run.want = run.cache.pages.cpu().numpy()
    plain = run.cache.attend(run.batch([120], [new], table), q)
    run.check_attend(batch, q, plain)
    assert torch.equal(out[~sees.to(DEV)], plain[~sees.to(DEV)])


def test_rows_of_no_sequence_are_left_as_they_were():
    run, batch, q, _ = attend_case("bf16", 64, 2, 1, 32, [10, 20], [3, 40], seed=3)
    more = torch.cat([q, q[:9]])
    wide = paged.PagedBatch(batch.lengths, batch.new_offsets, batch.page_table, 52, 41, 60)
    out = torch.full((52, 2, 64), 5.0, device=DEV, dtype=torch.bfloat16)
    run.max_length = 60
    run.cache.attend(wide, more, out=out)
    run.check_attend(wide, q, out[:43])
    assert bool((out[43:] == 5).all())


# ---------------------------------------------------------------- together

def test_a_layer_step_by_step_and_captured():
    """Norms, append and attention as a layer calls them: a prompt in chunks of different lengths, then single tokens, eager and from a
    captured graph that follows the lengths; and the bytes do not depend on how a prefix was cut into calls."""
    d, hq, hkv, page, seqs = 128, 8, 2, 64, 3
    table = np.random.default_rng(0).permutation(3 * 6).reshape(3, 6)
    run = Run("bf16", d, hq, hkv, page, 20, seqs, rope_base=10000.0, seed=11, fill=0)
    other = Run("bf16", d, hq, hkv, page, 20, seqs, rope_base=10000.0, seed=11, fill=0)
    w = (1 + 0.2 * torch.randn((2, d), generator=run.gen, device=DEV)).bfloat16()
    total = [150, 97, 33]
    x = {s: run.rows(total[s] + 8, hq + 2 * hkv) for s in range(seqs)}

    def layer(r, batch, rows):
        q, k, v = rows.split([hq, hkv, hkv], 1)
        q, k = paged.qk_norm_rope(q, k, w[0], w[1])
        q = r.cache.append(batch, k, v, q=q)
        return q, r.cache.attend(batch, q)

    have = [0, 0, 0]
    for step in ([64, 97, 0], [1, 0, 33], [85, 0, 0]):
        batch = run.batch(have, step, table, max_length=384)
        rows = torch.cat([x[s][have[s]:have[s] + step[s]] for s in range(seqs)])
        q, out = layer(run, batch, rows)
        run.want = run.cache.pages.cpu().numpy()
        run.check_attend(batch, q, out)
        have = [a + b for a, b in zip(have, step)]
    assert have == total
    for s in range(seqs):      # the same prefixes token by token, sequence by sequence
        for p in range(0, total[s], 7):
            n = min(7, total[s] - p)
            layer(other, other.batch([p], [n], table[s:s + 1], max_length=384), x[s][p:p + n])
    assert torch.equal(run.cache.pages, other.cache.pages)

    # single tokens: eager on one cache, a graph on the other
    tokens = [torch.cat([x[s][total[s] + i:total[s] + i + 1] for s in range(seqs)]) for i in range(8)]
    eager = []
    for i in range(8):
        eager.append(layer(run, run.batch([n + i for n in total], [1] * seqs, table, max_length=384), tokens[i])[1])
    run.want = run.cache.pages.cpu().numpy()
    rows = torch.empty_like(tokens[0])
    batch = other.batch(total, [1] * seqs, table, max_length=384)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        rows.copy_(tokens[0])
        layer(other, batch, rows)      # a first run outside the capture; it writes what the first replay writes
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        _, out = layer(other, batch, rows)
    for i in range(8):
        rows.copy_(tokens[i])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager[i]), i
        batch.lengths += 1
    torch.cuda.synchronize()
    assert torch.equal(run.cache.pages, other.cache.pages)


def test_norms_before_the_cascading_cache():
    """Normalised, un-rotated queries and keys go into the cascading cache as its own inputs do."""
    from paper_2406_17808_amd.cache import CascadeKVCache
    cfg = B.make_config(batch=1, n_q_heads=8, n_kv_heads=2, head_dim=128, dtype=B.CASCADE_BF16, n_sink=4, cascade_sizes=[32, 32], ema_beta=0.9,
                        rope_base=10000.0, max_chunk=48)
    gen = torch.Generator(device=DEV).manual_seed(2)
    x = torch.randn((48, 12, 128), generator=gen, device=DEV).bfloat16()
    q, k, v = x[:, :8], x[:, 8:10], x[:, 10:].contiguous()
    w = (1 + 0.2 * torch.randn((2, 128), generator=gen, device=DEV)).bfloat16()
    qn, kn = paged.qk_norm_rope(q, k, w[0], w[1])
    cache = CascadeKVCache(cfg, DEV)
    out = cache.prefill_chunk(qn[None], kn[None], v[None])[0]
    # a first chunk is causal attention with positions 0, 1, ...
    pos = np.arange(48)
    qr, kr, vv = M.rotate(f64(qn), pos, 10000.0), M.rotate(f64(kn), pos, 10000.0), f64(v)
    for h in range(8):
        want, weighted, spread = M.attend(qr[:, h], kr[:, h // 4], vv[:, h // 4], pos[None] <= pos[:, None], 1 / math.sqrt(128))
        # the rotated queries and keys are rounded to bf16 there: the logits of a row are off by up to 2 * 2^-8 of their size
        tol = M.attend_tolerance(torch.bfloat16, want, weighted, spread, 128, 48) + 2 * (2 * 2.0 ** -8 * spread)[:, None] * weighted
        assert (np.abs(f64(out)[:, h] - want) <= tol).all()
    cache.close()


def test_another_stream_and_another_current_device_context():
    run, batch, q, out = attend_case("bf16", 128, 4, 1, 64, [300], [1], seed=9)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = run.cache.attend(batch, q)
    side.synchronize()
    assert torch.equal(out, again)
