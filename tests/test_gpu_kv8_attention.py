"""Attention over the 8-bit cache against the oracle in 64 bits.

Bounds, per query row, with u = 2^-24 and A_c = sum_i w_i |v_ic| (exact weights):
  a logit is a sum of d products in fp32, of bf16 parts whose products are exact: |error| <= D = (2 d + 32) u max_i sum_j |q_j k_ij| scale,
    which also covers the rounding of its scaling and of the exponent's argument; the exponential adds 2^-21
  an unnormalised weight is then off by a factor of at most 1 + D + 2^-21, and the sum of n of them by another n u
  the weights enter the product with V rounded to bf16 once at most (2^-8 each) for bf16, and to 2^-22 or better for fp32
  the output is rounded to its type: half a step, 2^-8 for bf16 and 2^-24 for fp32
  lse: D + 2^-21 + n u, and two roundings of its own magnitude."""
import math

import numpy as np
import pytest
import torch

from oracle import kv8_oracle as k8
from paper_2509_17396_amd import binding as ep
from tests import kv8_util as ku

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def check(dtype, q, k, v, scale, last, out, lse, got_weights=None, base=None):
    """One head: q [R, d], k, v [n, d] decoded, out, lse as the GPU gave them; got_weights: the accumulated ones, on `base`."""
    o, l, w = k8.attention(q, k, v, scale, last)
    n, d = k.shape
    seen = np.arange(n)[None, :] <= np.asarray(last)[:, None]
    reach = np.where(seen, np.abs(q) @ np.abs(k).T, 0.0).max(axis=1, initial=0.0) * scale
    delta = (2 * d + 32) * U * reach + 2.0 ** -21 + n * U
    A = w @ np.abs(v)
    part, step = (2.0 ** -8, 2.0 ** -8) if dtype == "bf16" else (2.0 ** -22, U)
    bound = (part + 2 * delta[:, None]) * A * (1 + 2.0 ** -7) + step * np.abs(o) + 1e-37
    assert np.array_equal(np.isnan(o), np.isnan(out)), np.argwhere(np.isnan(o) != np.isnan(out))[:4]
    off = np.abs(np.nan_to_num(out) - np.nan_to_num(o)) / np.nan_to_num(bound, nan=1.0)
    assert off.max(initial=0.0) <= 1.0, (off.max(), np.unravel_index(off.argmax(), off.shape))
    empty = l == -math.inf
    assert np.array_equal(empty, lse == -math.inf) and (out[empty] == 0).all()
    fine = np.isfinite(l)
    assert np.array_equal(np.isnan(l), np.isnan(lse))
    assert (np.abs(lse - l)[fine] <= (delta + 2 * U * np.abs(l))[fine] * 1.01 + 1e-37).all()
    if got_weights is not None:
        add = w.sum(axis=0)
        bound_w = (2 * delta[:, None] * w).sum(axis=0) * 1.01 + len(q) * U * add + 2 * U * (np.abs(base[:n]) + add) + 1e-37
        diff = np.abs(got_weights[:n] - (base[:n] + add))
        assert np.array_equal(np.isnan(add), np.isnan(got_weights[:n]))
        assert (np.nan_to_num(diff) <= np.nan_to_num(bound_w)).all(), np.nanmax(diff / bound_w)
        assert np.array_equal(got_weights[n:], base[n:])


def run(cache, dtype, G, p, n_cached, n_block, causal, accumulate, seed=0, uneven=False, scale=0.0, spread=1.0, pad_q=0, edit=None,
        repeat=1):
    rng = np.random.default_rng(seed)
    nb, H, d, T = cache.nb, cache.H, cache.d, cache.T
    q = torch.from_numpy((spread * rng.standard_normal((nb, G * H, p, d))).astype(np.float32)).to(ku.DTYPES[dtype])
    if edit:
        edit(q, cache)
    whole = torch.zeros((nb, G * H, p + (pad_q > 0), d + 8 * pad_q), dtype=q.dtype)
    whole[:, :, :p, :d] = q
    qd = whole.cuda()
    n_dev, n_host = ku.lengths(rng, nb, H, n_cached) if uneven else (None, np.full((nb, H), n_cached))
    # behind a head's last row: the NaN code, an infinite scale where a whole block is behind it
    for b in range(nb):
        for h in range(H):
            n = int(n_host[b, h]) + n_block
            cache.view["k"][b, h, n:], cache.view["v"][b, h, n:] = 0x7F, 0xFF
            for name in ("k_scale", "v_scale"):
                cache.view[name][b, h, -(-n // T):] = math.inf
    prm = ku.params(nb, G * H, H, d, p, n_cached, n_block, dtype=dtype, causal=causal, scale=scale, q_strides=whole.stride()[:3])
    host, before = cache.host(), cache.snapshot()
    out = torch.full((nb, G * H, p, d), 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full((nb, G * H, p), 7.0, dtype=torch.float32, device="cuda")
    ws, untouched = ku.guarded_workspace(ep.epicache_kv8_workspace_size(prm, cache.kv8))
    for _ in range(repeat):
        ep.epicache_kv8_attention(prm, cache.kv8, qd, n_dev, out, lse, ws, accumulate=accumulate)
    torch.cuda.synchronize()
    assert untouched()
    for name in ("k", "v", "k_scale", "v_scale", "position") + (() if accumulate else ("weight",)):
        assert torch.equal(cache.whole[name].view(torch.uint8), before[name].view(torch.uint8)), name
    got_w = cache.view["weight"].cpu().numpy().astype(np.float64)
    o, l = out.double().cpu().numpy(), lse.double().cpu().numpy()
    scale = scale or 1.0 / math.sqrt(d)
    for b in range(nb):
        for h in range(H):
            n = int(n_host[b, h]) + n_block
            kc, vc, ks, vs, w0, _ = host[b][h]
            k, v = (k8.decode(c[:n], s, T) for c, s in ((kc, ks), (vc, vs)))
            last = np.tile(int(n_host[b, h]) + np.arange(p) if causal else np.full(p, n - 1), G)
            heads = slice(h * G, (h + 1) * G)
            check(dtype, q[b, heads].double().numpy().reshape(G * p, d), k, v, scale, last, o[b, heads].reshape(G * p, d),
                  l[b, heads].reshape(-1), got_w[b, h] if accumulate and repeat == 1 else None, w0.astype(np.float64))
    return out, lse, cache.view["weight"].clone()


TOKENS = [  # dtype, d, T, items, heads, G, n_cached, n_block, uneven, pad
    ("bf16", 128, 32, 2, 3, 4, 64, 1, False, 0), ("bf16", 128, 32, 1, 2, 3, 1025, 1, True, 1), ("bf16", 64, 16, 2, 2, 7, 333, 1, True, 2),
    ("f32", 96, 16, 2, 3, 1, 200, 1, True, 1), ("f32", 128, 32, 1, 2, 4, 2000, 1, False, 0), ("bf16", 256, 128, 1, 2, 8, 700, 1, True, 0),
    ("f32", 16, 16, 1, 1, 1, 0, 1, False, 0), ("bf16", 48, 64, 2, 2, 16, 129, 1, True, 3), ("bf16", 80, 128, 1, 2, 17, 300, 1, False, 0),
    ("f32", 256, 32, 1, 2, 5, 95, 1, True, 0), ("bf16", 112, 32, 1, 2, 2, 31, 1, False, 0), ("bf16", 192, 64, 1, 1, 40, 500, 1, False, 0),
    ("f32", 160, 128, 3, 1, 3, 777, 1, True, 0), ("bf16", 128, 32, 64, 8, 1, 40, 1, True, 0), ("bf16", 128, 64, 1, 1, 4, 9000, 1, False, 0)]


@pytest.mark.parametrize("accumulate", [False, True], ids=["plain", "accumulate"])
@pytest.mark.parametrize("case", TOKENS, ids=["-".join(map(str, c)) for c in TOKENS])
def test_single_tokens(case, accumulate):
    dtype, d, T, nb, H, G, n_cached, n_block, uneven, pad = case
    cache = ku.Cache(nb, H, n_cached + n_block + 4, d, T, seed=3, pad=pad, plain_scales=d == 96)
    run(cache, dtype, G, 1, n_cached, n_block, int(uneven), accumulate, uneven=uneven, pad_q=pad)


PATCHES = [  # dtype, d, T, items, heads, G, p, n_cached, n_block, causal, uneven
    ("bf16", 128, 32, 2, 2, 4, 64, 300, 64, 1, True), ("bf16", 128, 32, 1, 2, 4, 37, 130, 0, 0, False),
    ("bf16", 64, 16, 2, 2, 3, 50, 333, 50, 1, True), ("f32", 96, 16, 1, 2, 2, 33, 200, 33, 1, True),
    ("f32", 128, 32, 1, 1, 4, 100, 64, 100, 1, False), ("bf16", 256, 64, 1, 2, 2, 65, 100, 65, 1, True),
    ("bf16", 128, 32, 1, 1, 4, 300, 0, 300, 1, False), ("bf16", 128, 128, 1, 2, 1, 200, 500, 77, 0, True),
    ("bf16", 80, 32, 1, 2, 7, 17, 95, 17, 1, True), ("f32", 64, 16, 1, 2, 1, 129, 40, 129, 1, True),
    ("bf16", 16, 16, 1, 1, 2, 2, 0, 2, 1, False), ("f32", 256, 128, 1, 1, 3, 40, 150, 40, 1, False),
    ("bf16", 192, 32, 1, 1, 8, 9, 257, 9, 1, False), ("bf16", 128, 64, 3, 1, 4, 5, 1000, 5, 1, True),
    ("bf16", 128, 32, 1, 1, 1, 513, 511, 513, 1, False)]


@pytest.mark.parametrize("accumulate", [False, True], ids=["plain", "accumulate"])
@pytest.mark.parametrize("case", PATCHES, ids=["-".join(map(str, c)) for c in PATCHES])
def test_patches_and_blocks(case, accumulate):
    dtype, d, T, nb, H, G, p, n_cached, n_block, causal, uneven = case
    cache = ku.Cache(nb, H, n_cached + n_block + 9, d, T, seed=4, plain_scales=T == 128)
    run(cache, dtype, G, p, n_cached, n_block, causal, accumulate, uneven=uneven, pad_q=p % 2)


@pytest.mark.parametrize("p", [1, 40])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sharp_and_flat_rows(dtype, p):
    for spread in (60.0, 0.0):  # one key takes all; all keys alike
        cache = ku.Cache(1, 2, 400, 64, 32, seed=5)
        run(cache, dtype, 4, p, 390, 0, 0, True, spread=spread, scale=0.25)


@pytest.mark.parametrize("p", [1, 40])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_blocks_of_very_different_scales(dtype, p):
    """Values 2^-30 times the others', that only the sharpest rows show, and a block of keys far above the rest."""
    cache = ku.Cache(1, 1, 320, 128, 32, seed=6)
    cache.view["v_scale"][:, :, 3:6] *= 2.0 ** -30
    cache.view["k_scale"][:, :, 4] *= 64.0
    cache.view["v_scale"][:, :, 8] = 2.0 ** -126
    run(cache, dtype, 4, p, 320, 0, 0, True)


def test_not_finite():
    """A NaN value shows in the rows that see it and in no other; infinite queries give NaN; logits of -inf are weights of 0."""
    for dtype in ("bf16", "f32"):
        for p in (1, 6, 70):
            def edit(q, cache):
                n = 100
                cache.view["v"][0, 0, n + p - 1, 5] = 0x7F      # the last row: the last query alone sees it
                cache.view["v"][0, 1, 17, 3] = 0xFF             # all see it
                cache.view["k"][0, 2, n + p - 1, 8] = 0x7F      # a key that is not a number, for the last query
                cache.view["k"][0, 3, :, :] = 0x38              # all keys positive:
                q[0, 6, 0, 0] = -math.inf                       # .. no weight at all
                q[0, 7, p - 1, 2] = math.inf
            run(ku.Cache(1, 4, 180, 64, 16, seed=7), dtype, 2, p, 100, p, 1, True, edit=edit)


@pytest.mark.parametrize("G", [1, 3])
@pytest.mark.parametrize("dtype,p", [("bf16", 9), ("bf16", 40), ("bf16", 150), ("bf16", 300), ("f32", 9), ("f32", 150)])
def test_not_a_number_inside_a_block(dtype, p, G):
    """Values that are not numbers among the block's own rows: the queries from there on see them, those before do not."""
    def edit(q, cache):
        for h, (row, column) in enumerate(((0, 3), (p // 2, 60), (p // 3, 17))):
            cache.view["v"][0, h, 100 + row, column] = 0x7F
            cache.view["v"][0, h, 100 + p - 1, column + 1] = 0xFF
    run(ku.Cache(1, 3, 100 + p, 64, 16, seed=9), dtype, G, p, 100, p, 1, True, edit=edit)


@pytest.mark.parametrize("dtype,p", [("bf16", 1), ("bf16", 80), ("f32", 1), ("bf16", 6)])
def test_the_same_bits_every_time(dtype, p):
    got = [run(ku.Cache(2, 2, 3000, 128, 32, seed=8), dtype, 4, p, 2900, p, 1, True, repeat=2) for _ in range(2)]
    for a, b in zip(*got):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_offsets_beyond_32_bits():
    C, d, T, H = 1 << 20, 256, 32, 17
    k, v, ks, vs, w, pos = ep.alloc_kv8(1, H, C, d, T)
    kv8 = ep.make_kv8(k, v, ks, vs, T, w, pos)
    rng = np.random.default_rng(1)
    codes = rng.integers(0, 127, (50, d), dtype=np.uint8)
    n_old = C - 1
    k[0, H - 1, C - 50:], v[0, H - 1, C - 50:] = (torch.from_numpy(codes).cuda().view(torch.float8_e4m3fn) for _ in range(2))
    q = torch.from_numpy(rng.standard_normal((1, H, 1, d)).astype(np.float32)).cuda().bfloat16() * 0.01
    out, lse = torch.empty_like(q), torch.empty((1, H, 1), device="cuda")
    prm = ku.params(1, H, H, d, 1, n_old, 1)
    ep.epicache_kv8_attention(prm, kv8, q, None, out, lse, ep.alloc_kv8_workspace(prm, kv8), accumulate=True)
    torch.cuda.synchronize()
    x = k8.VALUES[codes]
    qh = q[0, H - 1, 0].double().cpu().numpy()
    z = x @ qh / 16.0
    top = max(z.max(), 0.0)
    total = np.exp(z - top).sum() + (C - 50) * math.exp(-top)   # all other keys are zero
    want = (np.exp(z - top)[:, None] * x).sum(axis=0) / total
    A = (np.exp(z - top)[:, None] * np.abs(x)).sum(axis=0) / total
    D = (2 * d + 32) * U * (np.abs(x) @ np.abs(qh)).max() / 16 + 2.0 ** -21 + C * U
    assert (np.abs(out[0, H - 1, 0].double().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2 * D) * A).all()
    assert abs(float(lse[0, H - 1, 0]) - (top + math.log(total))) <= D + 2 * U * 20
    got = w[0, H - 1, C - 50:].double().cpu().numpy()
    assert np.allclose(got, np.exp(z - top) / total, rtol=2 * D, atol=0)
