"""Rows appended to the 8-bit cache, bit for bit against the oracle: codes, scales, weights, positions, and nothing else."""
import numpy as np
import pytest
import torch

from oracle import kv8_oracle as k8
from paper_2509_17396_amd import binding as ep
from tests import kv8_util as ku

pytestmark = pytest.mark.gpu


def new_rows(rng, nb, H, n, d, dtype, kind):
    x = rng.standard_normal((nb, H, n, d)) * np.exp(1.5 * rng.standard_normal((nb, H, n, 1)))
    if kind == "spread":  # many powers of two, down to what rounds to zero, and the exact borders of a scale
        x = rng.choice([-1, 1], x.shape) * 2.0 ** rng.integers(-40, 20, x.shape) * rng.choice([1.0, 1.75, 1.8125, 1.0625], x.shape)
        x[:, :, :: 3] *= 2.0 ** -30
        x[..., 0] = 0
    if kind == "odd":
        x.reshape(-1)[rng.integers(0, x.size, x.size // 7)] = rng.choice([np.inf, -np.inf, np.nan, -0.0, 3e38, 1e-45])
        x[:, :, n // 2] = np.inf
    if kind == "zero":
        x = x * 0
    return torch.from_numpy(x.astype(np.float32)).to(ku.DTYPES[dtype])


CASES = [  # dtype, d, T, items, heads, n_cached, n_block, uneven, kind, pad
    ("bf16", 128, 32, 2, 3, 64, 1, False, "normal", 0), ("bf16", 128, 32, 1, 2, 0, 97, False, "normal", 1),
    ("bf16", 64, 16, 3, 2, 50, 33, True, "normal", 3), ("f32", 96, 16, 2, 5, 90, 70, True, "spread", 2),
    ("f32", 16, 16, 1, 1, 0, 1, False, "normal", 0), ("bf16", 256, 128, 2, 2, 200, 150, True, "normal", 1),
    ("f32", 256, 64, 1, 3, 31, 129, True, "odd", 0), ("bf16", 48, 64, 2, 2, 63, 65, False, "odd", 2),
    ("bf16", 80, 128, 2, 2, 127, 1, True, "spread", 1), ("f32", 112, 32, 2, 2, 40, 40, True, "zero", 0),
    ("bf16", 192, 16, 1, 4, 15, 2, False, "spread", 0), ("f32", 160, 32, 1, 2, 32, 500, False, "normal", 0),
    ("bf16", 240, 128, 1, 2, 130, 127, True, "normal", 0)]


@pytest.mark.parametrize("case", CASES, ids=["-".join(map(str, c)) for c in CASES])
def test_append_matches_the_oracle(case):
    dtype, d, T, nb, H, n_cached, n_block, uneven, kind, pad = case
    rng = np.random.default_rng(7)
    cache = ku.Cache(nb, H, n_cached + n_block + 5, d, T, seed=1, pad=pad, plain_scales=kind == "odd")
    wide = torch.zeros((nb, H, n_block + 1, d + 8), dtype=ku.DTYPES[dtype])
    kn, vn = new_rows(rng, nb, H, n_block, d, dtype, kind), new_rows(rng, nb, H, n_block, d, dtype, "normal")
    kd, vd = wide.clone().cuda(), wide.clone().cuda()
    kd[:, :, :n_block, :d], vd[:, :, :n_block, :d] = kn.cuda(), vn.cuda()
    n_dev, n_host = ku.lengths(rng, nb, H, n_cached) if uneven else (None, np.full((nb, H), n_cached))
    first = torch.from_numpy(rng.integers(-5, 1000, nb).astype(np.int32)).cuda() if uneven else None
    prm = ku.params(nb, 2 * H, H, d, 1, n_cached, n_block, dtype=dtype, kv_strides=wide.stride()[:3])
    want, before = cache.host(), cache.snapshot()
    for b in range(nb):
        for h in range(H):
            k8.append(want[b][h], T, int(n_host[b, h]), kn[b, h].double().numpy(), vn[b, h].double().numpy(),
                      None if first is None else int(first[b]))
    for turn in range(2):  # the same rows again: the same cache
        ep.epicache_kv8_append(prm, cache.kv8, kd, vd, n_dev, first)
        torch.cuda.synchronize()
        cache.assert_is(want, before, f"turn {turn}")


def test_broadcast_rows_and_no_books():
    """Heads may share their new rows (strides of 0), and weights and positions may be missing."""
    rng = np.random.default_rng(3)
    cache = ku.Cache(2, 3, 64, 64, 16, with_books=False)
    rows = new_rows(rng, 1, 1, 20, 64, "bf16", "normal")
    prm = ku.params(2, 3, 3, 64, 1, 30, 20, kv_strides=(0, 0, 64))
    want, before = cache.host(), cache.snapshot()
    for b in range(2):
        for h in range(3):
            books = want[b][h][4:]
            k8.append(want[b][h][:4] + [x.copy() for x in books], 16, 30, rows[0, 0].double().numpy(), rows[0, 0].double().numpy(), 0)
    ep.epicache_kv8_append(prm, cache.kv8, rows.cuda(), rows.cuda())
    torch.cuda.synchronize()
    cache.assert_is(want, before, "broadcast")


def test_row_by_row_scales_grow():
    rng = np.random.default_rng(5)
    cache = ku.Cache(1, 2, 48, 64, 16)
    want, before = cache.host(), cache.snapshot()
    n = torch.zeros((1, 2), dtype=torch.int32, device="cuda")
    for i in range(40):
        x = new_rows(rng, 1, 2, 1, 64, "bf16", "normal") * float(1 + 7 * (i % 5 == 4) * i)
        x = x.to(torch.bfloat16)
        prm = ku.params(1, 2, 2, 64, 1, 40, 1)
        ep.epicache_kv8_append(prm, cache.kv8, x.cuda(), x.cuda(), n)
        n += 1
        for h in range(2):
            k8.append(want[0][h], 16, i, x[0, h].double().numpy(), x[0, h].double().numpy(), None)
    torch.cuda.synchronize()
    cache.assert_is(want, before, "forty rows")


def test_offsets_beyond_32_bits():
    """A cache of more than 4 GiB: the last head's rows lie behind 2^32 bytes."""
    C, d, T, H = 1 << 20, 256, 32, 17
    k, v, ks, vs, w, pos = ep.alloc_kv8(1, H, C, d, T)
    assert k.stride(1) * (H - 1) >= 1 << 32
    kv8 = ep.make_kv8(k, v, ks, vs, T, w, pos)
    rng = np.random.default_rng(1)
    x = new_rows(rng, 1, H, 3, d, "bf16", "normal")
    n_old = C - 3
    ep.epicache_kv8_append(ku.params(1, H, H, d, 1, n_old, 3), kv8, x.cuda(), x.cuda())
    torch.cuda.synchronize()
    for h in (0, H - 1):
        rows = x[0, h].double().numpy()
        codes, scale = np.zeros((T, d), np.uint8), np.ones(1)
        k8.put_rows(codes, scale, T, np.arange(T - 3, T), rows, np.arange(T - 3))
        assert np.array_equal(k[0, h, C - T:].view(torch.uint8).cpu().numpy(), codes) and float(ks[0, h, -1]) == scale[0]
        assert np.array_equal(v[0, h, C - T:].view(torch.uint8).cpu().numpy(), codes) and float(vs[0, h, -1]) == scale[0]
    assert int(k[0, :, :C - T].view(torch.uint8).count_nonzero()) == 0
