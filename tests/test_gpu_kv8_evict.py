"""Eviction from the 8-bit cache by accumulated weight, bit for bit against the oracle: which rows, codes, scales, books."""
import numpy as np
import pytest
import torch

from oracle import kv8_oracle as k8
from paper_2509_17396_amd import binding as ep
from tests import kv8_util as ku

pytestmark = pytest.mark.gpu


def weights(rng, shape, kind):
    w = rng.exponential(size=shape)
    if kind == "ties":
        w = rng.integers(0, 4, shape) * 0.5
    if kind == "equal":
        w = np.ones(shape)
    if kind == "odd":
        w = rng.choice([np.nan, -np.nan, np.inf, -np.inf, 0.0, -0.0, 1.0, -1.0, 1e-45], shape)
    if kind == "zeros":
        w = np.where(rng.random(shape) < 0.9, 0.0, w)
    if kind == "rising":
        w = np.sort(w, axis=-1)
    if kind == "cluster":
        w = 1.0 + 1e-6 * w + 1e4 * (rng.random(shape) < 0.01)
    return torch.from_numpy(w.astype(np.float32))


CASES = [  # d, T, items, heads, n_cached, n_block, budget, recent, uneven, kind, pad
    (128, 32, 2, 3, 64, 1, 64, 8, False, "plain", 0), (64, 16, 1, 2, 1, 0, 1, 0, False, "plain", 0),
    (64, 16, 3, 2, 50, 33, 41, 5, True, "ties", 3), (96, 16, 2, 5, 90, 70, 77, 77, True, "odd", 2),
    (16, 16, 1, 1, 0, 40, 1, 1, False, "plain", 0), (256, 128, 2, 2, 200, 150, 333, 3, True, "plain", 1),
    (256, 64, 1, 3, 300, 129, 200, 0, True, "equal", 0), (48, 64, 2, 2, 63, 65, 128, 9, False, "plain", 2),
    (80, 128, 2, 2, 600, 1, 500, 60, True, "rising", 1), (112, 32, 2, 2, 1000, 500, 777, 50, True, "zeros", 0),
    (128, 32, 1, 2, 2048, 2048, 2048, 64, False, "plain", 0), (64, 32, 1, 2, 5000, 3700, 4100, 100, False, "cluster", 0),
    (128, 32, 300, 1, 100, 1, 100, 10, True, "plain", 0), (64, 16, 1, 2, 200, 50, 1000, 7, True, "plain", 0),
    (64, 64, 1, 1, 20000, 13000, 17000, 700, False, "ties", 0), (64, 64, 1, 2, 40000, 1, 40000, 100, False, "plain", 0)]


@pytest.mark.parametrize("budgets", [False, True], ids=["one_budget", "budgets"])
@pytest.mark.parametrize("case", CASES, ids=["-".join(map(str, c)) for c in CASES])
def test_evict_matches_the_oracle(case, budgets):
    d, T, nb, H, n_cached, n_block, budget, recent, uneven, kind, pad = case
    rng = np.random.default_rng(11)
    cache = ku.Cache(nb, H, n_cached + n_block + 3, d, T, seed=2, pad=pad, plain_scales=kind == "odd")
    cache.view["weight"].copy_(weights(rng, cache.view["weight"].shape, kind))
    if kind == "odd":  # NaN codes move as they are
        cache.view["k"][:, :, ::5, ::7] = 0x7F
    n_dev, n_host = ku.lengths(rng, nb, H, n_cached) if uneven else (None, np.full((nb, H), n_cached))
    m_host = rng.integers(0, budget + 1, nb) if budgets else np.full(nb, budget)
    m_raw = m_host.copy()
    if budgets:
        m_raw[0], m_host[0] = budget + 9, budget
        if nb > 1:
            m_raw[1], m_host[1] = -4, 0
    m_dev = torch.from_numpy(m_raw.astype(np.int32)).cuda() if budgets else None
    prm = ku.params(nb, 2 * H, H, d, 1, n_cached, n_block, budget=budget)
    most = min(budget, n_cached + n_block)
    want, before = cache.host(), cache.snapshot()
    w_rows, w_kept = np.full((nb, H, most), -1, np.int32), np.zeros((nb, H), np.int32)
    for b in range(nb):
        for h in range(H):
            keep, row_from = k8.evict(want[b][h], T, int(n_host[b, h]) + n_block, int(m_host[b]), recent)
            w_kept[b, h] = keep
            w_rows[b, h, :keep] = row_from
    ws, untouched = ku.guarded_workspace(ep.epicache_kv8_workspace_size(prm, cache.kv8))
    rows = torch.full((nb, H, most), 77, dtype=torch.int32, device="cuda")
    kept = n_dev if n_dev is not None else torch.full((nb, H), -7, dtype=torch.int32, device="cuda")  # in place of the lengths
    ep.epicache_kv8_evict(prm, cache.kv8, recent, n_dev, m_dev, kept, ws, row_from=None if nb == 3 else rows)
    torch.cuda.synchronize()
    assert np.array_equal(kept.cpu().numpy(), w_kept)
    if nb != 3:
        assert np.array_equal(rows.cpu().numpy(), w_rows)
    cache.assert_is(want, before, "evict")
    assert untouched()


def test_without_positions_a_rows_index_stands_for_it():
    rng = np.random.default_rng(4)
    cache = ku.Cache(1, 2, 100, 64, 16)
    kv8 = ep.make_kv8(cache.view["k"], cache.view["v"], cache.view["k_scale"], cache.view["v_scale"], 16, cache.view["weight"])
    want, before = cache.host(), cache.snapshot()
    for h in range(2):
        stand_in = want[0][h][:5] + [np.arange(100, dtype=np.int32)]
        k8.evict(stand_in, 16, 100, 60, 20)
    kept = torch.zeros((1, 2), dtype=torch.int32, device="cuda")
    prm = ku.params(1, 2, 2, 64, 1, 80, 20, budget=60)
    ep.epicache_kv8_evict(prm, kv8, 20, None, None, kept, ep.alloc_kv8_workspace(prm, kv8))
    torch.cuda.synchronize()
    assert kept.tolist() == [[60, 60]]
    cache.assert_is(want, before, "no positions")
