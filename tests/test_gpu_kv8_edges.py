"""The 8-bit cache's calls where they are easily forgotten: heads without a single row, no new rows at all, many heads, steps of many rows
replayed from a graph, and the splits of keys and of rows that small tests do not reach."""
import numpy as np
import pytest
import torch

from oracle import kv8_oracle as k8
from paper_2509_17396_amd import binding as ep
from tests import kv8_util as ku
from tests.test_gpu_kv8_attention import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d,p", [("bf16", 128, 1), ("bf16", 128, 40), ("f32", 80, 1), ("f32", 80, 40), ("bf16", 256, 9), ("bf16", 64, 150)])
def test_attention_over_heads_without_a_row(dtype, d, p):
    cache = ku.Cache(3, 2, 300, d, 32, seed=11)
    out, lse, _ = run(cache, dtype, 4, p, 290, 0, 0, True, uneven=True)
    assert bool((out[-1, -4:] == 0).all()) and bool((lse[-1, -4:] == -float("inf")).all())


def test_evict_and_append_without_new_rows():
    cache = ku.Cache(2, 3, 130, 64, 16, seed=12)
    rng = np.random.default_rng(2)
    n_dev, n_host = ku.lengths(rng, 2, 3, 120)
    prm = ku.params(2, 3, 3, 64, 1, 120, 0, budget=70)
    want, before = cache.host(), cache.snapshot()
    ep.epicache_kv8_append(prm, cache.kv8, None, None, n_dev)
    kept = np.array([[k8.evict(want[b][h], 16, int(n_host[b, h]), 70, 10)[0] for h in range(3)] for b in range(2)])
    ep.epicache_kv8_evict(prm, cache.kv8, 10, n_dev, None, n_dev, ep.alloc_kv8_workspace(prm, cache.kv8))
    torch.cuda.synchronize()
    assert np.array_equal(n_dev.cpu().numpy(), kept) and kept.min() == 0
    cache.assert_is(want, before, "no new rows")


@pytest.mark.parametrize("dtype,d,G,p,n_cached,n_block,causal", [
    ("bf16", 128, 4, 1, 30000, 1, 1),        # one head: its keys in as many splits as there are
    ("bf16", 96, 1, 700, 100, 700, 1),       # the rows of few keys in several splits
    ("f32", 128, 2, 300, 60, 300, 1), ("bf16", 256, 1, 400, 200, 0, 0), ("bf16", 128, 1, 200, 5000, 200, 1)])
def test_one_head_alone(dtype, d, G, p, n_cached, n_block, causal):
    run(ku.Cache(1, 1, n_cached + n_block, d, 32, seed=13), dtype, G, p, n_cached, n_block, causal, True)


def test_many_heads():
    """As many as fill the grid's second axis more than once over the chip, in every call."""
    nb, H, d, T, n_old = 1500, 8, 16, 16, 20
    cache = ku.Cache(nb, H, n_old + 1, d, T, seed=14)
    rng = np.random.default_rng(3)
    x = torch.from_numpy(rng.standard_normal((nb, H, 1, d)).astype(np.float32)).cuda()
    q = torch.from_numpy(rng.standard_normal((nb, H, 1, d)).astype(np.float32)).cuda()
    prm = ku.params(nb, H, H, d, 1, n_old, 1, budget=n_old, dtype="f32", causal=1)
    ws = ep.alloc_kv8_workspace(prm, cache.kv8)
    want = cache.host()
    out, lse = torch.empty_like(q), torch.empty((nb, H, 1), device="cuda")
    kept = torch.zeros((nb, H), dtype=torch.int32, device="cuda")
    ep.epicache_kv8_append(prm, cache.kv8, x, x)
    ep.epicache_kv8_attention(prm, cache.kv8, q, None, out, lse, ws, accumulate=False)
    ep.epicache_kv8_evict(prm, cache.kv8, 1, None, None, kept, ws)
    torch.cuda.synchronize()
    assert bool((kept == n_old).all()) and bool(out.isfinite().all())
    got = cache.host()
    for b, h in ((0, 0), (700, 5), (nb - 1, H - 1), (1023, 7), (1311, 0)):
        row = x[b, h].double().cpu().numpy()
        k8.append(want[b][h], T, n_old, row, row, None)
        k = k8.decode(want[b][h][0], want[b][h][2], T)
        v = k8.decode(want[b][h][1], want[b][h][3], T)
        o, l, _ = k8.attention(q[b, h].double().cpu().numpy(), k, v, d ** -0.5, np.array([n_old]))
        assert np.allclose(out[b, h].double().cpu().numpy(), o, rtol=1e-4, atol=1e-4 * np.abs(v).max())
        k8.evict(want[b][h], T, n_old + 1, n_old, 1)
        for i in range(6):
            live = slice(None) if i in (2, 3) else slice(n_old)
            assert np.array_equal(want[b][h][i][live], got[b][h][i][live]), (b, h, i)


@pytest.mark.parametrize("p", [40, 300])
def test_blocks_replayed_from_a_graph(p):
    """Attention of many rows with accumulated weights, captured on a stream of its own; eager calls between the replays."""
    n_cached, d, G, H = 500, 128, 2, 2
    cache = ku.Cache(1, H, n_cached + p, d, 32, seed=15)
    prm = ku.params(1, G * H, H, d, p, n_cached, p, causal=1)
    ws = ep.alloc_kv8_workspace(prm, cache.kv8)
    q = torch.zeros((1, G * H, p, d), dtype=torch.bfloat16, device="cuda")
    out, lse = torch.empty_like(q), torch.empty((1, G * H, p), device="cuda")
    weight = cache.view["weight"]

    def call():
        weight.zero_()
        ep.epicache_kv8_attention(prm, cache.kv8, q, None, out, lse, ws, accumulate=True)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    g = torch.Generator(device="cuda")
    for turn in range(6):
        g.manual_seed(turn)
        q.copy_(torch.randn(q.shape, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in (out, lse, weight)]
        call()
        torch.cuda.synchronize()
        for a, b in zip(replayed, (out, lse, weight)):
            assert torch.equal(a.view(torch.uint8), b.contiguous().view(torch.uint8)), turn
        assert abs(float(weight.double().sum()) - G * H * p) < 1e-3 * G * H * p   # every query gives away 1
