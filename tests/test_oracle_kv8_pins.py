"""Pins of the 8-bit cache's oracle: hand-worked values, torch's e4m3 conversion, brute force, invariants, planted mistakes."""
import math

import numpy as np
import pytest
import torch

from oracle import kv8_oracle as k8


def test_code_values_are_torchs():
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(np.isnan(t), np.isnan(k8.VALUES)) and np.isnan(k8.VALUES[[0x7F, 0xFF]]).all()
    fine = ~np.isnan(t)
    assert np.array_equal(t[fine], k8.VALUES[fine]) and k8.VALUES[126] == k8.LARGEST


def test_encode_is_round_to_nearest_even():
    grid = k8.VALUES[:127]
    mid = (grid[1:] + grid[:-1]) / 2
    assert np.array_equal(k8.encode(grid), np.arange(127))
    assert np.array_equal(k8.encode(mid), [c + c % 2 for c in range(126)])          # ties to the even code
    assert np.array_equal(k8.encode(mid * (1 + 1e-9)), np.arange(1, 127))
    assert np.array_equal(k8.encode(mid * (1 - 1e-9)), np.arange(126))
    x = np.concatenate([np.linspace(-448, 448, 20011), [-0.0, math.inf, -math.inf, math.nan]]).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    fine = np.isfinite(x)
    assert np.array_equal(k8.encode(x)[fine], want[fine]) and (k8.encode(x)[~fine] == 0x7F).all()


@pytest.mark.parametrize("amax,scale", [(0.0, 2.0 ** -126), (448.0, 1.0), (448.00003, 2.0), (1.0, 2.0 ** -8), (1.75, 2.0 ** -8),
                                        (1.7500001, 2.0 ** -7), (3e38, 2.0 ** 120), (1e-45, 2.0 ** -126), (896.0, 2.0)])
def test_scales(amax, scale):
    assert k8.scale_for(amax) == scale


def one_head(rng, C, d, T):
    return [rng.integers(0, 127, (C, d), dtype=np.uint8) for _ in range(2)] + \
        [2.0 ** rng.integers(-6, 3, -(-C // T)) for _ in range(2)] + \
        [rng.exponential(size=C).astype(np.float32), np.arange(C, dtype=np.int32)]


def test_append_by_hand():
    """block of 2 would not be allowed by the library, but shows the rule: 448 fits scale 1; 1000 needs 4, and 448 at scale 4 is 112."""
    cache = [np.zeros((4, 1), np.uint8), np.zeros((4, 1), np.uint8), np.ones(2), np.ones(2), np.ones(4, np.float32), np.zeros(4, np.int32)]
    k8.append(cache, 2, 0, np.array([[448.0]]), np.array([[0.0]]), 7)
    assert cache[2][0] == 1.0 and k8.VALUES[cache[0][0, 0]] == 448.0 and cache[3][0] == 2.0 ** -126
    k8.append(cache, 2, 1, np.array([[1000.0], [1.0]]), np.array([[-0.0], [math.inf]]), 9)
    assert list(cache[2]) == [4.0, 2.0 ** -8]
    assert [k8.VALUES[c] for c in cache[0][:3, 0]] == [112.0, 256.0, 256.0]   # 1000 / 4 = 250 rounds to 256
    assert cache[1][1, 0] == 0x80 and cache[1][2, 0] == 0x7F
    assert list(cache[5]) == [7, 9, 10, 0] and list(cache[4]) == [0, 0, 0, 1]


def test_appending_row_by_row_or_at_once_ends_at_the_same_scales():
    rng = np.random.default_rng(0)
    rows = rng.standard_normal((50, 16)) * np.exp(2 * rng.standard_normal((50, 1)))
    a, b = one_head(rng, 64, 16, 16), None
    b = [x.copy() for x in a]
    k8.append(a, 16, 0, rows, rows, None)
    for i in range(50):
        k8.append(b, 16, i, rows[i:i + 1], rows[i:i + 1], None)
    assert np.array_equal(a[2][:4], b[2][:4])
    err = np.abs(k8.decode(b[0], b[2], 16)[:50] - rows)
    # rounded once or, where the scale grew, twice: half a step is 2^-4 of a value, or half of the smallest step 2^-9
    step = np.repeat(b[2], 16)[:50, None] * 2.0 ** -10
    assert (err <= 2 * np.maximum(np.abs(rows) * 2.0 ** -4 * 1.07, step)).all()


def test_attention_is_torchs_softmax():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((5, 8)), rng.standard_normal((9, 8)), rng.standard_normal((9, 8))
    last = np.array([8, 3, 0, -1, 100])
    out, lse, w = k8.attention(q, k, v, 0.5, last)
    for r in range(5):
        n = min(last[r] + 1, 9)
        if n == 0:
            assert (out[r] == 0).all() and lse[r] == -math.inf and (w[r] == 0).all()
            continue
        z = torch.from_numpy(0.5 * k[:n] @ q[r])
        assert np.allclose(w[r, :n], torch.softmax(z, 0).numpy()) and (w[r, n:] == 0).all()
        assert np.allclose(lse[r], torch.logsumexp(z, 0).item()) and np.allclose(out[r], torch.softmax(z, 0).numpy() @ v[:n])


def test_choice_by_hand():
    w = np.array([5, 1, 3, 3, 2, 3, 0.5], dtype=np.float32)
    pos = np.arange(7, dtype=np.int32)
    assert [list(x) if i else x for i, x in enumerate(k8.choose(w, pos, 7, 3, 0))] == [3, [0, 3, 2]]   # 5, then the first two 3s
    assert list(k8.choose(w, pos, 7, 3, 1)[1]) == [0, 6, 2]                 # the latest is kept whatever it weighs
    assert list(k8.choose(w, pos[::-1].copy(), 7, 3, 1)[1]) == [0, 3, 2]     # here row 0 is the latest
    assert list(k8.choose(w, pos, 7, 9, 2)[1]) == list(range(7)) and k8.choose(w, pos, 0, 3, 0)[0] == 0
    odd = np.array([math.nan, math.inf, -0.0, 0.0, -math.inf, math.nan], dtype=np.float32)
    assert list(k8.choose(odd, pos, 6, 2, 0)[1]) == [0, 5] and list(k8.choose(odd, pos, 6, 4, 0)[1]) == [0, 1, 5, 3]


def brute_choose(w, pos, n, budget, recent):
    """Rows that stay: those that fewer than K others beat."""
    key = [(int(pos[i]) > max(pos[:n]) - recent, 0 if int(pos[i]) > max(pos[:n]) - recent else k8.order(w[i]), -i) for i in range(n)]
    keep = min(budget, n)
    kept = [i for i in range(n) if sum(key[j] > key[i] for j in range(n)) < keep]
    out = list(range(keep))
    holes, tail = [i for i in out if i not in kept], [i for i in kept if i >= keep]
    for a, b in zip(holes, tail):
        out[a] = b
    assert len(holes) == len(tail)
    return out


def test_choice_against_counting():
    rng = np.random.default_rng(2)
    for _ in range(200):
        n = int(rng.integers(1, 30))
        w = rng.integers(0, 6, n).astype(np.float32)
        pos = rng.permutation(100)[:n].astype(np.int32)
        budget = int(rng.integers(1, 35))
        recent = int(rng.integers(0, budget + 1))
        assert list(k8.choose(w, pos, n, budget, recent)[1]) == brute_choose(w, pos, n, budget, recent)


def test_evict_moves_what_it_says():
    rng = np.random.default_rng(3)
    cache = one_head(rng, 64, 16, 16)
    was = [x.copy() for x in cache]
    keep, row_from = k8.evict(cache, 16, 60, 37, 5)
    assert keep == 37 and len(set(row_from)) == 37
    for c in (0, 1):
        before = k8.decode(was[c], was[2 + c], 16)
        after = k8.decode(cache[c], cache[2 + c], 16)[:37]
        err = np.abs(after - before[row_from])
        step = np.repeat(cache[2 + c], 16)[:37, None] * 2.0 ** -10  # half of the smallest step
        assert (err <= step).all()
        assert np.array_equal(cache[c][37:], was[c][37:])
        assert (cache[2 + c][:3] >= 2.0 ** -126).all()
    assert np.array_equal(cache[4][:37], was[4][row_from]) and np.array_equal(cache[5][:37], was[5][row_from])
    total = sorted(was[4][:60])
    dropped = [was[4][i] for i in range(60) if i not in set(row_from)]
    assert max(dropped) <= min(was[4][i] for i in row_from if i < 55) and len(total) == 60


@pytest.mark.parametrize("mistake", ["scale_halved", "ties_up", "not_recent"])
def test_planted_mistakes_are_seen(mistake, monkeypatch):
    if mistake == "scale_halved":
        monkeypatch.setattr(k8, "scale_for", lambda a: 2.0 ** math.floor(math.log2(max(a, 1e-30) / 448)))
        with pytest.raises(AssertionError):
            test_append_by_hand()
    elif mistake == "ties_up":
        good = k8.choose
        monkeypatch.setattr(k8, "choose", lambda w, p, n, b, r: (min(b, n), (n - 1 - good(w[:n][::-1], p[:n][::-1], n, b, r)[1]).astype(np.int32)))
        with pytest.raises(AssertionError):
            test_choice_by_hand()
    else:
        good = k8.choose
        monkeypatch.setattr(k8, "choose", lambda w, p, n, b, r: good(w, p, n, b, 0))
        with pytest.raises(AssertionError):
            test_choice_by_hand()
