"""Caches for the tests of the 8-bit cache: random contents inside larger buffers whose other bytes must not change."""
import ctypes

import numpy as np
import torch

from oracle import kv8_oracle as k8
from paper_2509_17396_amd import binding as ep

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
NAMES = ("k", "v", "k_scale", "v_scale", "weight", "position")


class Cache:
    """nb x H heads of C rows of d codes, T rows a scale.  pad: extra bytes per row, rows per head and entries per array around it."""

    def __init__(self, nb, H, C, d, T, seed=0, device="cuda", pad=0, plain_scales=False, with_books=True):
        rng = np.random.default_rng(seed)
        self.nb, self.H, self.C, self.d, self.T = nb, H, C, d, T
        self.blocks = -(-C // T)
        self.whole, self.view = {}, {}
        for name in NAMES:
            if name in ("k", "v"):
                shape = (nb, H, C + pad, d + 16 * pad)
                host = torch.from_numpy(rng.integers(0, 127, shape, dtype=np.uint8) + 128 * rng.integers(0, 2, shape, dtype=np.uint8))
                host[:, :, C:] = 0x7F
            elif name.endswith("scale"):
                shape = (nb, H, self.blocks + pad)
                s = 2.0 ** rng.integers(-11, -6, shape) * (1.0 if not plain_scales else rng.uniform(0.6, 1.9, shape))
                host = torch.from_numpy(s.astype(np.float32))
            elif name == "weight":
                host = torch.from_numpy(rng.exponential(size=(nb, H, C + pad)).astype(np.float32))
            else:
                host = torch.from_numpy(np.stack([rng.permutation(4 * (C + pad))[:C + pad] for _ in range(nb * H)]).reshape(
                    nb, H, C + pad).astype(np.int32))
            self.whole[name] = host.to(device)
            last = {"k": C, "v": C, "k_scale": self.blocks, "v_scale": self.blocks}.get(name, C)
            self.view[name] = self.whole[name][:, :, :last, :d] if name in ("k", "v") else self.whole[name][:, :, :last]
        books = (self.view["weight"], self.view["position"]) if with_books else (None, None)
        self.kv8 = ep.make_kv8(self.view["k"], self.view["v"], self.view["k_scale"], self.view["v_scale"], T, *books)

    def host(self):
        """[item][head] -> the oracle's six arrays (copies; scales in 64 bits)."""
        a = {n: self.view[n].cpu().numpy().copy() for n in NAMES}
        return [[[a[n][b, h].copy() if not n.endswith("scale") else a[n][b, h].astype(np.float64) for n in NAMES]
                 for h in range(self.H)] for b in range(self.nb)]

    def snapshot(self):
        return {n: t.clone() for n, t in self.whole.items()}

    def assert_is(self, want, before, what):
        """The six arrays equal `want` ([item][head], oracle's), bit for bit, and everything around them is as `before`."""
        for i, n in enumerate(NAMES):
            expect = before[n].clone()
            view = expect[:, :, :self.view[n].shape[2], :self.d] if n in ("k", "v") else expect[:, :, :self.view[n].shape[2]]
            host = np.stack([np.stack([want[b][h][i] for h in range(self.H)]) for b in range(self.nb)])
            view.copy_(torch.from_numpy(host.astype(view.cpu().numpy().dtype)))
            got = self.whole[n]
            same = (got == expect) if not got.is_floating_point() else (got.view(torch.int32) == expect.view(torch.int32))
            assert bool(same.all()), f"{what}: {n} differs at {(~same).nonzero()[:4].tolist()}: " \
                f"{got[~same][:4].tolist()} for {expect[~same][:4].tolist()}"


def params(nb, Hq, Hkv, d, p, n_cached, n_block, budget=1, dtype="bf16", causal=0, scale=0.0, q_strides=None, kv_strides=None):
    q = q_strides or (Hq * p * d, p * d, d)
    rows = max(n_block, 1)
    kv = kv_strides or (Hkv * rows * d, rows * d, d)
    return ep.Params(ctypes.sizeof(ep.Params), nb, Hq, Hkv, d, n_cached, n_block, budget, p,
                     ep.DTYPE_F32 if dtype == "f32" else ep.DTYPE_BF16, 0, scale, causal, 0, *q, *kv)


def guarded_workspace(nbytes, device="cuda"):
    """(workspace of nbytes, check()): the bytes behind it must stay as they were."""
    whole = torch.full((nbytes + 4096,), 0xA5, dtype=torch.uint8, device=device)
    return whole[:nbytes], lambda: bool((whole[nbytes:] == 0xA5).all())


def lengths(rng, nb, H, n_cached, device="cuda"):
    """Uneven old rows, one head full, one empty, one beyond the bound and one below zero (they are clamped): (device, host)."""
    n = rng.integers(0, n_cached + 1, (nb, H)).astype(np.int32)
    flat = n.reshape(-1)
    raw = flat.copy()
    raw[0] = n_cached + 5
    if flat.size > 1:
        raw[-1] = -3
    return torch.from_numpy(raw.reshape(nb, H).copy()).to(device), np.clip(raw, 0, n_cached).reshape(nb, H)
