"""Many rows over long 8-bit caches on the GPU: shares of more than 64 blocks, groups of 64 blocks that nothing in a workgroup sees, slots out of
the order of tokens."""
import numpy as np
import pytest
import torch

import full_dense as fd
from paper_2505_23666_amd import binding as lb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}


def tokens(rng, shape, dtype, gain=1.0):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32) * np.float32(gain)).to(TORCH[dtype]).to(DEV)


def filled(rng, B, Hq, Hkv, d, cap, n, dtype, out):
    """Blocks of several scales, keys and values apart."""
    c = lb.LolaFullCache(B, Hq, Hkv, d, cap, dtype=dtype, out_dtype=out, device=DEV)
    size = torch.from_numpy(np.ldexp(1.0, rng.integers(-3, 4, (1, Hkv, -(-n // 64), 1, 1))).astype(np.float32)).to(DEV).expand(-1, -1, -1, 64, -1).reshape(1, Hkv, -1, 1)[:, :, :n]
    k, v = tokens(rng, (B, Hkv, n, d), dtype), tokens(rng, (B, Hkv, n, d), dtype)
    c.append((k * size.clamp(max=1.5)).to(TORCH[dtype]), (v * size).to(TORCH[dtype]))
    return c


def check(c, q, gather, out):
    before = c.weight.double() if gather else None
    y = c.attend(q, gather=gather)
    want, w = fd.attend(c, q)
    # (rows that see a few small values beside blocks of larger ones: per row, outputs within a part of the row's own size)
    size = want.norm(dim=-1)
    off = torch.where(size > 0, (y.double() - want).norm(dim=-1) / size.clamp(min=1e-30), (y.double() - want).norm(dim=-1))
    print(f"off by {float(off.max()):.3g}", flush=True)
    assert float(off.max()) <= (2e-5 if out == "f32" else 2.0 ** -7)
    assert fd.distance(y, want) <= (1e-6 if out == "f32" else 2.0 ** -8 + 2.0 ** -11)
    if gather:
        for b, h in ((b, h) for b in range(c.B) for h in range(c.Hkv)):
            n = int(c.count[b, h])
            assert fd.distance(c.weight[b, h, :n], before[b, h, :n] + w[b, h, :n]) <= 1e-6


# B, Hq, Hkv, pairs, T: one share of 86 blocks; two shares of 70; a prompt of its own cache, one share of 130 blocks and two of 65
SHAPES = [(16, 4, 1, 5500, 200), (4, 16, 4, 8960, 500), (1, 8, 8, 8300, 8300), (2, 2, 2, 8300, 8300)]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("f32", "f32")])
def test_shares_of_more_than_64_blocks(shape, dtype, out):
    B, Hq, Hkv, n, T = shape
    rng = np.random.default_rng(n)
    c = filled(rng, B, Hq, Hkv, 32, n, n, dtype, out)
    check(c, tokens(rng, (B, Hq, T, 32), dtype), T < 1000, out)


@pytest.mark.parametrize("d,dtype,out", [(32, "f32", "f32"), (64, "bf16", "bf16"), (128, "bf16", "f32")])
def test_slots_out_of_the_order_of_tokens(d, dtype, out):
    """The call's own tokens lie in the middle of the cache, so that the early rows pass over whole groups of blocks between ones they see."""
    rng = np.random.default_rng(d)
    for B, Hq, Hkv, n, T in ((1, 8, 8, 12500, 8300), (2, 2, 2, 12500, 8300)):
        c = filled(rng, B, Hq, Hkv, d, n, n, dtype, out)
        i = torch.arange(n, device=DEV).int()
        c.idx[:, :, :n] = torch.cat((i[:2100], i[n - T:], i[2100:n - T]))
        check(c, tokens(rng, (B, Hq, T, d), dtype), False, out)


@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("gather", [False, True])
def test_many_rows_after_an_eviction(dtype, out, gather):
    """Late tokens in early slots: an eviction moves them there, then more tokens come."""
    rng = np.random.default_rng(9)
    c = filled(rng, 2, 4, 2, 64, 9000, 7000, dtype, out)
    c.weight.copy_(torch.rand(c.weight.shape, device=DEV))
    c.evict(5000, 4, 300)
    k, v = tokens(rng, (2, 2, 900, 64), dtype), tokens(rng, (2, 2, 900, 64), dtype, 4.0)
    c.append(k, v)
    assert int((c.idx[:, :, :5000] >= 6000).sum()) > 0
    check(c, tokens(rng, (2, 4, 1500, 64), dtype), gather, out)      # (queries of tokens that the eviction's survivors came from, too)
