"""The 8-bit full-context cache on the GPU: what is not finite, in queries and in tokens, reaches the outputs as NaN, through every kernel."""
import numpy as np
import pytest
import torch

from paper_2505_23666_amd import binding as lb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}

# heads, head_dim, capacity, pairs held before, new tokens: the generation step in one workgroup and in shares, with two column tiles, a few rows
# with a mask, the many-row kernel in one share and in several, the widest head
FORMS = [(4, 64, 128, 1, 1), (4, 128, 4096, 700, 1), (32, 64, 4096, 300, 1), (4, 64, 4096, 300, 5), (4, 64, 128, 0, 40), (4, 128, 4096, 600, 50),
         (2, 256, 512, 100, 1), (2, 256, 512, 100, 30)]


def tokens(rng, shape, dtype):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(TORCH[dtype]).to(DEV)


def bits(x, value):
    """value: the bits of a 16- or 32-bit number of x's type, as one of its elements."""
    i = torch.int16 if x.dtype == torch.bfloat16 else torch.int32
    top = 1 << (15 if i == torch.int16 else 31)
    return torch.tensor([value - 2 * top if value >= top else value], dtype=i).view(x.dtype)[0]


@pytest.mark.parametrize("form", FORMS, ids=lambda f: "-".join(map(str, f)))
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
def test_tokens_that_are_not_finite(form, dtype, out):
    """A NaN key: NaN for the queries that see it, in the output's type too, and for no other."""
    Hq, d, cap, held, T = form
    rng = np.random.default_rng(held + T)
    c = lb.LolaFullCache(2, Hq, 1, d, cap, dtype=dtype, out_dtype=out, device=DEV)
    if held:
        k = tokens(rng, (2, 1, held, d), dtype)
        c.append(k, k)
    k, q = tokens(rng, (2, 1, T, d), dtype), tokens(rng, (2, Hq, T, d), dtype)
    at = T // 2
    k[1, 0, at, d - 1] = float("nan")
    for gather in (False, True):
        if gather or T > 1:
            if not gather:
                c.append(k, k)
            y = c.attend(q, gather=gather)
        else:
            y = c.step(*(x[:, :, 0].contiguous() for x in (q, k, k)))[:, :, None]
        y = y.float().cpu()
        assert torch.isfinite(y[0]).all() and torch.isfinite(y[1, :, :at]).all(), gather
        assert torch.isnan(y[1, :, at:]).all(), (gather, y[1, :, at:].flatten()[:4])


@pytest.mark.parametrize("form", FORMS, ids=lambda f: "-".join(map(str, f)))
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
def test_queries_that_are_not_finite(form, dtype, out):
    """A query with an element that is not finite, NaN of any bits: NaN where it sees a pair, whatever the keys' signs, and no weight."""
    Hq, d, cap, held, T = form
    rng = np.random.default_rng(held + T + 1)
    values = (0x7F80, 0xFF80, 0x7F81, 0xFFFF) if dtype == "bf16" else (0x7F800000, 0xFF800000, 0x7F800001, 0xFFFFFFFF, 0x7F80FFFF)
    for n, v in enumerate(values * 2):
        c = lb.LolaFullCache(2, Hq, 1, d, cap, dtype=dtype, out_dtype=out, device=DEV)
        if held:
            k = tokens(rng, (2, 1, held, d), dtype).abs()      # (keys of one sign: logits that are all -inf or all +inf; then some zero keys too)
            if n >= len(values):
                k[:, :, ::3] = 0
            c.append(k, k)
        k, q = tokens(rng, (2, 1, T, d), dtype).abs(), tokens(rng, (2, Hq, T, d), dtype)
        at, col, h = T // 2, (n * 37 + 5) % d, Hq - 1
        clean = q.clone()
        q[1, h, at, col] = bits(q, v).to(DEV)
        if T > 1:
            c.append(k, k)
            y = c.attend(q, gather=True)
        else:
            y = c.step(*(x[:, :, 0].contiguous() for x in (q, k, k)), gather=True)[:, :, None]
        y, w = y.float().cpu(), c.weight.clone()
        assert torch.isnan(y[1, h, at]).all(), (hex(v), y[1, h, at, :4])
        y[1, h, at] = 0.0
        assert torch.isfinite(y).all(), hex(v)
        assert torch.isfinite(w[:, 0, :held + T]).all()
        got, rows = w[:, 0, :held + T].double().sum(1).tolist(), Hq * T
        assert abs(got[0] - rows) < 1e-4 * rows and abs(got[1] - (rows - 1)) < 1e-4 * rows, (hex(v), got)
        # a query that sees nothing: zeros, whatever it holds
        c.reset()
        q = torch.cat((q, clean), 2)
        y = c.attend(q[:, :, at:at + T].contiguous()).float()
        assert not y.any(), hex(v)
