"""How near the 8-bit full-context cache's outputs and weights are to 64 bits as a whole (2-norm), which a bound per element cannot pin down.

fp32 outputs: every number that goes into an output has 2^-22 of relative error or less (queries as three bf16 parts 2^-24, weights as two fp16
parts 2^-22, the exponential 2^-22, fp32 sums 2^-24 a term, partly cancelling), a logit of size x adds x 2^-24 for each of the some ten sums of
its products: with |x| < 10 the whole is a few 2^-23, below 1e-6.  A lost part costs more: queries in two parts 2^-16 of a logit, 2e-6 and more in
the output, weights in one part 2^-12, 1e-4.  bf16 outputs: the rounding of the result is 2^-8 of an element at most, weights in one fp16 part 2^-11."""
import math

import numpy as np
import pytest
import torch

import full_dense as fd
from paper_2505_23666_amd import binding as lb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
NORM = {"f32": 1e-6, "bf16": 2.0 ** -8 + 2.0 ** -11}


def tokens(rng, shape, dtype, gain=1.0):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32) * np.float32(gain)).to(TORCH[dtype]).to(DEV)


# Hq, Hkv, capacity, pairs held before, new tokens: step in one workgroup, in shares, two column tiles; few rows, in two tiles; many rows in one
# share, in several
FORMS = [(4, 2, 192, 150, 1), (8, 1, 4096, 3000, 1), (20, 1, 2048, 900, 1), (4, 1, 2048, 1000, 4), (8, 2, 2048, 500, 5), (4, 2, 512, 0, 300), (8, 2, 4096, 2000, 70)]


@pytest.mark.parametrize("d", [32, 64, 128, 256])
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
def test_distance_from_64_bits(d, dtype, out):
    for Hq, Hkv, cap, held, T in FORMS:
        rng = np.random.default_rng(d + held)
        c = lb.LolaFullCache(2, Hq, Hkv, d, cap, dtype=dtype, out_dtype=out, device=DEV)
        if held:
            c.append(tokens(rng, (2, Hkv, held, d), dtype, 1.3), tokens(rng, (2, Hkv, held, d), dtype))
        q, k, v = tokens(rng, (2, Hq, T, d), dtype), tokens(rng, (2, Hkv, T, d), dtype, 1.3), tokens(rng, (2, Hkv, T, d), dtype)
        if T > 1:
            c.append(k, v)
            y = c.attend(q)
        else:
            y = c.step(*(x[:, :, 0].contiguous() for x in (q, k, v)))[:, :, None]
        want, _ = fd.attend(c, q)
        off = fd.distance(y, want)
        print(f"outputs d {d} {dtype}->{out} {(Hq, Hkv, cap, held, T)}: {off:.3g}", flush=True)
        assert off <= NORM[out], (Hq, Hkv, cap, held, T, off)


@pytest.mark.parametrize("d", [32, 64, 128, 256])
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("f32", "f32")])
def test_huge_values_of_pairs_without_weight(d, dtype, out):
    """Pairs whose values are 2^50 times the others', in the first blocks, that a query does not see or gives no weight to (2^-92): its output is the
    other pairs' mean as if they were not there.  Relative to each row's own output, not to the largest value of the stream.  (A pair with weight in a block
    of huge values is another matter: it may be off by 2^(e - 10) as stored.)"""
    # (as many streams as leave every wavefront several blocks: one workgroup per stream, two column tiles in shares; few rows; many rows in one share, in two)
    for B, Hq, cap, held, T in ((256, 2, 1088, 1000, 1), (256, 20, 1088, 1000, 1), (256, 4, 1088, 1000, 4), (256, 8, 1088, 1000, 4), (128, 4, 1088, 900, 100),
                                (64, 4, 2112, 1900, 100)):
        rng = np.random.default_rng(d + T)
        c = lb.LolaFullCache(B, Hq, 1, d, cap, dtype=dtype, out_dtype=out, device=DEV)
        n = held + T
        k, v = (tokens(rng, (1, 1, n, d), dtype, gain).repeat(B, 1, 1, 1) for gain in (0.3, 1.0))
        q = tokens(rng, (B, Hq, T, d), dtype, 0.3)
        q[..., 0] = 8.0 * math.sqrt(d)
        k[..., 0] = 0.0
        late = T // 2
        k[:, :, :64, 0] = -8.0                  # logits 64 below: weights of 2^-92
        if late:
            k[:, :, 64 + late:128, 0] = -8.0
        v[:, :, :64] *= 2.0 ** 50
        c.append(k, v)
        if late:          # slots 64 .. hold the call's latest tokens, with huge values and large weights for the queries that see them
            move = torch.arange(n, device=DEV)
            move[64:64 + late], move[n - late:] = torch.arange(n - late, n, device=DEV), torch.arange(64, 64 + late, device=DEV)
            c.idx[:, :, :n] = move.int()
            c.v_scale[:, :, 1] *= 2.0 ** 50
        y = c.attend(q).double()
        want, _ = fd.attend(c, q)
        rows = slice(0, T - late)
        off = ((y - want).norm(dim=-1) / want.norm(dim=-1))[:, :, rows]
        print(f"huge values d {d} {dtype}->{out} {(B, Hq, cap, held, T)}: {float(off.max()):.3g}", flush=True)
        assert float(off.max()) <= 2 * NORM[out], (B, Hq, cap, held, T)
        assert torch.isfinite(y).all()


@pytest.mark.parametrize("d", [32, 128])
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("f32", "f32")])
def test_far_logits(d, dtype, out):
    """Logits of 2^23 and 2^25 (in powers of two) either way, where fp32 holds no fraction or not every whole number: the pairs with the largest share the weight, in blocks
    of unequal scales; a query all of whose logits are as far below gives all of them the same."""
    for B, Hq, cap, held, T in ((256, 2, 1088, 1000, 1), (256, 20, 1088, 1000, 1), (2, 4, 1088, 1000, 4), (2, 4, 4096, 3000, 100), (128, 4, 1088, 900, 100)):
        rng = np.random.default_rng(d + T)
        c = lb.LolaFullCache(B, Hq, 1, d, cap, dtype=dtype, out_dtype=out, device=DEV)
        n = held + T
        k, v = torch.zeros((B, 1, n, d), dtype=TORCH[dtype], device=DEV), tokens(rng, (1, 1, n, d), dtype).repeat(B, 1, 1, 1)
        k[..., 0], k[..., 1] = -1.0, -1.0
        k[:, :, ::37, 0] = 1.0
        v *= 2.0 ** torch.from_numpy(rng.integers(-2, 3, (1, 1, -(-n // 64)))).to(DEV).repeat_interleave(64, 2)[:, :, :n, None].to(v.dtype)
        c.append(k, v)
        q = torch.zeros((B, Hq, T, d), dtype=TORCH[dtype], device=DEV)
        q[:, ::2, :, 0] = q[:, 1::2, :, 1] = 2.0 ** 25 * (1.0 if d == 32 else 8.0)
        y = c.attend(q).double()
        want, _ = fd.attend(c, q)
        assert fd.distance(y, want) <= NORM[out], (B, Hq, cap, held, T, fd.distance(y, want))


@pytest.mark.parametrize("d", [32, 64, 128, 256])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_distance_of_gathered_weights(d, dtype):
    """A weight is off by its own exponential and normaliser (2^-23 each) and by what its logit is off (as above), which differ in sign from row to
    row: over a few hundred rows below 1.5e-7 (2^-22.7); a normaliser that errs to one side does not average out.  Of single steps 1e-6, as outputs."""
    for Hq, Hkv, cap, held, T in ((4, 2, 192, 150, 1), (8, 1, 4096, 3000, 1), (4, 1, 2048, 1000, 4), (8, 2, 1024, 0, 1000), (8, 2, 4096, 3000, 260)):
        rng = np.random.default_rng(d + held + 1)
        c = lb.LolaFullCache(2, Hq, Hkv, d, cap, dtype=dtype, device=DEV)
        if held:
            c.append(tokens(rng, (2, Hkv, held, d), dtype, 1.3), tokens(rng, (2, Hkv, held, d), dtype))
        q, k, v = tokens(rng, (2, Hq, T, d), dtype), tokens(rng, (2, Hkv, T, d), dtype, 1.3), tokens(rng, (2, Hkv, T, d), dtype)
        c.append(k, v)
        c.attend(q, gather=True)
        _, want = fd.attend(c, q)
        n = held + T
        off = fd.distance(c.weight[:, :, :n], want[:, :, :n])
        print(f"weights d {d} {dtype} {(Hq, Hkv, cap, held, T)}: {off:.3g}", flush=True)
        assert off <= (1e-6 if T < 10 else 1.5e-7), (Hq, Hkv, cap, held, T, off)


@pytest.mark.parametrize("d", [32, 64, 128, 256])
@pytest.mark.parametrize("dtype,out,below", [("bf16", "f32", 17), ("f32", "f32", 17), ("bf16", "bf16", 26)])
def test_small_weights_beside_a_large_one_without_value(d, dtype, out, below):
    """A sink: one pair takes nearly all of the weight and has the value zero, so that a row's output is made of weights of 2^-17 (2^-26) alone.  fp32
    outputs: a logit of 17 is off by 3 roundings of 2^-24 of it (the scale's two and its own), 2.2e-6 of the weights, their own two parts by 2^-21 at
    most: 3e-6 in all.  bf16 outputs: the rounding of the result and 2^-10 for the weights."""
    for B, Hq, cap, held, T in ((256, 2, 1088, 1000, 1), (2, 4, 4096, 3000, 1), (256, 20, 1088, 1000, 1), (2, 4, 1088, 1000, 4), (2, 4, 4096, 3000, 100), (128, 4, 1088, 900, 100)):
        rng = np.random.default_rng(d + T)
        c = lb.LolaFullCache(B, Hq, 1, d, cap, dtype=dtype, out_dtype=out, device=DEV)
        n = held + T
        k, v = (tokens(rng, (1, 1, n, d), dtype, gain).repeat(B, 1, 1, 1) for gain in (0.3, 1.0))
        k[..., 0] = 0.0
        k[:, :, 5] = 0.0
        k[:, :, 5, 0] = 8.0
        v[:, :, 5] = 0.0
        c.append(k, v)
        q = tokens(rng, (B, Hq, T, d), dtype, 1.0)
        q[..., 0] = below * math.log(2.0) * math.sqrt(d) / 8.0
        y = c.attend(q).double()
        want, _ = fd.attend(c, q)
        off = fd.distance(y, want)
        print(f"small weights d {d} {dtype}->{out} {(B, Hq, cap, held, T)}: {off:.3g}", flush=True)
        assert off <= (3e-6 if out == "f32" else NORM[out] + 2.0 ** -10), (B, Hq, cap, held, T, off)
