"""The norms that the GPU tests hold the 8-bit full-context cache to notice a lost operand part: the mistake is planted here, in the 64-bit formula."""
import numpy as np
import pytest

import full_oracle as fo

BOUND = 1e-6        # fp32 outputs
WEIGHTS = 1.5e-7    # gathered weights over many rows


def cut(x, parts):
    """x as the sum of its first `parts` bf16 parts, 8 bits each, cut off."""
    rest, total = np.asarray(x, np.float32), np.zeros(np.shape(x))
    for _ in range(parts):
        p = (rest.view(np.uint32) & 0xFFFF0000).view(np.float32)
        total, rest = total + p, rest - p
    return total


def halves(p, parts, shift):
    """Weights held times 2^shift as the sum of `parts` fp16 numbers."""
    rest, total = p * 2.0 ** shift, 0.0
    for _ in range(parts):
        h = rest.astype(np.float16).astype(np.float64)
        total, rest = total + h, rest - h
    return total * 2.0 ** -shift


def outputs(s, q, query_parts, weight_parts, shift):
    K, V = s.pairs()
    x = (q if query_parts is None else cut(q, query_parts)) @ K.T / np.sqrt(q.shape[1])
    e = np.exp(x - x.max(1, keepdims=True))
    total = e.sum(1, keepdims=True)
    return (e if weight_parts is None else halves(e, weight_parts, shift)) @ V / total, (e / total).sum(0)


@pytest.mark.parametrize("d", [32, 64, 128, 256])
@pytest.mark.parametrize("n,rows", [(151, 2), (3001, 8), (1004, 4), (370, 70)])
def test_a_lost_part_is_noticed(d, n, rows):
    rng = np.random.default_rng(d + n)
    s = fo.Stream(-(-n // 64) * 64, d)
    s.append(rng.standard_normal((n, d)) * 1.3, rng.standard_normal((n, d)))
    q = rng.standard_normal((rows, d)).astype(np.float32)
    want, weight = outputs(s, q, None, None, 0)
    off = lambda x, y: np.linalg.norm(x - y) / np.linalg.norm(y)  # noqa: E731
    for shift in (13, 14):
        assert off(outputs(s, q, 3, 2, shift)[0], want) < BOUND / 3          # what the format itself costs
        assert off(outputs(s, q, 3, 1, shift)[0], want) > 10 * BOUND         # one fp16 part
    y, w = outputs(s, q, 2, 2, 14)                                           # two parts of the queries
    assert off(y, want) > BOUND and off(w, weight) > 3 * WEIGHTS
