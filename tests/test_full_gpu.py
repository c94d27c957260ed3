"""The 8-bit full-context cache on the GPU against its 64-bit oracle.

Codes, scales, indices, counts: equal.  Outputs: |y - y64| <= top (off + P) + 1 ulp, with `off` from the oracle (roundings of the
logits and sums), top the largest |v|, and P what the probabilities' own rounding to the matrix cores' operand type may cost: for fp32
outputs two fp16 parts, 2^-21 each way, for bf16 outputs one fp16 number, 2^-11 each way (numerator and what it is divided by).
The last rounding to the output's type is half a step: 2^-8 of the value for bf16, 2^-23 with what precedes it for fp32."""
import numpy as np
import pytest
import torch

import full_oracle as fo
from paper_2505_23666_amd import binding as lb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}


def rng_tokens(rng, shape, dtype, gain=1.0):
    x = torch.from_numpy(rng.standard_normal(shape).astype(np.float32) * gain).to(TORCH[dtype])
    return x, x.double().numpy()


class Pair:
    """A cache and its oracle, fed the same tokens."""

    def __init__(self, B, Hq, Hkv, d, cap, dtype="bf16", out="f32", tokens_first=False, scale=0.0, poison=True):
        self.c = lb.LolaFullCache(B, Hq, Hkv, d, cap, dtype=dtype, out_dtype=out, tokens_first=tokens_first, scale=scale, device=DEV)
        if poison:   # what no token was written to is never read: NaN codes, scales and weights, indices that every query would see
            self.c.k.view(torch.uint8).fill_(0x7F)
            self.c.v.view(torch.uint8).fill_(0xFF)
            self.c.k_scale.fill_(float("nan"))
            self.c.v_scale.fill_(float("inf"))
            self.c.weight.fill_(float("nan"))
            self.c.idx.fill_(-7)
        self.o = fo.FullOracle(B, Hq, Hkv, d, self.c.capacity, scale)
        self.dtype, self.out, self.tf = dtype, out, tokens_first

    def lay(self, x):
        return (x.transpose(1, 2) if self.tf else x).contiguous().to(DEV)

    def append(self, k, v, lens=None):
        self.c.append(self.lay(k), self.lay(v), None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV))
        self.o.append(k.double().numpy(), v.double().numpy(), lens)

    def check_memory(self, weights=True):
        c = self.c
        get = {n: getattr(c, n).float().cpu().numpy() if n in ("k", "v") else getattr(c, n).cpu().numpy() for n in c.FIELDS}
        for b, h, s in self.o.each():
            n, nb = s.count, (s.count + 63) // 64
            assert get["count"][b, h] == n and get["n_tokens"][b, h] == s.n
            assert np.array_equal(get["k_scale"][b, h, :nb], np.ldexp(1.0, s.ek[:nb])), (b, h)
            assert np.array_equal(get["v_scale"][b, h, :nb], np.ldexp(1.0, s.ev[:nb])), (b, h)
            for name, want in (("k", s.k), ("v", s.v)):
                diff = ~((get[name][b, h, :n] == want[:n]) | (np.isnan(get[name][b, h, :n]) & np.isnan(want[:n])))
                assert not diff.any(), f"{name}[{b},{h}]: {int(diff.sum())} codes differ, first at {np.argwhere(diff)[0]}"
            assert np.array_equal(get["idx"][b, h, :n], s.idx[:n]), (b, h)
            if weights:
                assert np.array_equal(np.isnan(get["weight"][b, h, :n]), np.isnan(s.weight[:n]))
                ok = ~np.isnan(s.weight[:n])
                assert np.array_equal(get["weight"][b, h, :n][ok].astype(np.float64), s.weight[:n][ok]), (b, h)

    def check_out(self, y, q, lens=None, gather=False, before=None):
        """y: the GPU's outputs [B, Hq, T, d]; before: the GPU's weights before the call, from which the oracle goes on."""
        if before is not None:
            for b, h, s in self.o.each():
                s.weight[:s.count] = before[b, h, :s.count].double().cpu().numpy()
        want, off, top, woff = self.o.attend(q.double().numpy(), lens, gather)
        y = (y.transpose(1, 2) if self.tf else y).double().cpu().numpy()
        P = 2.0 ** -21 * 2 if self.out == "f32" else 2.0 ** -11 * 2
        ulp = 2.0 ** -23 if self.out == "f32" else 2.0 ** -8
        nan = np.isnan(want)
        assert np.array_equal(nan, np.isnan(y))
        bound = (top * (off + P))[..., None] + ulp * np.abs(want) + 1e-37
        err = np.abs(np.where(nan, 0, y) - np.where(nan, 0, want))
        worst = (err / np.where(nan, 1, bound)).max() if err.size else 0.0
        assert worst <= 1, f"outputs {worst:.3g} times what roundings allow, at {np.unravel_index((err / bound).argmax(), err.shape)}"
        if gather:
            w = self.c.weight.double().cpu().numpy()
            for b, h, s in self.o.each():
                n = s.count
                # (plus the sum's own rounding of up to T * g terms, each at most the sum)
                lim = woff[b, h] + (2.0 ** -24 * (q.shape[2] * self.o.g + 4) + 2.0 ** -21) * s.weight[:n] + 1e-37
                assert (np.abs(w[b, h, :n] - s.weight[:n]) <= lim).all(), (b, h, np.abs(w[b, h, :n] - s.weight[:n]).max())
        return worst

    def attend(self, q, lens=None, gather=False):
        before = self.c.weight.clone() if gather else None
        y = self.c.attend(self.lay(q), None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV), gather=gather)
        torch.cuda.synchronize()
        return self.check_out(y, q, lens, gather, before)

    def step(self, q, k, v, gather=False):
        """q, k, v [B, H, 1, d]"""
        self.o.append(k.double().numpy(), v.double().numpy())
        before = self.c.weight.clone() if gather else None
        y = self.c.step(*(x[:, :, 0].contiguous().to(DEV) for x in (q, k, v)), gather=gather)
        torch.cuda.synchronize()
        if gather:   # the new pair's weight begins at zero
            for b, h, s in self.o.each():
                before[b, h, s.count - 1] = 0.0
        y = y[:, None] if self.tf else y[:, :, None]
        return self.check_out(y, q, None, gather, before)

    def tokens(self, rng, T, gain=1.0):
        B, Hq, Hkv, d = self.c.B, self.c.Hq, self.c.Hkv, self.c.d
        return (rng_tokens(rng, (B, Hq, T, d), self.dtype)[0], rng_tokens(rng, (B, Hkv, T, d), self.dtype, gain)[0],
                rng_tokens(rng, (B, Hkv, T, d), self.dtype, gain)[0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 128, 256])
@pytest.mark.parametrize("tokens_first", [False, True])
def test_append_codes(dtype, d, tokens_first):
    """Every way of cutting tokens into calls; magnitudes that make a block's exponent grow, tiny and zero blocks, ties."""
    rng = np.random.default_rng(d)
    p = Pair(2, 4, 2, d, 640, dtype, tokens_first=tokens_first)
    for T, gain, lens in ((1, 1, None), (1, 8, None), (61, 0.01, None), (1, 1, None), (3, 300, [3, 0]), (1, 1, None), (64, 1e-30, None), (65, 0, [1, 65]),
                          (130, 2.0, [130, 97]), (2, 1e30, None), (200, 1.0, [200, 5])):
        _, k, v = p.tokens(rng, T, gain)
        if T == 130:   # multiples of 1/16: many ties
            k, v = ((x * 16).round() / 16 for x in (k, v))
            k, v = k.to(TORCH[dtype]), v.to(TORCH[dtype])
        p.append(k, v, lens)
        p.check_memory()


def test_append_special_values():
    rng = np.random.default_rng(5)
    p = Pair(1, 2, 2, 64, 256)
    q, k, v = p.tokens(rng, 100)
    k[0, 0, 3, 7] = float("nan")
    v[0, 0, 40, 1] = float("inf")
    v[0, 1, 70, 63] = float("-inf")
    k[0, 1, 64:100] = 0
    v[0, 1, 64:99] = 0
    p.append(k, v)
    p.check_memory()
    p.attend(q)     # queries before token 3 see no NaN, those from it on see nothing else
    p.append(*p.tokens(rng, 70)[1:])
    p.check_memory()


def test_append_beyond_capacity():
    """The host refuses what it knows will not fit; the device stores what fits."""
    rng = np.random.default_rng(6)
    p = Pair(2, 2, 1, 32, 128)
    _, k, v = p.tokens(rng, 100)
    p.append(k, v, [100, 60])
    q, k, v = p.tokens(rng, 40)
    with pytest.raises(lb.LolaError, match="evict"):
        p.append(k, v)
    p.append(k[:, :, :28], v[:, :, :28])      # the first sequence is full now, the second is not
    p.check_memory()
    lb.lola_full_append(p.c.cfg, p.c.st, k.to(DEV), v.to(DEV), None, 40)
    p.o.append(k.double().numpy(), v.double().numpy())
    p.check_memory()
    assert p.c.count[:, 0].tolist() == [128, 128] and p.c.n_tokens[:, 0].tolist() == [168, 128]
    p.attend(q)


CASES = [  # B, Hq, Hkv, d, context, T
    (1, 1, 1, 64, 0, 1), (2, 4, 2, 32, 63, 1), (2, 8, 2, 128, 64, 1), (1, 6, 2, 64, 200, 1), (1, 5, 1, 128, 129, 1), (2, 14, 2, 128, 300, 1),
    (1, 32, 1, 64, 100, 1), (1, 40, 1, 32, 77, 1), (1, 2, 2, 256, 333, 1), (3, 8, 8, 64, 700, 1),
    (1, 4, 1, 128, 70, 2), (2, 6, 2, 64, 190, 5), (1, 4, 2, 256, 65, 3), (1, 14, 2, 32, 40, 9),
    (2, 4, 1, 64, 0, 33), (1, 8, 2, 128, 0, 64), (1, 6, 2, 64, 0, 65), (2, 8, 2, 128, 0, 257), (1, 7, 1, 32, 0, 130), (1, 2, 1, 256, 0, 150),
    (1, 8, 2, 128, 500, 40), (2, 4, 4, 64, 321, 129), (1, 8, 1, 32, 1000, 17),
]


@pytest.mark.parametrize("shape", CASES, ids=lambda s: "-".join(map(str, s)))
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
def test_attend(shape, dtype, out):
    B, Hq, Hkv, d, ctx, T = shape
    rng = np.random.default_rng(sum(shape))
    for tokens_first, ragged, gather in ((False, False, False), (True, True, True)):
        p = Pair(B, Hq, Hkv, d, ctx + T, dtype, out, tokens_first)
        if ctx:
            p.append(*p.tokens(rng, ctx, 1.3)[1:], [max(1, ctx - 37 * b) for b in range(B)] if ragged else None)
        q, k, v = p.tokens(rng, T)
        lens = [(0, T, (T + 1) // 2)[(b + 1) % 3] for b in range(B)] if ragged and T > 1 else None
        p.append(k, v, lens)
        worst = p.attend(q, lens, gather)
        print(f"attend {shape} {dtype}->{out} {'ragged' if ragged else ''}: {worst:.3f} of the bound", flush=True)
        if gather:     # a second call adds to the weights
            p.attend(q, lens, True)
        p.check_memory(weights=False)


def test_attend_empty_and_extreme():
    """Empty caches and rows that see nothing give zeros; lens outside 0 .. T count as the nearer end; large logits; a peaked row."""
    rng = np.random.default_rng(11)
    p = Pair(3, 4, 2, 64, 256, out="bf16")
    q, k, v = p.tokens(rng, 20)
    y = p.c.attend(q.to(DEV))
    assert not y.any()
    p.append(k, v, [0, -5, 99])       # -5 counts as 0, 99 as 20
    assert p.c.count[:, 0].tolist() == [0, 0, 20]
    p.attend(q, [0, -5, 99], gather=True)
    p.attend(q)                        # the first two sequences have no pairs: 20 queries each that see nothing
    # more queries than tokens: the oldest see nothing
    q2 = p.tokens(rng, 50)[0]
    p.attend(q2, gather=True)
    big = Pair(1, 2, 1, 128, 300, scale=3.0)
    q, k, v = big.tokens(rng, 257, 4.0)
    big.append(k, v)
    big.attend(q, gather=True)


def test_attend_scales_far_apart():
    """Blocks whose scales differ by many powers of two: values of a block of 1e-20 beside one of 1e3, an all-zero block."""
    rng = np.random.default_rng(12)
    for out in ("f32", "bf16"):
        p = Pair(1, 4, 1, 64, 64 * 6, out=out)
        for gain in (1.0, 1e-20, 1e3, 0.0, 1e-3):
            _, k, v = p.tokens(rng, 64)
            p.append(k, v * gain)
        q, k, v = p.tokens(rng, 3)
        p.append(k, v)
        p.check_memory()
        p.attend(q)
        q = p.tokens(rng, 60)[0]
        p.attend(q)


@pytest.mark.parametrize("g,d", [(20, 64), (32, 128), (17, 32), (16, 256), (17, 256)])
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("f32", "f32")])
def test_steps_of_wide_groups(g, d, dtype, out):
    """Generation steps with 16 to 32 query heads per kv head (two column tiles; at d = 256 the prompt kernel from 17 on), a block filling up."""
    rng = np.random.default_rng(g + d)
    p = Pair(1, 2 * g, 2, d, 640, dtype, out)
    p.append(*p.tokens(rng, 61)[1:])
    for t in range(6):
        p.step(*p.tokens(rng, 1, 0.5 * 2 ** t), gather=t % 2 == 1)     # (growing magnitudes: the block is rescaled in the step)
        p.check_memory(weights=False)


def test_step_of_many_streams():
    """More streams than compute units: one workgroup of eight wavefronts each, caches beyond 512 slots."""
    rng = np.random.default_rng(77)
    p = Pair(65, 16, 4, 32, 1024, out="f32")
    p.append(*p.tokens(rng, 700)[1:], [700 - 10 * b for b in range(65)])
    p.step(*p.tokens(rng, 1))
    p.step(*p.tokens(rng, 1), gather=True)
    p.check_memory(weights=False)


def test_single_tokens_with_lens():
    """attend of one token where some sequences have none."""
    rng = np.random.default_rng(78)
    for cap in (128, 4096):
        p = Pair(3, 8, 2, 64, cap)
        p.append(*p.tokens(rng, 70)[1:])
        q, k, v = p.tokens(rng, 1)
        p.append(k, v, [1, 0, 1])
        p.check_memory()
        p.attend(q, [1, 0, 1], gather=True)


def test_step_on_a_full_cache():
    """The library stores what fits: the token of a full stream is counted and not stored, its query sees what is there."""
    rng = np.random.default_rng(79)
    for gather in (False, True):
        p = Pair(2, 4, 1, 64, 128)
        p.append(*p.tokens(rng, 128)[1:], [128, 100])
        q, k, v = p.tokens(rng, 1)
        before = p.c.weight.clone()
        y = torch.empty((2, 4, 64), device=DEV)
        ws = torch.empty(lb.lola_full_workspace_bytes(p.c.cfg, 1, True), dtype=torch.uint8, device=DEV)
        lb.lola_full_step(p.c.cfg, p.c.st, *(x[:, :, 0].contiguous().to(DEV) for x in (q, k, v)), int(gather), y, ws)
        p.o.append(k.double().numpy(), v.double().numpy())
        before[1, 0, 100] = 0
        p.check_memory(weights=False)
        p.check_out(y[:, :, None], q, None, gather, before if gather else None)
        with pytest.raises(lb.LolaError, match="evict"):
            p.c.step(*(x[:, :, 0].contiguous().to(DEV) for x in (q, k, v)))


def test_weights_beside_nan_tokens():
    """Queries that see a NaN token add no weight; those before it do."""
    rng = np.random.default_rng(80)
    for T in (6, 100):
        p = Pair(1, 4, 1, 64, 256)
        q, k, v = p.tokens(rng, T)
        k[0, 0, T // 2, 3] = float("nan")
        p.append(k, v)
        p.attend(q, gather=True)


def test_large_fp32_queries():
    """fp32 queries up to the largest finite number enter the products unchanged (tiny keys keep the logits finite)."""
    rng = np.random.default_rng(81)
    for T in (1, 40):
        p = Pair(1, 4, 1, 64, 128, "f32")
        q, k, v = p.tokens(rng, T)
        q = torch.sign(q) * 3.4e38
        p.append(k * 2.0 ** -100, v)
        p.c.cfg.softmax_scale = p.o.scale = 2.0 ** -28
        p.attend(q)


def test_captured_calls_and_the_bound_on_the_host():
    """Replays are not seen by the host: calls outside the graph look at the counts; a workspace that a graph uses outlives a larger one."""
    rng = np.random.default_rng(82)
    c = lb.LolaFullCache(1, 4, 1, 64, 256, device=DEV)
    tok = [x.to(DEV) for x in (rng_tokens(rng, (1, 4, 64), "bf16")[0], rng_tokens(rng, (1, 1, 64), "bf16")[0], rng_tokens(rng, (1, 1, 64), "bf16")[0])]
    c.step(*tok)
    out = torch.empty((1, 4, 64), device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.step(*tok, out=out, gather=True)
    used = c.workspace
    for _ in range(250):
        graph.replay()
    assert int(c.count.max()) == 251
    kv = tok[1][:, :, None].expand(1, 1, 6, 64).contiguous()
    with pytest.raises(lb.LolaError, match="evict"):
        c.append(kv, kv)
    c.append(kv[:, :, :5].contiguous(), kv[:, :, :5].contiguous())
    q = tok[0][:, :, None].expand(1, 4, 200, 64).contiguous()
    c.attend(q, gather=True)
    assert c.workspace is used or any(w is used for w in c._outgrown)
    graph.replay()      # full: the token is not stored
    torch.cuda.synchronize()
    assert int(c.count.max()) == 256 and int(c.n_tokens.max()) == 257
    c.evict(10)
    c.append(kv, kv)
    assert int(c.count.max()) == 16


@pytest.mark.parametrize("d", [32, 64, 128, 256])
@pytest.mark.parametrize("n,keep,first,recent", [(200, 64, 0, 0), (200, 100, 4, 10), (130, 129, 0, 1), (300, 1, 0, 0), (300, 0, 0, 0), (257, 192, 3, 0),
                                                 (64, 64, 0, 0), (640, 77, 40, 37), (640, 600, 0, 16)])
def test_evict(d, n, keep, first, recent):
    rng = np.random.default_rng(n + keep)
    p = Pair(2, 2, 2, d, 640)
    for part in (n // 3, n - n // 3):
        _, k, v = p.tokens(rng, part)
        k, v = (x * torch.from_numpy(np.ldexp(1.0, rng.integers(-6, 7, (1, 1, part, 1)))).to(x.dtype) for x in (k, v))   # (powers of two: exact)
        p.append(k, v, [part, max(1, part - 9)])
    # weights with many ties, zeros of both signs, infinities and NaN
    w = rng.integers(0, 6, (2, 2, p.c.capacity)).astype(np.float32) / 4
    w[rng.random(w.shape) < 0.05] = -0.0
    w[rng.random(w.shape) < 0.02] = np.inf
    w[rng.random(w.shape) < 0.02] = np.nan
    p.c.weight.copy_(torch.from_numpy(w))
    for b, h, s in p.o.each():
        s.weight[:] = w[b, h]
    p.c.workspace = torch.full((lb.lola_full_workspace_bytes(p.c.cfg, 0),), 0xA5, dtype=torch.uint8, device=DEV)
    p.c.evict(keep, first, recent)
    p.o.evict(keep, first, recent)
    p.check_memory()
    p.c.evict(keep, first, recent)      # nothing left to do
    p.check_memory()
    q, k, v = p.tokens(rng, 30)         # the cache goes on from there
    p.append(k, v)
    p.check_memory()
    p.attend(q)


@pytest.mark.parametrize("d,cap,n,keep", [(32, 2048, 2000, 1000), (64, 2048, 1900, 777), (128, 1344, 1344, 640), (256, 1280, 1280, 601), (64, 10240, 9000, 1000),
                                          (32, 36864, 35000, 3000)])
def test_evict_from_longer_caches(d, cap, n, keep):
    """Many pairs move, blocks of very different scales among them."""
    rng = np.random.default_rng(cap + d)
    p = Pair(1, 2, 2, d, cap)
    _, k, v = p.tokens(rng, n)
    k, v = (x * torch.from_numpy(np.ldexp(1.0, rng.integers(-9, 10, (1, 2, n, 1)))).to(x.dtype) for x in (k, v))
    p.append(k, v)
    w = rng.integers(0, 400, (1, 2, cap)).astype(np.float32) / 64
    w[rng.random(w.shape) < 0.01] = np.nan
    p.c.weight.copy_(torch.from_numpy(w))
    for b, h, s in p.o.each():
        s.weight[:] = w[b, h]
    for to in (keep, keep - keep // 3):
        p.c.evict(to, 4, 50)
        p.o.evict(to, 4, 50)
        p.check_memory()


def test_evict_many_pairs_and_streams():
    """Distinct weights over several thousand slots: ranks that differ in their lowest bits alone."""
    rng = np.random.default_rng(3)
    p = Pair(3, 3, 3, 32, 5120)
    _, k, v = p.tokens(rng, 5000)
    p.append(k, v, [5000, 4100, 2500])
    w = (1.0 + rng.permutation(3 * 3 * 5120).reshape(3, 3, 5120) * 2.0 ** -23).astype(np.float32)
    p.c.weight.copy_(torch.from_numpy(w))
    for b, h, s in p.o.each():
        s.weight[:] = w[b, h]
    p.c.evict(3333, 5, 100)
    p.o.evict(3333, 5, 100)
    p.check_memory()


@pytest.mark.parametrize("dtype,out,heads", [("bf16", "bf16", (8, 2, 128)), ("bf16", "f32", (6, 2, 64)), ("f32", "f32", (4, 1, 32))])
def test_generation_under_a_budget(dtype, out, heads):
    """As a server runs it: a ragged batch of prompts whose attention gathers weights, cut to a budget; steps that go on gathering, an
    eviction every few; a further turn of several tokens on the cache whose slots are out of order by now."""
    rng = np.random.default_rng(heads[0])
    Hq, Hkv, d = heads
    p = Pair(2, Hq, Hkv, d, 320, dtype, out)
    q, k, v = p.tokens(rng, 200)
    p.append(k, v, [200, 131])
    p.attend(q, [200, 131], gather=True)

    def evict():
        w = p.c.weight.double().cpu().numpy()
        for b, h, s in p.o.each():      # the oracle ranks by the weights that the GPU ranks by
            s.weight[:s.count] = w[b, h, :s.count]
        p.c.evict(100, first=4, recent=20)
        p.o.evict(100, 4, 20)
        p.check_memory()

    evict()
    for t in range(24):
        p.step(*p.tokens(rng, 1), gather=t % 2 == 0)
        if t % 7 == 6:
            evict()
    q, k, v = p.tokens(rng, 90)
    p.append(k, v, [41, 90])
    p.attend(q, [41, 90], gather=True)
    evict()
    p.step(*p.tokens(rng, 1))


def test_step_is_append_and_attend():
    rng = np.random.default_rng(21)
    a, b = Pair(4, 8, 2, 128, 512, out="bf16"), Pair(4, 8, 2, 128, 512, out="bf16")
    q, k, v = a.tokens(rng, 200)
    for p in (a, b):
        p.append(k, v, [200, 1, 63, 64])
    for _ in range(3):
        q, k, v = (x.to(DEV) for x in a.tokens(rng, 1))
        y = a.c.step(q[:, :, 0].contiguous(), k[:, :, 0].contiguous(), v[:, :, 0].contiguous(), gather=True)
        b.c.append(k, v)
        z = b.c.attend(q, gather=True)[:, :, 0]
        for n in a.c.FIELDS:
            x, w = getattr(a.c, n), getattr(b.c, n)
            live = [slice(None)] * x.dim()
            assert torch.equal(x.view(torch.uint8)[..., :0], w.view(torch.uint8)[..., :0])
            for s in range(4):
                c = int(a.c.count[s, 0])
                m = {"k": c, "v": c, "idx": c, "weight": c, "k_scale": (c + 63) // 64, "v_scale": (c + 63) // 64}.get(n)
                i, j = (x[s], w[s]) if m is None else (x[s, :, :m], w[s, :, :m])
                if n == "weight":   # (the step may sum a row's shares in another split)
                    assert torch.allclose(i, j, rtol=1e-5, atol=1e-7)
                else:
                    assert torch.equal(i.contiguous().view(torch.uint8), j.contiguous().view(torch.uint8)), n
        assert torch.allclose(y.float(), z.float(), rtol=2.0 ** -7, atol=1e-5)


def test_repeatable_and_other_stream():
    """The same calls twice give the same bits; on a stream of their own too."""
    rng = np.random.default_rng(31)
    results = []
    tok = None
    for side in (False, False, True):
        p = Pair(2, 8, 2, 64, 1024)
        if tok is None:
            tok = [[x.to(DEV) for x in p.tokens(rng, n)] for n in (700, 64, 1, 1)]
        s = torch.cuda.Stream() if side else torch.cuda.current_stream()
        s.wait_stream(torch.cuda.current_stream())
        outs = []
        with torch.cuda.stream(s):
            for q, k, v in tok[:2]:
                p.c.append(k, v)
                outs.append(p.c.attend(q, gather=True))
            p.c.evict(333, 2, 50)
            for q, k, v in tok[2:]:
                outs.append(p.c.step(q[:, :, 0].contiguous(), k[:, :, 0].contiguous(), v[:, :, 0].contiguous(), gather=True))
        s.synchronize()
        results.append(outs + [p.c.weight[:, :, :335].clone(), p.c.k[:, :, :335].view(torch.uint8).clone(), p.c.idx[:, :, :335].clone()])
    for r in results[1:]:
        for x, y in zip(results[0], r):
            assert torch.equal(x, y)


def test_graph_replays():
    """A step with weights and an eviction captured once and replayed, eager work between the replays, against the same calls made one by one."""
    rng = np.random.default_rng(41)
    a, b = Pair(2, 8, 2, 64, 512), Pair(2, 8, 2, 64, 512)
    q, k, v = (x.to(DEV) for x in a.tokens(rng, 300))
    for p in (a, b):
        p.c.append(k, v)
        p.c.attend(q, gather=True)
        p.c.evict(256, 2, 20)
    steps = [[x[:, :, 0].contiguous().to(DEV) for x in a.tokens(rng, 1)] for _ in range(6)]
    fixed = [x.clone() for x in steps[0]]
    out = torch.empty((2, 8, 64), device=DEV)
    a.c.evict(256, 2, 20)     # (the workspace exists before the capture)
    a.c._ws(1, True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.c.step(*fixed, out=out, gather=True)
        a.c.evict(256, 2, 20)
    for t, s in enumerate(steps):
        for f, x in zip(fixed, s):
            f.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        want = b.c.step(*s, gather=True)
        b.c.evict(256, 2, 20)
        torch.zeros(1 << 20, device=DEV).sum().item()
        assert torch.equal(out, want), t
        for n in ("count", "n_tokens"):
            assert torch.equal(getattr(a.c, n), getattr(b.c, n))
        for n in ("k", "v", "idx", "weight"):
            assert torch.equal(getattr(a.c, n)[:, :, :256].view(torch.uint8), getattr(b.c, n)[:, :, :256].view(torch.uint8)), (t, n)


def test_graphs_that_share_a_workspace_and_calls_side_by_side():
    """Nothing lives in a workspace between calls: two captured graphs of different caches share one and are replayed in turn; and two
    caches with workspaces of their own go through the same calls on two streams at once."""
    rng = np.random.default_rng(43)
    ps = [Pair(2, 8, 2, 64, 2048) for _ in range(4)]
    q, k, v = (x.to(DEV) for x in ps[0].tokens(rng, 1500))
    tok = [[x[:, :, 0].contiguous().to(DEV) for x in ps[0].tokens(rng, 1)] for _ in range(8)]
    for p in ps:
        p.c.append(k, v)
        p.c.attend(q, gather=True)
    want = []
    for x in tok:
        want.append(ps[0].c.step(*x, gather=True))
        ps[0].c.evict(1400, 2, 50)
    graphs, fixed = [], [x.clone() for x in tok[0]]
    ps[1].c._ws(1, 1)
    ps[2].c.workspace = ps[1].c.workspace
    outs = [torch.empty((2, 8, 64), device=DEV) for _ in range(2)]
    for p, out in zip(ps[1:3], outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            p.c.step(*fixed, out=out, gather=True)
            p.c.evict(1400, 2, 50)
    for x, y in zip(tok, want):
        for f, z in zip(fixed, x):
            f.copy_(z)
        for g, out in zip(graphs, outs):
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, y)
    # side by side with another cache on another stream
    other = Pair(2, 8, 2, 64, 2048)
    other.c.append(k, v)
    other.c.attend(q, gather=True)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = ([], [])
    torch.cuda.synchronize()
    for x in tok:
        for st, p, o in zip(streams, (ps[3], other), got):
            with torch.cuda.stream(st):
                o.append(p.c.step(*x, gather=True))
                p.c.evict(1400, 2, 50)
    torch.cuda.synchronize()
    for o in got:
        for y, z in zip(o, want):
            assert torch.equal(y, z)


def test_offsets_beyond_32_bits():
    """A second stream whose rows begin beyond 2^32 bytes: zero keys weigh all pairs alike, so the output is the mean of the values."""
    cap, d = 1 << 24, 256
    mem = {n: torch.zeros((1, 2, cap, d), dtype=torch.float8_e4m3fn, device=DEV) for n in ("k", "v")}
    mem.update(k_scale=torch.ones((1, 2, cap // 64), device=DEV), v_scale=torch.ones((1, 2, cap // 64), device=DEV),
               idx=torch.arange(cap, dtype=torch.int32, device=DEV).expand(1, 2, cap).contiguous(), weight=torch.zeros((1, 2, cap), device=DEV),
               count=torch.full((1, 2), cap - 100, dtype=torch.int32, device=DEV), n_tokens=torch.full((1, 2), cap - 100, dtype=torch.int64, device=DEV))
    c = lb.LolaFullCache(1, 2, 2, d, cap, buffers=mem, device=DEV)
    k = torch.zeros((1, 2, d), dtype=torch.bfloat16, device=DEV)
    v = torch.full((1, 2, d), 1.0, dtype=torch.bfloat16, device=DEV)
    mem["v"].view(torch.uint8)[0, 1, cap - 128:cap - 64] = 0x38       # 1.0
    y = c.step(k, k, v, gather=True)
    n = cap - 99
    assert int(c.count.min()) == n
    assert torch.allclose(y[0, 1], torch.full((d,), 29 / n, device=DEV), rtol=1e-4) and torch.allclose(y[0, 0], torch.full((d,), 1 / n, device=DEV), rtol=1e-4)
    assert torch.allclose(c.weight[:, :, [0, 5, n - 1]], torch.full((1, 2, 3), 1 / n, device=DEV), rtol=1e-4)
    c.weight[:, :, cap // 2:n] += 1
    c.evict(cap // 2, 0, 0)
    assert int(c.idx[0, 1, :cap // 2].min()) >= 0 and int((c.idx[0, 1, :cap // 2] >= cap // 2).sum()) == n - cap // 2
    assert float(c.v[0, 1, :cap // 2].float().sum()) == 29 * d


def test_python_refusals():
    c = lb.LolaFullCache(2, 4, 2, 64, 100, device=DEV)
    assert c.capacity == 128
    bf = dict(dtype=torch.bfloat16, device=DEV)
    k, q = torch.zeros((2, 2, 8, 64), **bf), torch.zeros((2, 4, 8, 64), **bf)
    bad = [lambda: c.append(k.float(), k.float()), lambda: c.append(k, k[:, :, :4].contiguous()), lambda: c.append(k.transpose(1, 2), k.transpose(1, 2)),
           lambda: c.append(k.cpu(), k.cpu()), lambda: c.append(q, q), lambda: c.attend(k), lambda: c.append(k, k, torch.zeros(2, device=DEV)),
           lambda: c.append(k, k, torch.zeros(3, dtype=torch.int32, device=DEV)), lambda: c.attend(q, out=torch.empty((2, 4, 8, 64), **bf)),
           lambda: c.step(q[:, :, 0].contiguous(), k, k), lambda: c.step(q[:, :, 0], k[:, :, 0].contiguous(), k[:, :, 0].contiguous()),
           lambda: c.evict(129), lambda: c.evict(10, 6, 5), lambda: c.evict(-1),
           lambda: lb.LolaFullCache(2, 4, 2, 64, 128, weights=False, device=DEV).evict(10),
           lambda: lb.LolaFullCache(2, 4, 2, 64, 128, weights=False, device=DEV).attend(q, gather=True),
           lambda: lb.LolaFullCache(2, 4, 2, 60, 128, device=DEV), lambda: lb.LolaFullCache(2, 4, 2, 64, 128, buffers={"k": k}, device=DEV)]
    for i, f in enumerate(bad):
        with pytest.raises(lb.LolaError):
            f()
            print("accepted:", i)
    assert int(c.count.sum()) == 0
