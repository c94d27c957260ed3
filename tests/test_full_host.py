"""Host-side checks of the 8-bit full-context cache that need no GPU: sizes, refusals before anything is launched, and the oracle's
own number format against torch's."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

import full_oracle as fo
from paper_2505_23666_amd import binding as lb


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(lb.LIB_PATH):
        from paper_2505_23666_amd import build
        build.build_library()
    return lb.lib()


def cfg(**kw):
    base = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=128, capacity=256, dtype=lb.LOLA_BF16, out_dtype=lb.LOLA_F32, tokens_first=0,
                softmax_scale=0.0)
    base.update(kw)
    return lb.LolaFullConfig(**base)


def test_state_bytes(L):
    tot, fb = lb.lola_full_state_bytes(cfg())
    assert fb == [4 * 256 * 128, 4 * 256 * 128, 4 * 4 * 4, 4 * 4 * 4, 4 * 256 * 4, 4 * 256 * 4, 4 * 4, 4 * 8] and tot == sum(fb)
    # offsets beyond 32 bits
    assert lb.lola_full_state_bytes(cfg(batch=64, capacity=1 << 20))[1][0] == 128 * (1 << 20) * 128
    for bad in (dict(batch=0), dict(n_q_heads=7), dict(n_kv_heads=0), dict(head_dim=96), dict(capacity=0), dict(capacity=100), dict(capacity=(1 << 26) + 64),
                dict(dtype=2), dict(out_dtype=-1), dict(tokens_first=2), dict(batch=40000)):
        assert lb.lola_full_state_bytes(cfg(**bad)) == (0, [0] * 8), bad


def test_workspace_bytes(L):
    c = cfg()
    assert lb.lola_full_workspace_bytes(c, 0) > 0
    assert lb.lola_full_workspace_bytes(c, 4096, True) >= lb.lola_full_workspace_bytes(c, 1, False)
    assert lb.lola_full_workspace_bytes(c, -1) == 0
    assert lb.lola_full_workspace_bytes(c, (1 << 22) + 1) == 0      # four query heads per kv head: more than 2^24 rows
    assert lb.lola_full_workspace_bytes(c, 1, 2) == 0
    assert lb.lola_full_workspace_bytes(cfg(head_dim=100), 1) == 0


def test_refusals_before_launch(L):
    """No GPU is present here: whatever reached a launch would come back as LOLA_ERR_HIP."""
    vp, fake, big = C.c_void_p, 0x1000, 1 << 40
    c, st = cfg(), lb.LolaFullState(*[fake] * 8)
    no_w = lb.LolaFullState(*[fake] * 5, None, fake, fake)
    app = lambda cc=c, s=st, k=fake, v=fake, lens=None, T=4: L.lola_full_append(C.byref(cc), C.byref(s), vp(k), vp(v), vp(lens), T, None)
    att = lambda cc=c, s=st, q=fake, lens=None, T=4, gather=0, out=fake, ws=fake, n=big: L.lola_full_attend(
        C.byref(cc), C.byref(s), vp(q), vp(lens), T, gather, vp(out), vp(ws), n, None)
    stp = lambda cc=c, s=st, q=fake, k=fake, v=fake, gather=0, out=fake, ws=fake, n=big: L.lola_full_step(
        C.byref(cc), C.byref(s), vp(q), vp(k), vp(v), gather, vp(out), vp(ws), n, None)
    evi = lambda cc=c, s=st, keep=64, first=0, recent=0, ws=fake, n=big: L.lola_full_evict(C.byref(cc), C.byref(s), keep, first, recent, vp(ws), n, None)
    for i in range(8):
        f = [fake] * 8
        f[i] = None
        s = lb.LolaFullState(*f)
        if i != 5:
            assert app(s=s) == att(s=s) == stp(s=s) == evi(s=s) == L.lola_full_init(C.byref(c), C.byref(s), None) == -1
        f[i] = fake + 8
        s = lb.LolaFullState(*f)
        assert app(s=s) == att(s=s) == stp(s=s) == evi(s=s) == -4
    assert L.lola_full_append(None, C.byref(st), vp(fake), vp(fake), None, 4, None) == -1
    assert L.lola_full_attend(C.byref(c), None, vp(fake), None, 4, 0, vp(fake), vp(fake), big, None) == -1
    assert app(k=None) == app(v=None) == att(q=None) == att(out=None) == stp(q=None) == stp(k=None) == stp(v=None) == stp(out=None) == -1
    assert att(s=no_w, gather=1) == stp(s=no_w, gather=1) == evi(s=no_w) == -1       # no weights to add to or to rank by
    assert app(k=fake + 2) == app(v=fake + 8) == app(lens=fake + 4) == att(q=fake + 8) == att(out=fake + 4) == att(lens=fake + 4) == att(ws=fake + 8) == -4
    assert stp(q=fake + 4) == stp(k=fake + 4) == stp(v=fake + 4) == stp(out=fake + 4) == stp(ws=fake + 1) == evi(ws=fake + 1) == -4
    assert app(T=-1) == att(T=-1) == att(gather=2) == stp(gather=-1) == app(T=(1 << 22) + 1) == att(T=(1 << 22) + 1) == -2
    assert evi(keep=-1) == evi(keep=257) == evi(first=-1) == evi(recent=-1) == evi(first=40, recent=25) == -2
    assert evi(first=2 ** 31 - 1, recent=2 ** 31 - 1) == -2
    assert att(gather=1, ws=None, n=0) == att(gather=1, n=16) == evi(ws=None, n=0) == evi(n=64) == stp(gather=1, n=16) == -6
    for bad, rc in ((dict(head_dim=96), -2), (dict(capacity=100), -2), (dict(dtype=5), -3), (dict(out_dtype=9), -3), (dict(tokens_first=3), -2)):
        cc = cfg(**bad)
        assert app(cc) == att(cc) == stp(cc) == evi(cc) == L.lola_full_init(C.byref(cc), C.byref(st), None) == rc
    # nothing to do: nothing is looked at
    assert app(k=None, v=None, T=0) == att(q=None, out=None, T=0, ws=None, n=0) == 0
    assert evi(keep=256, ws=None, n=0) == 0


def test_oracle_number_format():
    """The oracle's rounding is torch's conversion to float8_e4m3fn for every bf16 number up to 448, ties and subnormals among them."""
    bits = torch.arange(0, 1 << 16, dtype=torch.int32).to(torch.int16)
    x = bits.view(torch.bfloat16).float()
    x = x[x.abs() <= 448]
    assert np.array_equal(fo.e4m3(x.numpy()), x.to(torch.float8_e4m3fn).float().numpy().astype(np.float64))
    assert fo.exponent(448.0) == 0 and fo.exponent(448.0001) == 1 and fo.exponent(224.0) == -1 and fo.exponent(224.1) == 0
    assert fo.exponent(0.0) == -100 and fo.exponent(2.0 ** -140) == -100 and fo.exponent(3.4e38) == 120
