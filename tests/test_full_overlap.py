"""Outputs that overlap a call's own inputs: refused before anything is launched, except the queries' own place where that is safe."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

from paper_2505_23666_amd import binding as lb

BASE = 0x100000


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(lb.LIB_PATH):
        from paper_2505_23666_amd import build
        build.build_library()
    return lb.lib()


@pytest.mark.parametrize("dtype,out_dtype", [(0, 0), (1, 1), (1, 0), (0, 1)])
def test_overlaps_are_refused(L, dtype, out_dtype):
    """No GPU is needed: whatever gets as far as a launch comes back as LOLA_ERR_HIP there, and is not called here with one."""
    vp, far, big = C.c_void_p, 0x40000000, 1 << 40
    c = lb.LolaFullConfig(2, 8, 2, 128, 256, dtype, out_dtype, 0, 0.0)
    st = lb.LolaFullState(*[far + i * 0x1000000 for i in range(8)])
    size = lambda heads, T, bf16: 2 * heads * T * 128 * (2 if bf16 else 4)  # noqa: E731
    att = lambda q, out, T, gather: L.lola_full_attend(C.byref(c), C.byref(st), vp(q), None, T, gather, vp(out), vp(16 * far), big, None)  # noqa: E731
    stp = lambda q, k, v, out, gather=0: L.lola_full_step(C.byref(c), C.byref(st), vp(q), vp(k), vp(v), gather, vp(out), vp(16 * far), big, None)  # noqa: E731
    for T in (1, 4, 100):
        nq, no = size(8, T, dtype), size(8, T, out_dtype)
        for gather in (0, 1):
            assert att(BASE, BASE + 16, T, gather) == att(BASE, BASE + nq - 16, T, gather) == att(BASE, BASE - no + 16, T, gather) == -5
            if (gather and T == 100) or dtype != out_dtype:
                assert att(BASE, BASE, T, gather) == -5
    nq, nk, no = size(8, 1, dtype), size(2, 1, dtype), size(8, 1, out_dtype)
    clear = 0x10000
    assert stp(BASE, BASE + clear, BASE + 2 * clear, BASE + 16) == stp(BASE, BASE + clear, BASE + 2 * clear, BASE + nq - 16) == -5
    assert stp(BASE, BASE + clear, BASE + 2 * clear, BASE + clear) == stp(BASE, BASE + clear, BASE + 2 * clear, BASE + clear + nk - 16) == -5
    assert stp(BASE, BASE + clear, BASE + 2 * clear, BASE + 2 * clear) == stp(BASE, BASE + clear, BASE + 2 * clear, BASE + 2 * clear - no + 16) == -5
    c.n_q_heads = 66      # 33 query heads per kv head: the kernels of many rows, also in a step
    assert att(BASE, BASE, 1, 1) == stp(BASE, BASE + 16 * clear, BASE + 32 * clear, BASE, 1) == -5


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_outputs_in_the_queries_place(dtype):
    """The outputs may take the queries' place: the same bits as beside them, in every kernel; with weights over many rows the call is refused."""
    dt, dev = (torch.bfloat16 if dtype == "bf16" else torch.float32), "cuda:0"
    rng = np.random.default_rng(1)
    x = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(dt).to(dev)  # noqa: E731
    for Hq, d, cap, held, T, tokens_first in ((4, 64, 192, 150, 1, False), (8, 128, 4096, 3000, 1, False), (20, 64, 2048, 900, 1, True), (4, 128, 2048, 1000, 4, True),
                                              (4, 64, 512, 0, 300, False), (8, 64, 4096, 2000, 70, True), (2, 256, 512, 0, 333, False)):
        c = lb.LolaFullCache(2, Hq, 2, d, cap, dtype=dtype, out_dtype=dtype, tokens_first=tokens_first, device=dev)
        lay = (lambda t: t.transpose(1, 2).contiguous()) if tokens_first else (lambda t: t)
        if held:
            c.append(lay(x(2, 2, held, d)), lay(x(2, 2, held, d)))
        q, k, v = lay(x(2, Hq, T, d)), lay(x(2, 2, T, d)), lay(x(2, 2, T, d))
        c.append(k, v)
        want = c.attend(q)
        place = q.clone()
        assert c.attend(place, out=place) is place
        assert torch.equal(place, want), (Hq, d, cap, held, T)
        if T * Hq // 2 > (16 if d == 256 else 32):
            with pytest.raises(lb.LolaError, match="no kernel"):
                c.attend(q, out=q, gather=True)
        else:
            c.weight.zero_()
            want, weight = c.attend(q, gather=True), c.weight.clone()
            c.weight.zero_()
            place = q.clone()
            c.attend(place, out=place, gather=True)
            n = held + T
            assert torch.equal(place, want) and torch.equal(c.weight[:, :, :n], weight[:, :, :n]), (Hq, d, cap, held, T)
    assert c.step(*(t[:, :, 0].contiguous() for t in (q, k, v))).shape == (2, 2, 256)
    q1, k1, v1 = (t[:, :, 0].contiguous() for t in (q, k, v))
    with pytest.raises(lb.LolaError):
        c.step(q1, k1, v1, out=k1)
