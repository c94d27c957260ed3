"""Softmax attention over the whole context, held in 8 bits: the layers that a converted model keeps as they were, and the
other way of spending less memory on a context.  Four calls of `LolaFullCache` (the binding of include/lola.h):

* `append` quantises new keys and values into the cache (e4m3 codes, one power-of-two scale for each block of 64 slots and kv head),
* `attend` is softmax attention of the newest tokens' queries over it, adding up on request what weight every cached pair received,
* `step` is both for one new token of every sequence, the generation step,
* `evict` cuts the cache to a number of pairs, those that received the most weight beside the first and the most recent ones.

The kinds of cases are what a program does with them: `step`; `prompt` (a new request: reset, append, attend); `chunk` (a long
prompt's next piece, or a further turn, on a cache that is already long); `turn` (new tokens, then back to the budget); `compress` (a
long prompt is appended and cut to a budget by the weights that its attention gathered).

The plain forms are torch products, sums and comparisons on the same buffers in 32 bits; `exact` follows the definition in 64.
"""
import math

import torch

own = False
DEV = "cuda:0"
BLOCK = 64
FIRST = 4      # slots of a sequence's first tokens that an eviction keeps

# Head shapes: Llama-3.1-8B and Llama-3.2-1B as in workloads.py, the 8B shape over 2 and 8 GPUs, the ungrouped 32-head shape of
# the paper's layer-latency table; below them generic ones (odd groups, the narrowest and the widest head)
HEADS = {"8b": (32, 8, 128), "1b": (32, 8, 64), "8b_tp2": (16, 4, 128), "8b_tp8": (4, 1, 128), "mha": (32, 32, 128),
         "g3": (6, 2, 64), "g5": (5, 1, 128), "g7": (14, 2, 128), "d32": (8, 4, 32), "d256": (8, 2, 256)}


def case(name, kind, heads, B, ctx, *, T=1, slack=0, dtype="bf16", out="f32", ragged=False, gather=False, tokens_first=False, gone=0, keep=0):
    """ctx: pairs that the cache holds before the call; T: new tokens per sequence; slack: room for further passes; gone: tokens
    evicted earlier; ragged: sequences of unequal lengths, padded to T."""
    Hq, Hkv, d = HEADS[heads]
    cap = -(-(ctx + T + slack) // BLOCK) * BLOCK
    c = {"kind": kind, "heads": heads, "Hq": Hq, "Hkv": Hkv, "d": d, "B": B, "ctx": ctx, "T": T, "cap": cap, "dtype": dtype, "out": out,
         "ragged": ragged, "gather": gather, "tokens_first": tokens_first, "gone": gone, "keep": keep}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one user of the 1B model, some way into a conversation: the smallest call, all latency
        case("step_1b_b1", "step", "1b", 1, 1500, slack=512),
        # batch-64 serving of the 8B model, conversations of all lengths up to 4096, outputs in bf16
        case("step_8b_b64", "step", "8b", 64, 4096, slack=192, out="bf16", ragged=True),
        # one context of 128 Ki tokens: a single sequence's long cache, split over the chip
        case("step_8b_128k", "step", "8b", 1, 131072, slack=512),
        # generation under a budget: every step adds its weights to those that the next eviction ranks by; tokens have been evicted
        case("step_8b_gather", "step", "8b", 16, 8191, slack=256, ragged=True, gather=True, gone=20000),
        # fp32 storage (the head shape of configuration 1), a prompt of 256
        case("prompt_f32", "prompt", "d32", 2, 0, T=257, dtype="f32"),
        # short chat prompts of odd and unequal lengths, padded, as the projections lay them out
        case("prompt_8b_short", "prompt", "8b", 8, 0, T=333, out="bf16", ragged=True, tokens_first=True),
        # four 4096-token prompts on the 8B model (configuration 3's shape): the largest products
        case("prompt_8b_4k", "prompt", "8b", 4, 0, T=4096, out="bf16"),
        # a 2000-token prompt of the 1B model whose attention also gathers the weights that an eviction needs
        case("prompt_1b_gather", "prompt", "1b", 2, 0, T=2000, gather=True),
        # the next 512 tokens of a long prompt on the 8B shape: few rows, many keys
        case("chunk_8b_32k", "chunk", "8b", 1, 32768, T=512, slack=2048, out="bf16"),
        # a budget of 2048 pairs per sequence kept over a further turn of 64 tokens, 16 conversations
        case("turn_8b_b16", "turn", "8b", 16, 2048, T=64, slack=64, keep=2048, gone=5000),
        # 128 sequences of the 1B shape that fall back to their budget after every 16 tokens, odd budget
        case("turn_1b_b128", "turn", "1b", 128, 1111, T=16, slack=64, keep=1111, gone=300),
        # a long prompt of each of four sequences cut to a sixteenth
        case("compress_8b_32k", "compress", "8b", 4, 0, T=32768, keep=2048),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("step", "step", "prompt", "prompt", "chunk", "turn", "compress"))
    heads = rng.choice(tuple(HEADS))
    Hq, Hkv, d = HEADS[heads]
    kw = dict(dtype="f32" if rng.random() < 0.2 else "bf16", out=rng.choice(("f32", "bf16")), ragged=rng.random() < 0.5, tokens_first=rng.random() < 0.5)
    pairs = 64 * 8 * 2048 * 128 // (Hkv * d)       # of one call: no more codes than the largest listed step
    if kind == "step":
        ctx = _log_int(rng, 1, 65536)
        return case(None, kind, heads, _log_int(rng, 1, max(1, min(128, pairs // (ctx + 512)))), ctx, slack=512, gather=rng.random() < 0.3,
                    gone=rng.choice((0, 0, 777)), **kw)
    rows = 32 * 4096 * 4096 // Hq                  # rows x slots of one call: a quarter of the largest listed prompt
    if kind == "prompt":
        T = _log_int(rng, 2, 4096 if kw["dtype"] == "bf16" else 1024)
        return case(None, kind, heads, _log_int(rng, 1, max(1, min(32, rows // (T * T)))), 0, T=T, gather=rng.random() < 0.3, **kw)
    if kind == "chunk":
        T = _log_int(rng, 2, 512)
        ctx = _log_int(rng, 100, min(32768, rows // T))
        return case(None, kind, heads, _log_int(rng, 1, max(1, min(16, rows // (T * (ctx + 5 * T))))), ctx, T=T, slack=4 * T, gather=rng.random() < 0.2, **kw)
    if kind == "turn":
        keep = _log_int(rng, 70, 8192)
        T = _log_int(rng, 1, 512)
        return case(None, kind, heads, _log_int(rng, 1, max(1, min(128, pairs // (2 * keep + 2 * T)))), keep, T=T, slack=T, keep=keep, gone=rng.randrange(1, 5000), **kw)
    T = _log_int(rng, 200, 32768)
    return case(None, kind, heads, _log_int(rng, 1, max(1, min(32, pairs // (2 * T)))), 0, T=T, keep=max(40, T // rng.randrange(2, 20)), **kw)


def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _lengths(c, top, least=1):
    """Lengths of the B sequences, from the case alone: all `top`, or down to about half of it."""
    return [max(min(least, top), top - (b * 611) % (top // 2 + 1)) if c["ragged"] else top for b in range(c["B"])]


def _keys(g, c, n):
    """Keys as attention meets them: 16 directions that many tokens share, columns of unequal size."""
    S = c["B"] * c["Hkv"]
    centres = torch.randn((S, 16, c["d"]), generator=g, device=DEV)
    pick = torch.randint(0, 16, (S, n), generator=g, device=DEV)
    k = torch.randn((S, n, c["d"]), generator=g, device=DEV).mul_(0.6) + torch.gather(centres, 1, pick[..., None].expand(-1, -1, c["d"]))
    k *= torch.exp(0.5 * torch.randn((c["d"],), generator=g, device=DEV))
    return k.view(c["B"], c["Hkv"], n, c["d"])


def _pow2(e):
    """2^e in 32 bits, from the exponent's bits (e: whole numbers from -126 to 127)."""
    return ((e + 127).to(torch.int32) << 23).view(torch.float32)


def _fit(a):
    """Least whole e >= -100 with a <= 448 * 2^e."""
    m, x = torch.frexp(a)
    return torch.where(a > 0, x - torch.where(m <= 0.875, 9, 8), -100).clamp(min=-100)


def _blocks(x, d):
    return x.view(x.shape[0], x.shape[1], -1, BLOCK, d)


def _memory(g, c):
    """A cache with ctx pairs per sequence (fewer in a ragged batch), blocks quantised as they would be by one append."""
    B, Hkv, cap, d, dtype = c["B"], c["Hkv"], c["cap"], c["d"], _type(c["dtype"])
    i32 = dict(dtype=torch.int32, device=DEV)
    held = torch.tensor(_lengths(c, c["ctx"], 1) if c["ctx"] else [0] * B, **i32)[:, None].expand(B, Hkv).contiguous()
    used = torch.arange(cap, **i32) < held[..., None]
    mem = {}
    for name in ("k", "v"):
        if not c["ctx"]:
            codes, scale = torch.zeros((B, Hkv, cap, d), device=DEV), torch.zeros((B, Hkv, cap // BLOCK), device=DEV)
        else:
            x = _keys(g, c, cap) if name == "k" else torch.randn((B, Hkv, cap, d), generator=g, device=DEV)
            x = _blocks(x.to(dtype).float() * used[..., None], d)
            scale = _pow2(_fit(x.abs().amax((3, 4))))
            codes = (x / scale[..., None, None]).view(B, Hkv, cap, d)
        mem[name], mem[name + "_scale"] = codes.to(torch.float8_e4m3fn), scale
    slot = torch.arange(cap, **i32).expand(B, Hkv, cap)
    mem["idx"] = torch.where(used, torch.where(slot < FIRST, slot, slot + c["gone"]), -1).contiguous()
    mem["weight"] = torch.rand((B, Hkv, cap), generator=g, device=DEV).square_() * used
    mem["count"] = held
    mem["n_tokens"] = held.long() + c["gone"]
    return mem


def prepare(c, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    B, Hq, Hkv, d, T, dtype = c["B"], c["Hq"], c["Hkv"], c["d"], c["T"], _type(c["dtype"])
    lay = (lambda x: x.transpose(1, 2).contiguous()) if c["tokens_first"] else (lambda x: x.contiguous())
    st = {"case": c, "mem": _memory(g, c), "passes": 0}
    st["k"] = lay(_keys(g, c, T).to(dtype))
    st["v"] = lay(torch.randn((B, Hkv, T, d), generator=g, device=DEV).to(dtype))
    if c["kind"] in ("step", "prompt", "chunk"):
        st["q"] = lay(torch.randn((B, Hq, T, d), generator=g, device=DEV).mul_(1.2).to(dtype))
    if c["kind"] == "step":      # one token of every sequence has no token axis
        st.update({n: st[n].view(B, -1, d) for n in ("q", "k", "v")})
    st["lens"] = torch.tensor(_lengths(c, T), dtype=torch.int32, device=DEV) if c["ragged"] and T > 1 else None
    if c["kind"] == "compress":
        st["gathered"] = torch.rand((B, Hkv, c["cap"]), generator=g, device=DEV).square_()
    st["start"] = (st["mem"]["count"].clone(), st["mem"]["n_tokens"].clone())
    st["room"] = (c["cap"] - c["ctx"]) // T      # passes until the slots are used up
    return st


# ---- plain forms

def _held(count, cap):
    return torch.arange(cap, device=DEV) < count[..., None]


def _heads_first(c, x):
    return x.transpose(1, 2) if c["tokens_first"] else x


def _append(st, k, v, lens):
    """k, v [B, Hkv, T, d].  The blocks that receive tokens are a window of the cache; what it held of them is rescaled."""
    c, mem = st["case"], st["mem"]
    B, Hkv, T, d = k.shape
    cap, nblk = c["cap"], c["cap"] // BLOCK
    count = mem["count"].long()
    n = torch.minimum((T if lens is None else lens.long()[:, None]) + torch.zeros_like(count), cap - count)
    told = T if lens is None else lens.long()[:, None]
    w = min(nblk, (T + 2 * BLOCK - 2) // BLOCK)
    b0 = (count // BLOCK).clamp(max=nblk - w)
    blk = b0[..., None] + torch.arange(w, device=DEV)                                  # [B, Hkv, w]
    slot = (blk[..., None] * BLOCK + torch.arange(BLOCK, device=DEV)).view(B, Hkv, -1)    # [B, Hkv, w * 64]
    tok = slot - count[..., None]
    new = (tok >= 0) & (tok < n[..., None])
    old = tok < 0
    at = tok.clamp(0, T - 1)[..., None].expand(-1, -1, -1, d)
    k, v = torch.gather(k.float(), 2, at), torch.gather(v.float(), 2, at)
    bad = ~(torch.isfinite(k).all(-1, keepdim=True) & torch.isfinite(v).all(-1, keepdim=True))
    v = torch.where(torch.isfinite(v), v, 0.0)
    k = torch.where(bad, 0.0, k)
    for name, x, nan in (("k", k, bad), ("v", v, None)):
        codes, scale = mem[name].view(torch.uint8), mem[name + "_scale"]
        x = _blocks(torch.where(new[..., None], x, 0.0), d)
        got = new.view(B, Hkv, w, BLOCK).any(-1)
        e_old = (torch.gather(scale, 2, blk).view(torch.int32) >> 23) - 127
        e_new = _fit(x.abs().amax((3, 4)))
        e = torch.where(got, torch.where(blk * BLOCK < count[..., None], torch.maximum(e_old, e_new), e_new), e_old.clamp(min=-100))
        where = slot[..., None].expand(-1, -1, -1, d)
        was = _blocks(torch.gather(codes, 2, where), d)
        shrunk = was.contiguous().view(torch.float8_e4m3fn).float() * _pow2((e_old - e).clamp(-40, 0))[..., None, None]
        put = (x * _pow2(-e)[..., None, None]).view(B, Hkv, -1, d)
        if nan is not None:
            put = torch.where(nan, float("nan"), put)
        put = torch.where(new[..., None], put, torch.where(old[..., None], shrunk.view(B, Hkv, -1, d), 0.0)).to(torch.float8_e4m3fn).view(torch.uint8)
        put = torch.where((new | old)[..., None], put, was.reshape(B, Hkv, -1, d))
        codes.scatter_(2, where, put)
        scale.scatter_(2, blk, torch.where(got, _pow2(e), torch.gather(scale, 2, blk)))
    there = torch.gather(mem["idx"], 2, slot)
    mem["idx"].scatter_(2, slot, torch.where(new, (mem["n_tokens"][..., None] + tok).to(torch.int32), there))
    mem["weight"].scatter_(2, slot, torch.where(new, 0.0, torch.gather(mem["weight"], 2, slot)))
    mem["count"] += n.to(torch.int32)
    mem["n_tokens"] += told


def _attend(st, q, lens, gather):
    """q [B, Hq, T, d] -> out, the same shape."""
    c, mem = st["case"], st["mem"]
    B, Hq, T, d = q.shape
    Hkv, cap, g = c["Hkv"], c["cap"], c["Hq"] // c["Hkv"]
    K = (_blocks(mem["k"].float(), d) * mem["k_scale"][..., None, None]).view(B, Hkv, cap, d)
    V = (_blocks(mem["v"].float(), d) * mem["v_scale"][..., None, None]).view(B, Hkv, cap, d)
    held = _held(mem["count"], cap)                                                         # [B, Hkv, cap]
    n = T if lens is None else lens.long()[:, None, None]
    i = torch.arange(T, device=DEV)
    pos = mem["n_tokens"][..., None] - n + i                                                # [B, Hkv, T]
    seen = held[:, :, None] & (mem["idx"][:, :, None].long() <= pos[..., None]) & (i < n).expand(B, Hkv, T)[..., None]
    s = (q.float().reshape(B, Hkv, g * T, d) @ K.transpose(2, 3)).view(B, Hkv, g, T, cap) * (1.0 / math.sqrt(d))
    seen = seen[:, :, None]
    s = torch.where(seen, s, float("-inf"))
    top = s.amax(-1, keepdim=True)
    s = torch.exp(s - torch.where(torch.isinf(top), 0.0, top))
    total = s.sum(-1, keepdim=True)
    y = (s.view(B, Hkv, g * T, cap) @ V).view(B, Hkv, g, T, d)
    y = torch.where(total == 0, 0.0, y / total).view(B, Hq, T, d)
    if gather:
        mem["weight"] += torch.where(torch.isfinite(total) & (total > 0), s / total, 0.0).sum((2, 3))
    return y.to(_type(c["out"]))


def _evict(st, keep, first, recent):
    c, mem = st["case"], st["mem"]
    B, Hkv, cap, d = c["B"], c["Hkv"], c["cap"], c["d"]
    if keep >= cap:
        return
    count = mem["count"].long()
    held = _held(count, cap)
    over = (count > keep)[..., None]
    slot = torch.arange(cap, device=DEV).expand(B, Hkv, cap)
    stays = (mem["idx"] < first) | (mem["idx"].long() >= mem["n_tokens"][..., None] - recent)
    rank = torch.where(stays, float("inf"), mem["weight"])
    rank = torch.where(held, rank, float("-inf"))
    order = torch.sort(rank, dim=-1, descending=True, stable=True).indices
    kept = torch.zeros_like(held).scatter_(2, order[..., :keep], True) & held
    free, moves = ~kept & (slot < keep) & over, kept & (slot >= keep) & over
    most = min(keep, cap - keep)
    to = torch.sort((~free).to(torch.uint8), dim=-1, stable=True).indices[..., :most]
    src = torch.sort((~moves).to(torch.uint8), dim=-1, stable=True).indices[..., :most]
    real = torch.arange(most, device=DEV) < moves.sum(-1, keepdim=True)                 # [B, Hkv, most]
    blk = to // BLOCK
    for name in ("k", "v"):
        codes, scale = mem[name], mem[name + "_scale"]
        raw = codes.view(torch.uint8)
        moved = torch.gather(raw, 2, src[..., None].expand(-1, -1, -1, d)).view(torch.float8_e4m3fn).float()
        e_src = (torch.gather(scale, 2, src // BLOCK).view(torch.int32) >> 23) - 127
        size = torch.nan_to_num(moved, nan=0.0).abs().amax(-1) * _pow2(e_src.clamp(min=-126))
        need = torch.where(real, _fit(size), -126).to(torch.int32)
        e_old = (scale.view(torch.int32) >> 23) - 127
        e = e_old.clone().scatter_reduce_(2, blk, need, "amax")
        where = torch.where(real, to, keep)[..., None].expand(-1, -1, -1, d)           # (slot `keep` is free afterwards)
        put = (moved * _pow2((e_src - torch.gather(e, 2, blk)).clamp(-40, 40))[..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
        was = raw[:, :, keep].clone()
        alive = (slot < keep) & over
        shrunk = (_blocks(codes.float(), d) * _pow2((e_old - e).clamp(-40, 0))[..., None, None]).view(B, Hkv, cap, d).to(torch.float8_e4m3fn).view(torch.uint8)
        raw.copy_(torch.where(alive[..., None], shrunk, raw))
        raw.scatter_(2, where, put)
        raw[:, :, keep] = was
        scale.copy_(torch.where(e > e_old, _pow2(e.clamp(min=-126)), scale))
    where = torch.where(real, to, keep)
    for name in ("idx", "weight"):
        x = mem[name]
        was = x[:, :, keep].clone()
        x.scatter_(2, where, torch.gather(x, 2, src))
        x[:, :, keep] = was
    mem["count"].clamp_(max=keep)


# ---- one pass

def _cache(st):
    """The handle that a program keeps for its cache, around the buffers in hand."""
    if "cache" not in st:
        from paper_2505_23666_amd import binding as lb
        c = st["case"]
        st["cache"] = lb.LolaFullCache(c["B"], c["Hq"], c["Hkv"], c["d"], c["cap"], dtype=c["dtype"], out_dtype=c["out"], tokens_first=c["tokens_first"],
                                       buffers=st["mem"], device=DEV)
    return st["cache"]


def _restart(st):
    """A fork of the conversation: the cache's lengths as they were before the first pass."""
    st["mem"]["count"].copy_(st["start"][0])
    st["mem"]["n_tokens"].copy_(st["start"][1])


def run(st):
    c, mem = st["case"], st["mem"]
    kind, gather = c["kind"], c["gather"]
    q, k, v, lens = st.get("q"), st["k"], st["v"], st["lens"]
    if kind in ("step", "chunk"):
        if st["passes"] == st["room"]:
            _restart(st)
            st["passes"] = 0
        st["passes"] += 1
    out = None
    recent = max(1, c["keep"] // 8)
    if own:
        cache = _cache(st)
        if kind == "step":
            out = cache.step(q, k, v, gather=gather)
        else:
            if kind in ("prompt", "compress"):
                cache.reset()
            cache.append(k, v, lens)
            if kind in ("prompt", "chunk"):
                out = cache.attend(q, lens, gather=gather)
            else:
                if kind == "compress":
                    mem["weight"].copy_(st["gathered"])
                cache.evict(c["keep"], first=FIRST, recent=recent)
    else:
        if kind == "step":
            _append(st, k[:, :, None], v[:, :, None], None)
            out = _attend(st, q[:, :, None], None, gather)[:, :, 0]
        else:
            if kind in ("prompt", "compress"):
                mem["count"].zero_()
                mem["n_tokens"].zero_()
            _append(st, _heads_first(c, k), _heads_first(c, v), lens)
            if kind in ("prompt", "chunk"):
                out = _attend(st, _heads_first(c, q), lens, gather)
                out = out.transpose(1, 2).contiguous() if c["tokens_first"] else out
            else:
                if kind == "compress":
                    mem["weight"].copy_(st["gathered"])
                _evict(st, c["keep"], FIRST, recent)
    return {"memory": mem} if out is None else {"out": out, "memory": mem}


def work(c):
    """Inputs and what the queries see of the cache read once, outputs and new or moved pairs written once."""
    e, eo = (2 if c["dtype"] == "bf16" else 4), (2 if c["out"] == "bf16" else 4)
    B, Hq, Hkv, d, T, g = c["B"], c["Hq"], c["Hkv"], c["d"], c["T"], c["Hq"] // c["Hkv"]
    held = _lengths(c, c["ctx"], 1) if c["ctx"] else [0] * B
    news = _lengths(c, T) if T > 1 else [1] * B
    pair = 2 * d + 2 * 4 / BLOCK
    by = fl = 0.0
    for a, n in zip(held, news):
        by += Hkv * n * (2 * d * e + pair + 8)                                     # the append (and idx, weight of new slots)
        if c["kind"] in ("step", "prompt", "chunk"):
            by += Hkv * (a + n) * (pair + (8 if c["gather"] else 0)) + Hq * n * d * (e + eo)
            fl += Hkv * g * (n * a + n * (n + 1) / 2) * 2 * d * (3 if c["gather"] and n > 1 else 2)
        else:
            total = a + n
            out = max(0, total - c["keep"])
            moved = out * c["keep"] / total if total else 0                         # survivors behind the budget, if they lie anywhere
            moved = min(moved, n) if c["kind"] == "turn" else moved
            by += Hkv * (total * 8 + moved * 2 * (pair + 8)) * (out > 0)
            fl += Hkv * n * 2 * d
    return {"bytes": by, "flops": fl}


# ---- the definition in 64 bits, apart from the forms above: sequence by sequence, pairs as values

def _two(e):
    """2^e in 64 bits, from the exponent's bits (a power function may be off by a rounding)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _e4m3(x):
    """Nearest multiple of the e4m3 step at x (ties to even), for |x| <= 448; NaN stays."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -40)))
    e = torch.where(x.abs() >= _two(e + 1), e + 1, torch.where(x.abs() < _two(e), e - 1, e)).clamp(min=-6)
    step = _two(e - 3)
    return torch.round(x / step) * step


def _exponent(a):
    """Least whole e >= -100 with a <= 448 * 2^e, for one number."""
    e = -100
    if a > 0:
        e = max(-100, math.ceil(math.log2(a / 448.0)) - 1)
        while a > math.ldexp(448.0, e):
            e += 1
    return e


def exact(c, seed):
    st = prepare(c, seed)
    mem = st["mem"]
    B, Hq, Hkv, d, T, g, cap = c["B"], c["Hq"], c["Hkv"], c["d"], c["T"], c["Hq"] // c["Hkv"], c["cap"]
    if c["kind"] == "step":
        st.update({n: st[n][:, :, None] for n in ("q", "k", "v")})
        hf = lambda x: x  # noqa: E731
    else:
        hf = (lambda x: x.transpose(1, 2)) if c["tokens_first"] else (lambda x: x)
    kind, keep = c["kind"], c["keep"]
    code = {n: mem[n].double() for n in ("k", "v")}
    size = {n: mem[n + "_scale"].double() for n in ("k", "v")}
    weight, idx = mem["weight"].double(), mem["idx"].clone()
    count, told = mem["count"].tolist(), mem["n_tokens"].tolist()
    news = st["lens"].tolist() if st["lens"] is not None else [T] * B
    y = torch.zeros((B, Hq, T, d), dtype=torch.float64, device=DEV)
    for b in range(B):
        for h in range(Hkv):
            a, n = count[b][h], news[b]
            for name in ("k", "v"):
                x = hf(st[name])[b, h, :n].double()
                c1, s1 = code[name][b, h], size[name][b, h]
                top = torch.zeros((a // BLOCK + n // BLOCK + 2) * BLOCK, dtype=torch.float64, device=DEV)
                off = a % BLOCK
                top[off:off + n] = x.abs().amax(1)
                tops = top.view(-1, BLOCK).amax(1).tolist()
                es, parts = [], range(a // BLOCK, (a + n - 1) // BLOCK + 1)
                for p, J in enumerate(parts):
                    e = _exponent(tops[p])
                    if J * BLOCK < a:
                        e_old = round(math.log2(float(s1[J])))
                        if e > e_old:
                            c1[J * BLOCK:a] = _e4m3(c1[J * BLOCK:a] * 2.0 ** (e_old - e))
                        e = max(e, e_old)
                    es.append(e)
                e = torch.tensor(es, dtype=torch.float64, device=DEV)
                s1[parts.start:parts.stop] = _two(e)
                c1[a:a + n] = _e4m3(x * _two(-e).repeat_interleave(BLOCK)[off:off + n, None])
            idx[b, h, a:a + n] = torch.arange(n, dtype=torch.int32, device=DEV) + told[b][h]
            weight[b, h, a:a + n] = 0
            count[b][h], told[b][h] = a + n, told[b][h] + n
            a += n
            if kind in ("step", "prompt", "chunk"):
                value = {name: code[name][b, h, :a] * size[name][b, h].repeat_interleave(BLOCK)[:a, None] for name in ("k", "v")}
                for r in range(g):
                    s = hf(st["q"])[b, h * g + r, :n].double() @ value["k"].t() / math.sqrt(d)
                    if n > 1:
                        place = told[b][h] - n + torch.arange(n, device=DEV)
                        s.masked_fill_(idx[b, h, :a].long()[None] > place[:, None], float("-inf"))
                    p = torch.softmax(s, -1)
                    y[b, h * g + r, :n] = p @ value["v"]
                    if c["gather"]:
                        weight[b, h, :a] += p.sum(0)
            elif a > keep:
                if kind == "compress":
                    weight[b, h] = st["gathered"][b, h].double()
                w = weight[b, h, :a].clone()
                w[(idx[b, h, :a] < FIRST) | (idx[b, h, :a] >= told[b][h] - max(1, keep // 8))] = float("inf")
                best = torch.argsort(-w, stable=True)[:keep].sort().values
                moved = best[best >= keep]
                there = torch.ones(keep, dtype=torch.bool, device=DEV)
                there[best[best < keep]] = False
                holes = there.nonzero()[:, 0]
                for name in ("k", "v"):
                    c1, s1 = code[name][b, h], size[name][b, h]
                    x = c1[moved] * s1[moved // BLOCK][:, None]
                    full = torch.zeros(keep + BLOCK, dtype=torch.float64, device=DEV)
                    full[holes] = x.abs().amax(1)
                    tops = full[:(keep + BLOCK - 1) // BLOCK * BLOCK].view(-1, BLOCK).amax(1).tolist()
                    was = torch.log2(s1).round()
                    was = was.clamp(min=-1000).long()
                    now = was.tolist()
                    for J in set((holes // BLOCK).tolist()):
                        now[J] = max(now[J], _exponent(tops[J]))
                        if now[J] > was[J]:
                            end = min(J * BLOCK + BLOCK, keep)
                            c1[J * BLOCK:end] = _e4m3(c1[J * BLOCK:end] * 2.0 ** (float(was[J]) - now[J]))
                    now = _two(torch.tensor(now, device=DEV).clamp(min=-1000))
                    grown = torch.zeros_like(s1, dtype=torch.bool)
                    grown[holes // BLOCK] = True
                    s1.copy_(torch.where(grown, now, s1))
                    c1[holes] = _e4m3(x / s1[holes // BLOCK][:, None])
                for x in (weight[b, h], idx[b, h]):
                    x[holes] = x[moved]
                count[b][h] = keep
            if kind == "compress" and a <= keep:
                weight[b, h] = st["gathered"][b, h].double()
    if kind == "compress":
        weight[..., :] = torch.where(torch.arange(cap, device=DEV) < keep, weight, st["gathered"].double())
    if kind == "step":
        y = y[:, :, 0]
    elif c["tokens_first"]:
        y = y.transpose(1, 2).contiguous()
    memory = {"k": code["k"], "v": code["v"], "k_scale": size["k"], "v_scale": size["v"], "idx": idx, "weight": weight,
              "count": torch.tensor(count, dtype=torch.int32, device=DEV), "n_tokens": torch.tensor(told, device=DEV)}
    return {"out": y, "memory": memory} if kind in ("step", "prompt", "chunk") else {"memory": memory}
