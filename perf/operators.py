"""Cases and plain forms of the attention and logits operators: rotary
positions, the paged 4-bit key/value cache, attention over it, and the log
probabilities read off the output head's logits.

`run` computes an operator in plain torch operations, or with `own` set calls
the library's entry point.  A case is a dict of plain values; its `op` names
the operator:
  rope      rows of heads rotated by their positions
  append    new tokens' keys rotated and stored with their values in the
            4-bit cache, their queries rotated, and the stored rows read back
  attn      attention of new tokens over the paged 4-bit cache
  logprobs  log probability of given tokens, entropy and top alternatives

Definitions.  Rotation and angles in 64 bits, one rounding to binary32.  The
cache holds 4-bit blocks of 32 (Q4_0 with an fp16 scale, or Q4_SYM with an
fp32 scale); the query of an attention row is quantized to 8 bits per 32 the
same way the library's products take their activations (Q8_0 or Q8_F32); the
key of position j is seen from position i when i - window < j <= i.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

PAGE = 64         # tokens of a cache page


# ------------------------------------------------------------------ cases
def listed():
    return [
        # the query heads of one decoded token: a call's latency
        dict(name="rope_1", op="rope", T=1, NH=16, D=256, n_rot=64, layout="half", scaling="none"),
        # the query heads of a long prompt, whole heads rotated in neighbouring
        # pairs, frequencies scaled by parts for eight times the trained length
        dict(name="rope_prompt5120", op="rope", T=5120, NH=32, D=128, n_rot=128,
             layout="interleaved", scaling="parts"),
        # a decode batch: one new token for each of 32 requests
        dict(name="append_batch32", op="append", B=32, L=4000, q=1, NH=16, NKV=2, D=256, n_rot=64,
             layout="half", scaling="none", fmt="q4_0"),
        # prompts of up to 947 tokens stored at once, fp32-scale format
        dict(name="append_prompt947", op="append", B=5, L=947, q=947, NH=32, NKV=8, D=128,
             n_rot=128, layout="half", scaling="linear", fmt="q4_sym"),
        # one decoded token after the 947-token prompt: latency
        dict(name="attn_decode_1x948", op="attn", B=1, L=948, q=1, NH=16, NKV=2, D=256, window=0,
             fmt="q4_0"),
        # one request with a long context: the cache split over the whole card
        dict(name="attn_decode_1x131072", op="attn", B=1, L=131072, q=1, NH=16, NKV=2, D=256,
             window=0, fmt="q4_0"),
        # a ragged decode batch
        dict(name="attn_decode_48x6000", op="attn", B=48, L=6000, q=1, NH=32, NKV=8, D=128,
             window=0, fmt="q4_0"),
        # four drafted tokens a request verified over a sliding window, fp32 scales
        dict(name="attn_verify_16x3000", op="attn", B=16, L=3000, q=4, NH=16, NKV=4, D=64,
             window=1024, fmt="q4_sym"),
        # the 947-token prompt attending to itself
        dict(name="attn_prompt_947", op="attn", B=1, L=947, q=947, NH=16, NKV=2, D=256, window=0,
             fmt="q4_0"),
        # the last 2048 tokens of two long prompts taken in pieces
        dict(name="attn_chunk_2x2048", op="attn", B=2, L=8192, q=2048, NH=32, NKV=8, D=128,
             window=0, fmt="q4_0"),
        # the sampled token of one decode step and 20 alternatives
        dict(name="logprobs_1", op="logprobs", T=1, V=151936, top=20, banned=0.0),
        # the 947-token prompt scored, some tokens banned
        dict(name="logprobs_947", op="logprobs", T=947, V=151936, top=5, banned=0.1),
    ]


def _log_int(rng, lo, hi):
    """An integer of [lo, hi], spread evenly over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


_HEADS = [(16, 2, 256), (32, 8, 128), (16, 4, 64), (8, 8, 128), (24, 2, 128), (64, 4, 128), (8, 1, 256)]


def draw(rng):
    op = rng.choice(["rope", "append", "attn", "attn", "attn", "logprobs"])
    NH, NKV, D = rng.choice(_HEADS)
    rot = dict(n_rot=rng.choice([D, D // 2, D // 4, D - 6]), layout=rng.choice(["half", "interleaved"]),
               scaling=rng.choice(["none", "linear", "parts"]))
    if op == "rope":
        return dict(op=op, T=_log_int(rng, 1, 4000), NH=NH, D=D, **rot)
    if op == "append":
        q = rng.choice([1, 1, _log_int(rng, 2, 900)])
        return dict(op=op, B=_log_int(rng, 1, 64 if q < 8 else 4), L=max(q, _log_int(rng, 1, 8000)),
                    q=q, NH=NH, NKV=NKV, D=D, fmt=rng.choice(["q4_0", "q4_sym"]), **rot)
    if op == "attn":
        q = rng.choice([1, 1, 1, rng.randint(2, 8), _log_int(rng, 9, 1500)])
        L = max(q, _log_int(rng, 1, 30000 if q == 1 else 6000))
        # at most 2^27 values of K, and of scores, in the plain form
        B = _log_int(rng, 1, 64)
        B = max(1, min(B, (1 << 27) // (L * NKV * D), (1 << 27) // (L * q * NH)))
        return dict(op=op, B=B, L=L, q=q, NH=NH, NKV=NKV, D=D, window=rng.choice([0, 0, 0, 128, 1000]),
                    fmt=rng.choice(["q4_0", "q4_0", "q4_sym"]))
    return dict(op=op, T=_log_int(rng, 1, 600), V=rng.randint(30000, 152000), top=rng.choice([0, 1, 5, 20, 32]),
                banned=rng.choice([0.0, 0.0, 0.5]))


def _lengths(c):
    """Tokens of each sequence, the new ones among them: the first has L, the
    others are spread over the upper four fifths."""
    f = (np.arange(c["B"]) * 0.6180339887) % 1.0
    n = np.maximum(1, np.round(c["L"] * (1.0 - 0.8 * f))).astype(np.int64)
    return n, np.minimum(n, c["q"])


# ------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _tile_bytes(c):
    nb = c["D"] // 32
    return nb * 1024 + nb * PAGE * (4 if c["fmt"] == "q4_sym" else 2)


def _cache(g, c):
    """A cache as earlier tokens left it: pages in any order of the pool, codes
    of all values, scales near those of N(0, 1) rows."""
    n, q = _lengths(c)
    per = -(-n // PAGE)
    cap = int(per.max()) + 1
    n_pages = int(per.sum()) + 3
    order = torch.randperm(n_pages, device="cuda", generator=g).to(torch.int32)
    first = torch.as_tensor(np.concatenate([[0], np.cumsum(per)[:-1]]), device="cuda")
    per_d = torch.as_tensor(per, device="cuda")
    at = torch.arange(cap, device="cuda")
    index = (first[:, None] + at[None, :]).clamp_(max=n_pages - 1)
    table = torch.where(at[None, :] < per_d[:, None], order[index], torch.full_like(order[index], -1))
    sym, nb = c["fmt"] == "q4_sym", c["D"] // 32

    def pool(is_k):
        rows = n_pages * c["NKV"]
        codes = torch.randint(0, 256, (rows, nb * 1024), dtype=torch.uint8, device="cuda", generator=g)
        if sym:   # the codes -7..7 only: the nibble of -8 becomes that of 0
            bad, zero = (8, 0) if is_k else (0, 8)
            lo, hi = codes & 15, codes >> 4
            codes = torch.where(lo == bad, zero, lo) | (torch.where(hi == bad, zero, hi) << 4)
        d = (2.0 + 0.8 * torch.rand(rows, nb * PAGE, device="cuda", generator=g)) / (7.0 if sym else 8.0)
        d = d * torch.where(torch.rand(rows, nb * PAGE, device="cuda", generator=g) < 0.5, -1.0, 1.0)
        d = d if sym else d.to(torch.float16)
        return torch.cat([codes, d.contiguous().view(torch.uint8)], 1).reshape(n_pages, c["NKV"], -1).contiguous()

    cu = np.concatenate([[0], np.cumsum(q)]).astype(np.int32)
    i32 = lambda a: torch.as_tensor(np.asarray(a, np.int32), device="cuda")
    pos = np.concatenate([np.arange(a - b, a) for a, b in zip(n, q)])
    return dict(k_pool=pool(True), v_pool=pool(False), table=table.to(torch.int32).contiguous(),
                kv_len=i32(n), cu=i32(cu), pos=i32(pos), T=int(cu[-1]),
                seq=i32(np.repeat(np.arange(c["B"]), q)).long(),
                row=i32(np.concatenate([np.arange(b) for b in q])).long(), qmax=int(q.max()))


def prepare(case, seed):
    g, c = _gen(seed), case
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)
    if c["op"] == "rope":
        # positions of a continued request: far ones where the scaling is for them
        far = 1 if c["scaling"] == "none" else 8
        start = int(torch.randint(0, 4096 * far, (1,), device="cuda", generator=g))
        pos = start + torch.arange(c["T"], device="cuda", dtype=torch.int32)
        return dict(case=c, x=r(c["T"], c["NH"], c["D"]), pos=pos.to(torch.int32),
                    out=torch.empty(c["T"], c["NH"], c["D"], device="cuda"))
    if c["op"] == "append":
        s = _cache(g, c)
        # one projection's rows hold q, k and v side by side
        qkv = r(s["T"], c["NH"] + 2 * c["NKV"], c["D"])
        s.update(case=c, q=qkv[:, :c["NH"]], k=qkv[:, c["NH"]:c["NH"] + c["NKV"]],
                 v=qkv[:, c["NH"] + c["NKV"]:], q_out=torch.empty(s["T"], c["NH"], c["D"], device="cuda"),
                 k_out=torch.empty(s["T"], c["NKV"], c["D"], device="cuda"),
                 v_out=torch.empty(s["T"], c["NKV"], c["D"], device="cuda"))
        return s
    if c["op"] == "attn":
        s = _cache(g, c)
        # scores of a spread of about two: some keys matter, most little
        s.update(case=c, q=2.0 * r(s["T"], c["NH"], c["D"]), out=torch.empty(s["T"], c["NH"], c["D"], device="cuda"),
                 lse=torch.empty(s["T"], c["NH"], device="cuda"))
        return s
    T, V = c["T"], c["V"]
    logits = 2.5 * r(T, V)
    if c["banned"]:
        off = torch.rand(T, V, device="cuda", generator=g) < c["banned"]
        logits = logits.masked_fill_(off, -math.inf)
    best = logits.argmax(1)
    # confident rows among the others, whose log probabilities are near zero
    logits[torch.arange(T, device="cuda"), best] += 12.0 * torch.rand(T, device="cuda", generator=g)
    target = torch.randint(0, V, (T,), device="cuda", generator=g)
    target = torch.where(torch.rand(T, device="cuda", generator=g) < 0.6, best, target)
    return dict(case=c, logits=logits, target=target.to(torch.int32))


# ------------------------------------------------------------------ plain forms
def _scaling(c):
    """Base, kind, factor and trained length of a case's frequencies."""
    return dict(base=10000.0 if c["scaling"] == "none" else 500000.0, kind=c["scaling"],
                factor=1.0 if c["scaling"] == "none" else 8.0, orig_len=4096)


def _frequencies(c):
    n, s = c["n_rot"], _scaling(c)
    i = torch.arange(n // 2, device="cuda", dtype=torch.float64)
    f = torch.pow(torch.tensor(s["base"], dtype=torch.float64, device="cuda"), -2.0 * i / n)
    if s["kind"] == "linear":
        return f / s["factor"]
    if s["kind"] == "parts":
        at = lambda turns: n * math.log(s["orig_len"] / (turns * 2 * math.pi)) / (2 * math.log(s["base"]))
        lo, hi = max(0, math.floor(at(32.0))), min(n - 1, math.ceil(at(1.0)))
        ramp = ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        return f * (1 - ramp) + f / s["factor"] * ramp
    return f


def _mscale(c):
    return 1.0 if c["scaling"] != "parts" else float(np.float32(1.0 + 0.1 * math.log(8.0)))


def _rotate(x, pos, f, c):
    """Heads rotated in 64 bits, rounded once."""
    n, ms = c["n_rot"], _mscale(c)
    a = pos.double()[:, None, None] * f
    cos, sin = torch.cos(a) * ms, torch.sin(a) * ms
    h = x[..., :n].double()
    if c["layout"] == "half":
        u, w = h[..., :n // 2], h[..., n // 2:]
        y = torch.cat([u * cos - w * sin, w * cos + u * sin], -1)
    else:
        u, w = h[..., 0::2], h[..., 1::2]
        y = torch.stack([u * cos - w * sin, w * cos + u * sin], -1).flatten(-2)
    return torch.cat([y.float(), x[..., n:]], -1)


def _round_away(v):
    r = torch.trunc(v)
    return torch.where((v - r).abs() >= 0.5, r + torch.sign(v), r)


def _q4(x, fmt):
    """4-bit rows: the values they stand for."""
    b = x.reshape(*x.shape[:-1], -1, 32)
    if fmt == "q4_0":
        m = torch.gather(b, -1, b.abs().argmax(-1, keepdim=True))
        d = (m * -0.125).to(torch.float16).float()
        inv = torch.where(d == 0, torch.zeros_like(d), 1.0 / d)
        q = torch.floor(b * inv + 8.5).clamp(0, 15) - 8.0
    else:
        d = b.abs().amax(-1, keepdim=True) / 7.0
        inv = torch.where(d == 0, torch.zeros_like(d), 1.0 / d)
        q = _round_away(b * inv).clamp(-7, 7)
    return (q * d).reshape(x.shape)


def _q8(x, fmt):
    """8-bit rows: the values they stand for."""
    b = x.reshape(*x.shape[:-1], -1, 32)
    d = b.abs().amax(-1, keepdim=True) / 127.0
    d = d.to(torch.float16).float() if fmt == "q4_0" else d
    inv = torch.where(d == 0, torch.zeros_like(d), 1.0 / d)
    return (_round_away(b * inv).clamp(-127, 127) * d).reshape(x.shape)


def _tiles(pool, table, c):
    """Codes [.., NB, 1024] and scales [.., NB, 64 tokens] of each sequence's
    pages (absent ones read as page 0)."""
    nb = c["D"] // 32
    t = pool[table.long().clamp(min=0)]                         # [B, P, NKV, bytes]
    codes = t[..., :nb * 1024].reshape(*t.shape[:3], nb, 1024)
    d = t[..., nb * 1024:].contiguous().view(torch.float32 if c["fmt"] == "q4_sym" else torch.float16).float()
    d = d.reshape(*t.shape[:3], nb, 4, 4, 4).transpose(-3, -2)  # [.., token / 16, token % 16 / 4, token % 4]
    return codes, d.reshape(*t.shape[:3], nb, PAGE)


def _keys(pool, table, c):
    """[B, NKV, P * 64, D] values of a key pool's pages."""
    codes, d = _tiles(pool, table, c)
    B, P, H, nb = codes.shape[:4]
    x = codes.reshape(B, P, H, nb, 4, 16, 4, 4)                 # dword, token % 16, token / 16, byte
    x = x.permute(0, 1, 2, 3, 6, 5, 4, 7).reshape(B, P, H, nb, PAGE, 16)
    x = torch.cat([x & 15, x >> 4], -1).float()
    x = torch.where(x > 7, x - 16, x) * d[..., None]            # two's complement nibbles
    return x.permute(0, 2, 1, 4, 3, 5).reshape(B, H, P * PAGE, nb * 32)


def _values(pool, table, c):
    codes, d = _tiles(pool, table, c)
    B, P, H, nb = codes.shape[:4]
    x = codes.reshape(B, P, H, nb, 4, 16, 4, 2, 2)              # token % 16 / 4, byte, token / 16, token % 2, token % 4 / 2
    x = x.permute(0, 1, 2, 3, 6, 4, 8, 7, 5)
    x = x.reshape(B, P, H, nb, PAGE, 16)
    x = (torch.cat([x & 15, x >> 4], -1).float() - 8.0) * d[..., None]
    return x.permute(0, 2, 1, 4, 3, 5).reshape(B, H, P * PAGE, nb * 32)


def _attend(s):
    c = s["case"]
    B, NH, NKV, D, fmt = s["kv_len"].numel(), c["NH"], c["NKV"], c["D"], c["fmt"]
    G, Q = NH // NKV, s["qmax"]
    k, v = _keys(s["k_pool"], s["table"], c), _values(s["v_pool"], s["table"], c)
    L = k.shape[2]
    q = torch.zeros(B, Q, NH, D, device="cuda")
    q[s["seq"], s["row"]] = _q8(s["q"], fmt)
    q = q.reshape(B, Q, NKV, G, D).permute(0, 2, 3, 1, 4).reshape(B, NKV, G * Q, D)
    sc = torch.matmul(q, k.transpose(2, 3)) * (D ** -0.5)
    at = torch.zeros(B, Q, dtype=torch.long, device="cuda")
    at[s["seq"], s["row"]] = s["pos"].long()
    j = torch.arange(L, device="cuda")
    seen = j <= at[..., None]
    if c["window"]:
        seen = seen & (j > at[..., None] - c["window"])
    sc = sc.reshape(B, NKV, G, Q, L).masked_fill_(~seen[:, None, None], -math.inf)
    m = sc.amax(-1, keepdim=True)
    p = torch.exp(sc.sub_(m))
    z = p.sum(-1, keepdim=True)
    o = torch.matmul(p.reshape(B, NKV, G * Q, L), v).reshape(B, NKV, G, Q, D) / z
    rows = lambda t: t.permute(0, 3, 1, 2, 4).reshape(B, Q, NH, -1)[s["seq"], s["row"]]
    return [rows(o), rows(m + torch.log(z))[..., 0]]


def _logprobs(s):
    x, t, n = s["logits"], s["target"].long(), s["case"]["top"]
    m = x.amax(1, keepdim=True)
    d = x - m
    e = torch.exp(d)
    # 64-bit sums: a confident row's log probability is the logarithm of a sum just above one
    z = e.sum(1, dtype=torch.float64)
    w = torch.where(e > 0, e * d, torch.zeros_like(e)).sum(1, dtype=torch.float64)
    logz = torch.log(z)
    lp = d.gather(1, t[:, None])[:, 0].double() - logz
    out = [lp.float(), (logz - w / z).float()]
    if n:
        v, i = torch.sort(x, dim=1, descending=True, stable=True)
        out += [i[:, :n].to(torch.int32), ((v[:, :n] - m).double() - logz[:, None]).float()]
    return out


# ------------------------------------------------------------------ one pass
def run(state):
    s, c = state, state["case"]
    if own:
        return _own(s, c)
    if c["op"] == "rope":
        if "f" not in s:      # made once, when a program loads its model
            s["f"] = _frequencies(c)
        return [_rotate(s["x"], s["pos"], s["f"], c)]
    if c["op"] == "append":
        if "f" not in s:
            s["f"] = _frequencies(c)
        k = _rotate(s["k"], s["pos"], s["f"], c)
        return [_rotate(s["q"], s["pos"], s["f"], c), _q4(k, c["fmt"]), _q4(s["v"], c["fmt"])]
    if c["op"] == "attn":
        return _attend(s)
    return _logprobs(s)


def _own(s, c):
    import paper_2606_24031_amd as w4
    if c["op"] in ("rope", "append") and "f" not in s:
        s["f"] = w4.rope_frequencies(c["n_rot"], **_scaling(c))
    if c["op"] in ("append", "attn") and "kv" not in s:
        s["kv"] = w4.KVCache(s["k_pool"], s["v_pool"], s["table"], s["kv_len"], s["cu"], c["D"],
                             c["fmt"])
    if c["op"] == "rope":
        return [w4.rope_rotate(s["x"], s["pos"], s["f"], layout=c["layout"], mscale=_mscale(c),
                               out=s["out"])]
    if c["op"] == "append":
        w4.kv_append(s["kv"], s["k"], s["v"], pos=s["pos"], inv_freq=s["f"], layout=c["layout"],
                     mscale=_mscale(c), q=s["q"], q_out=s["q_out"])
        return [s["q_out"], *w4.kv_read(s["kv"], s["T"], k_out=s["k_out"], v_out=s["v_out"])]
    if c["op"] == "attn":
        if "ws" not in s:
            s["ws"] = w4.attn_workspace(s["kv"], s["T"], c["NH"])
        return list(w4.attn_forward(s["kv"], s["q"], c["D"] ** -0.5, window=c["window"], out=s["out"],
                                    lse=s["lse"], workspace=s["ws"]))
    if "ws" not in s:
        s["ws"] = w4.logprobs_workspace(c["T"], c["V"], c["top"])
    r = w4.token_logprobs(s["logits"], s["target"], n_top=c["top"], workspace=s["ws"])
    return list(r) if c["top"] else list(r[:2])


# ------------------------------------------------------------------ cost
def work(case):
    c = case
    if c["op"] == "rope":
        n = c["T"] * c["NH"] * c["D"]
        return dict(bytes=8 * n + 4 * c["T"], flops=3 * c["T"] * c["NH"] * c["n_rot"])
    if c["op"] == "logprobs":
        return dict(bytes=4 * c["T"] * c["V"] + c["T"] * (12 + 8 * c["top"]), flops=5 * c["T"] * c["V"])
    n, q = _lengths(c)
    T = int(q.sum())
    block = 20 if c["fmt"] == "q4_sym" else 18
    if c["op"] == "append":
        # q in and out, k and v in, their blocks written, read back and returned
        kv = 2 * T * c["NKV"] * c["D"]
        return dict(bytes=8 * T * c["NH"] * c["D"] + 8 * kv + 2 * kv // 32 * block,
                    flops=3 * T * (c["NH"] + c["NKV"]) * c["n_rot"] + 4 * kv)
    keys = pairs = 0
    for a, b in zip(n.tolist(), q.tolist()):
        w = c["window"] or a
        at = np.arange(a - b, a)
        pairs += int(np.minimum(at + 1, w).sum())
        keys += a - max(0, a - b + 1 - w)
    return dict(bytes=2 * keys * c["NKV"] * c["D"] // 32 * block + 8 * T * c["NH"] * c["D"] + 4 * T * c["NH"],
                flops=4 * pairs * c["NH"] * c["D"])


# ------------------------------------------------------------------ 64 bits
def _angles(c, pos):
    """Rotation factors from the definition, on the host in 64 bits."""
    n, s = c["n_rot"], _scaling(c)
    f = [s["base"] ** (-2.0 * i / n) for i in range(n // 2)]
    if s["kind"] == "linear":
        f = [a / s["factor"] for a in f]
    if s["kind"] == "parts":
        pair = lambda turns: n / 2 * math.log(s["orig_len"] / (2 * math.pi * turns), s["base"])
        lo, hi = max(0, math.floor(pair(32))), min(n - 1, math.ceil(pair(1)))
        for i in range(n // 2):
            mix = min(1.0, max(0.0, (i - lo) / max(hi - lo, 0.001)))
            f[i] = f[i] * (1 - mix) + f[i] * mix / s["factor"]
    a = np.asarray(pos.cpu(), np.float64)[:, None] * np.asarray(f)[None, :]
    ms = _mscale(c)
    to = lambda v: torch.as_tensor(v * ms, device="cuda")[:, None, :]
    return to(np.cos(a)), to(np.sin(a))


def _rotated64(x, cs, c):
    n = c["n_rot"]
    y = x.double().clone()
    a = slice(0, n // 2) if c["layout"] == "half" else slice(0, n, 2)
    b = slice(n // 2, n) if c["layout"] == "half" else slice(1, n, 2)
    xa, xb = x[..., a].double(), x[..., b].double()
    y[..., a] = xa * cs[0] - xb * cs[1]
    y[..., b] = xb * cs[0] + xa * cs[1]
    return y


def _blocks64(x, levels, half_scale, top):
    """Values of symmetric blocks of 32 with scale amax / levels."""
    b = x.float().unflatten(-1, (-1, 32))
    if top is not None:      # Q4_0: the signed largest value stands at -8
        i = b.abs().max(-1, keepdim=True).indices
        d = (b.gather(-1, i) / -8.0).half().float()
        code = torch.floor(torch.where(d != 0, b * (1.0 / d), torch.zeros_like(b)) + 8.5).clamp(0, 15) - 8
    else:
        d = b.abs().max(-1, keepdim=True).values / levels
        d = d.half().float() if half_scale else d
        u = torch.where(d != 0, b * (1.0 / d), torch.zeros_like(b))
        code = (torch.floor(u.abs().double() + 0.5) * torch.sign(u)).clamp(-levels, levels)
    return (code.double() * d.double()).flatten(-2)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "rope":
        return [_rotated64(s["x"], _angles(c, s["pos"]), c)]
    if c["op"] == "append":
        cs = _angles(c, s["pos"])
        q4 = lambda x: _blocks64(x, 7.0, False, 8 if c["fmt"] == "q4_0" else None)
        # the cache stores the binary32 rotated key's block
        return [_rotated64(s["q"], cs, c), q4(_rotated64(s["k"], cs, c)), q4(s["v"])]
    if c["op"] == "logprobs":
        lp, ent = [], []
        for r0 in range(0, c["T"], 64):
            x = s["logits"][r0:r0 + 64].double()
            t = s["target"][r0:r0 + 64].long()
            m, at = x.max(1, keepdim=True)
            e = torch.exp(x - m).scatter_(1, at, 0.0)
            z1 = e.sum(1)
            ln = torch.log1p(z1)
            lp.append((x - m).gather(1, t[:, None])[:, 0] - ln)
            ent.append(ln - torch.nan_to_num(e * (x - m), nan=0.0).sum(1) / (1 + z1))
        out = [torch.cat(lp), torch.cat(ent)]
        if not c["top"]:
            return out
        x = s["logits"]
        v = x.topk(c["top"], dim=1).values.double()
        m = v[:, :1]
        ln = torch.cat([torch.log1p(torch.exp(x[r0:r0 + 64].double() - m[r0:r0 + 64]).sum(1) - 1)
                        for r0 in range(0, c["T"], 64)])
        return out + [None, v - m - ln[:, None]]
    NH, NKV, D = c["NH"], c["NKV"], c["D"]
    n, q = _lengths(c)
    xq = _blocks64(s["q"], 127.0, c["fmt"] == "q4_0", None)
    out, lse, r0 = [], [], 0
    nb, wide = D // 32, c["fmt"] == "q4_sym"
    for b in range(c["B"]):
        tok = torch.arange(int(n[b]), device="cuda")
        page, t = s["table"][b, tok // PAGE].long(), tok % PAGE
        rows = torch.arange(r0, r0 + int(q[b]), device="cuda")
        at = s["pos"][rows].long()
        hide = tok[None, :] > at[:, None]
        if c["window"]:
            hide |= tok[None, :] <= at[:, None] - c["window"]
        o_b, l_b = [], []
        for h in range(NKV):
            def scale(pool):
                d = pool[:, h, nb * 1024:].contiguous().view(torch.float32 if wide else torch.float16)
                at_d = (t % 16 // 4) * 16 + t // 16 * 4 + t % 4
                return torch.stack([d[page, i * PAGE + at_d] for i in range(nb)], 1).double()
            el = torch.arange(16, device="cuda")
            kb = (el // 4)[None, :] * 256 + (t % 16 * 16 + t // 16 * 4)[:, None] + (el % 4)[None, :]
            vb = (t % 16 // 4 * 256 + t // 16 * 4 + torch.tensor([0, 2, 1, 3], device="cuda")[t % 4])[:, None] + 16 * el
            def codes(pool, where, signed):
                by = torch.stack([pool[page[:, None], h, i * 1024 + where] for i in range(nb)], 1).int()
                v = torch.cat([by & 15, by >> 4], -1)
                return ((v + 8) % 16 - 8 if signed else v - 8).double()
            K = (codes(s["k_pool"], kb, True) * scale(s["k_pool"])[..., None]).flatten(1)
            V = (codes(s["v_pool"], vb, False) * scale(s["v_pool"])[..., None]).flatten(1)
            for a in range(NH // NKV):
                sc = (xq[rows, h * (NH // NKV) + a] @ K.T) / math.sqrt(D)
                sc = sc.masked_fill(hide, -math.inf)
                l_b.append(torch.logsumexp(sc, 1))
                o_b.append(torch.exp(sc - l_b[-1][:, None]) @ V)
        out.append(torch.stack(o_b, 1))
        lse.append(torch.stack(l_b, 1))
        r0 += int(q[b])
    return [torch.cat(out), torch.cat(lse)]
