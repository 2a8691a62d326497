"""Cases and plain forms of the operators around a layer's recurrence: the
product in 8-bit integers with one scale a row on either side, the short causal
convolution, and the selective state space scan.

`run` computes an operator in plain torch operations, or with `own` set calls
the library's entry point.  A case is a dict of plain values; its `op` names
the operator:
  q8    fp32 rows quantized to 8 bits with a scale each, times a weight matrix
        of 8-bit rows with a scale each, plus a bias
  conv  the short causal convolution over the rows of several sequences, with
        their states of the last inputs
  ssm   the selective state space scan over the rows of several sequences,
        with their states

Definitions.  A row's scale is amax / 127 and its codes round(x * (1 / scale)),
half away from zero, every step one binary32 operation; sums of code products
are exact integers.  The state space layer of head h: with delta =
softplus(dt + dt_bias), S <- exp(delta A) S + delta B x^T, y = (C^T S + D x)
SiLU(z).  A sequence reads its state in one slot of a pool and leaves it in
another, as a program does that may take its last tokens back.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

KPAD = 128        # rows of codes end on a multiple of this many, zeros past K


# ------------------------------------------------------------------ cases
def listed():
    return [
        # the in-projection of one decoded token of a linear-attention layer
        # (32 heads of 128 for q, k and v): the weights streamed once
        dict(name="q8_1", op="q8", M=1, N=12288, K=2048, bias=False),
        # the out-projection of a decode batch
        dict(name="q8_48", op="q8", M=48, N=2048, K=4096, bias=False),
        # odd sizes: a short prompt, an odd number of channels, rows that end
        # inside every tile
        dict(name="q8_odd", op="q8", M=333, N=4099, K=1541, bias=True),
        # the in-projection of the 947-token prompt
        dict(name="q8_947", op="q8", M=947, N=12288, K=2048, bias=False),
        # a long prompt: the matrix cores' own rate
        dict(name="q8_5120", op="q8", M=5120, N=12288, K=4096, bias=True),
        # one new token for each of 32 requests, the state space layer's
        # channels (64 heads of 64, B and C of 128): a call's latency
        dict(name="conv_32x1", op="conv", B=32, q=1, CH=4352, W=4, bias=True, silu=True, fresh=0.0),
        # prompts of up to 2048 tokens, q, k and v of the linear-attention
        # layers, no bias; half of them begin here
        dict(name="conv_prompts", op="conv", B=4, q=2048, CH=12288, W=4, bias=False, silu=True, fresh=0.5),
        # one decoded token of one request: latency
        dict(name="ssm_1x1", op="ssm", B=1, q=1, NH=64, P=64, N=128, NG=1, gate=True, fresh=0.0),
        # a decode batch: the states read and written
        dict(name="ssm_48x1", op="ssm", B=48, q=1, NH=64, P=64, N=128, NG=1, gate=True, fresh=0.0),
        # the 947-token prompt at the linear-attention layer's 32 heads of 128
        dict(name="ssm_947", op="ssm", B=1, q=947, NH=32, P=128, N=128, NG=8, gate=False, fresh=1.0),
        # prompts of up to 2000 tokens together, some continued
        dict(name="ssm_6x2000", op="ssm", B=6, q=2000, NH=64, P=64, N=128, NG=1, gate=True, fresh=0.5),
        # one long prompt: few workgroups and many steps
        dict(name="ssm_1x16384", op="ssm", B=1, q=16384, NH=64, P=64, N=128, NG=1, gate=True, fresh=1.0),
    ]


def _log_int(rng, lo, hi):
    """An integer of [lo, hi], spread evenly over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["q8", "q8", "conv", "ssm", "ssm"])
    if op == "q8":
        bias = rng.random() < 0.5
        if rng.random() < 0.2:     # an output head
            return dict(op=op, M=_log_int(rng, 1, 64), N=rng.randint(32000, 152000), K=rng.choice([1024, 2048]),
                        bias=bias)
        M, K = _log_int(rng, 1, 6000), rng.choice([512, 1024, 2048, 4096, _log_int(rng, 33, 9000)])
        N = rng.choice([1024, 2048, 4096, 8192, _log_int(rng, 64, 16000)])
        return dict(op=op, M=M, N=N, K=K, bias=bias)
    if op == "conv":
        CH = 4 * _log_int(rng, 64, 4096)
        q = rng.choice([1, 1, rng.randint(2, 8), _log_int(rng, 9, 5000)])
        B = max(1, min(_log_int(rng, 1, 64), 60_000_000 // (CH * q)))
        return dict(op=op, B=B, q=q, CH=CH, W=rng.choice([2, 3, 4, 4, 4]), bias=rng.random() < 0.5,
                    silu=rng.random() < 0.8, fresh=rng.choice([0.0, 0.5, 1.0]))
    NH, P, N = rng.choice([(64, 64, 128), (32, 128, 128), (32, 64, 64), (24, 64, 128), (16, 128, 256), (8, 96, 64),
                           (80, 64, 128)])
    q = rng.choice([1, 1, rng.randint(2, 8), _log_int(rng, 9, 6000), _log_int(rng, 9, 6000)])
    B = max(1, min(_log_int(rng, 1, 64), 8_000_000_000 // (q * NH * P * N)))
    return dict(op=op, B=B, q=q, NH=NH, P=P, N=N, NG=rng.choice([1, 1, 2, 8]), gate=rng.random() < 0.7,
                fresh=rng.choice([0.0, 0.5, 1.0]))


def _lengths(c):
    """Rows of each sequence: the first has q, the others are spread over the
    upper four fifths."""
    f = (np.arange(c["B"]) * 0.6180339887) % 1.0
    return np.maximum(1, np.round(c["q"] * (1.0 - 0.8 * f))).astype(np.int64)


# ------------------------------------------------------------------ inputs
def _sequences(g, c):
    """The plan of a call: cu_rows, the slots that states come from (-1: none,
    the sequence begins here) and go to, in any order of the pool."""
    n, B = _lengths(c), c["B"]
    slots = torch.randperm(2 * B, device="cuda", generator=g).to(torch.int32)
    src, dst = slots[:B].clone(), slots[B:].clone()
    src[torch.rand(B, device="cuda", generator=g) < c["fresh"]] = -1
    cu = torch.as_tensor(np.concatenate([[0], np.cumsum(n)]).astype(np.int32), device="cuda")
    seq = torch.as_tensor(np.repeat(np.arange(B), n), device="cuda")
    row = torch.as_tensor(np.concatenate([np.arange(k) for k in n]), device="cuda")
    return dict(cu=cu, src=src, dst=dst, n_slots=2 * B, T=int(n.sum()), seq=seq, row=row,
                n=torch.as_tensor(n, device="cuda"))


def _codes(x):
    """8-bit codes (fp32 whole numbers) and scales of fp32 rows."""
    d = x.abs().amax(-1, keepdim=True) / 127.0
    inv = 1.0 / d
    inv = torch.where((d == 0) | torch.isinf(inv), torch.zeros_like(inv), inv)
    v = x * inv
    r = torch.trunc(v)
    r = torch.where((v - r).abs() >= 0.5, r + torch.sign(v), r)
    return r.clamp_(-127, 127), d[..., 0]


def prepare(case, seed):
    g, c = torch.Generator(device="cuda").manual_seed(seed), case
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)
    u = lambda *s: torch.rand(*s, device="cuda", generator=g)
    if c["op"] == "q8":
        M, N, K = c["M"], c["N"], c["K"]
        # activations with a few large channels, weights of a trained layer's size
        x = r(M, K) * torch.where(u(K) < 0.01, 12.0, 1.0)
        wq, wd = _codes(0.02 * r(N, K))
        w = torch.zeros(N, -(-K // KPAD) * KPAD, dtype=torch.int8, device="cuda")
        w[:, :K] = wq.to(torch.int8)
        return dict(case=c, x=x, w=w, wd=wd, bias=0.1 * r(N) if c["bias"] else None,
                    out=torch.empty(M, N, device="cuda"))
    s = _sequences(g, c)
    T = s["T"]
    if c["op"] == "conv":
        CH, W = c["CH"], c["W"]
        # the convolved channels stand in a projection's rows after a gate
        rows = r(T, CH + 256)
        s.update(case=c, x=rows[:, 256:], w=r(W, CH) / math.sqrt(W), bias=0.1 * r(CH) if c["bias"] else None,
                 state=r(s["n_slots"], W - 1, CH), out=torch.empty(T, CH, device="cuda"))
        return s
    NH, P, N, NG = c["NH"], c["P"], c["N"], c["NG"]
    # the convolution's rows: x, B and C side by side; the projection's: z and dt
    xbc = torch.nn.functional.silu(r(T, NH * P + 2 * NG * N))
    proj = r(T, NH * P + NH)
    # steps of 0.001 to 0.1 and decays of 1 to 16, as such layers begin with
    step = torch.exp(u(NH) * (math.log(0.1) - math.log(0.001)) + math.log(0.001))
    s.update(case=c, x=xbc[:, :NH * P].unflatten(1, (NH, P)), b=xbc[:, NH * P:NH * P + NG * N].unflatten(1, (NG, N)),
             c=xbc[:, NH * P + NG * N:].unflatten(1, (NG, N)),
             z=proj[:, :NH * P].unflatten(1, (NH, P)) if c["gate"] else None, dt=proj[:, NH * P:],
             dt_bias=step + torch.log(-torch.expm1(-step)), a=-(1.0 + 15.0 * u(NH)), d=1.0 + 0.1 * r(NH),
             state=0.1 * r(s["n_slots"], NH, N, P), out=torch.empty(T, NH, P, device="cuda"))
    return s


# ------------------------------------------------------------------ plain forms
def _silu(v):
    return v / (1.0 + torch.exp(-v))


def _product(s):
    c = s["case"]
    K, (xq, xd) = c["K"], _codes(s["x"])
    w = s["w"][:, :K]
    acc = torch.zeros(c["M"], c["N"], dtype=torch.int32, device="cuda")
    for k in range(0, K, 1024):      # sums of up to 1024 products of 127 * 127 are exact in 32-bit floats
        acc += torch.matmul(xq[:, k:k + 1024], w[:, k:k + 1024].float().t()).to(torch.int32)
    y = acc.float() * (xd[:, None] * s["wd"][None, :])
    return y if s["bias"] is None else y + s["bias"]


def _from_slots(s):
    """The states that the sequences begin with."""
    old = s["state"][s["src"].long().clamp(min=0)]
    return old.masked_fill((s["src"] < 0).reshape(-1, *[1] * (old.dim() - 1)), 0.0)


def _conv(s):
    c = s["case"]
    W, B, CH = c["W"], c["B"], c["CH"]
    hist = _from_slots(s)                                        # [B, W - 1, CH]
    ext = torch.cat([hist.reshape(B * (W - 1), CH), s["x"]])     # states, then the rows
    t = torch.arange(s["T"], device="cuda")
    y = torch.zeros(s["T"], CH, device="cuda")
    for i in range(W):
        back = W - 1 - i
        at = torch.where(s["row"] >= back, B * (W - 1) + t - back, s["seq"] * (W - 1) + W - 1 + s["row"] - back)
        y += s["w"][i] * ext[at]
    if s["bias"] is not None:
        y += s["bias"]
    last = s["cu"][1:].long()[:, None] - (W - 1) + torch.arange(W - 1, device="cuda")     # row numbers
    j = last - s["cu"][:-1].long()[:, None]                                               # within the sequence
    at = torch.where(j >= 0, B * (W - 1) + last, torch.arange(B, device="cuda")[:, None] * (W - 1) + W - 1 + j)
    s["state"][s["dst"].long()] = ext[at]
    return [_silu(y) if c["silu"] else y, s["state"]]


def _scan(s):
    c = s["case"]
    B, Q, NH, P, N, NG = c["B"], c["q"], c["NH"], c["P"], c["N"], c["NG"]
    v = s["dt"] + s["dt_bias"]
    delta = torch.clamp(v, min=0.0) + torch.log1p(torch.exp(-v.abs()))
    rows = lambda a: torch.zeros(B, Q, *a.shape[1:], device="cuda").index_put_((s["seq"], s["row"]), a)
    x, d, b, cc = rows(s["x"]), rows(delta), rows(s["b"]), rows(s["c"])
    decay, dx = torch.exp(d * s["a"]), d[..., None] * x           # rows past a sequence's end: 1 and 0
    S = _from_slots(s).clone()
    y = torch.empty(B, Q, NH, P, device="cuda")
    for t in range(Q):
        bt = b[:, t].repeat_interleave(NH // NG, 1)
        ct = cc[:, t].repeat_interleave(NH // NG, 1)
        S = S * decay[:, t, :, None, None] + bt[..., None] * dx[:, t, :, None, :]
        y[:, t] = torch.matmul(ct[:, :, None, :], S)[:, :, 0]
    y = y[s["seq"], s["row"]] + s["d"][:, None] * s["x"]
    if s["z"] is not None:
        y = y * _silu(s["z"])
    s["state"][s["dst"].long()] = S
    return [y, s["state"]]


# ------------------------------------------------------------------ one pass
def run(state):
    s, c = state, state["case"]
    if own:
        return _own(s, c)
    return [_product(s)] if c["op"] == "q8" else _conv(s) if c["op"] == "conv" else _scan(s)


def _own(s, c):
    import paper_2606_24031_amd as w4
    if c["op"] == "q8":
        xq, xd = w4.q8_row_quantize(s["x"])
        return [w4.q8q8_gemm(xq, xd, s["w"], s["wd"], bias=s["bias"], out=s["out"])]
    if "plan" not in s:
        s["plan"] = w4.SeqPlan(s["cu"], s["n_slots"], src=s["src"], dst=s["dst"])
    if c["op"] == "conv":
        return [w4.short_conv(s["plan"], s["x"], s["w"], s["state"], bias=s["bias"],
                              act="silu" if c["silu"] else "none", out=s["out"]), s["state"]]
    if "ws" not in s:
        s["ws"] = w4.ssm_workspace(s["plan"], s["T"], c["NH"], c["NG"], c["N"], c["P"])
    return [w4.ssm_scan(s["plan"], s["x"], s["dt"], s["a"], s["b"], s["c"], s["state"], D=s["d"], z=s["z"],
                        dt_bias=s["dt_bias"], softplus=True, out=s["out"], workspace=s["ws"]), s["state"]]


# ------------------------------------------------------------------ cost
def work(case):
    c = case
    if c["op"] == "q8":
        M, N, K = c["M"], c["N"], c["K"]
        return dict(bytes=4 * M * K + N * K + 4 * M * N + 4 * N * (2 if c["bias"] else 1), flops=2 * M * N * K)
    T, B = int(_lengths(c).sum()), c["B"]
    if c["op"] == "conv":
        return dict(bytes=4 * c["CH"] * (2 * T + 2 * B * (c["W"] - 1) + c["W"]), flops=2 * c["W"] * T * c["CH"])
    NH, P, N, NG = c["NH"], c["P"], c["N"], c["NG"]
    # states in (where there are any) and out, x, y, z, B, C and dt; of a token
    # and state element a decay, an update and a read
    state = 4 * NH * N * P * (B * (2 if c["fresh"] == 0.0 else 1))
    return dict(bytes=state + 4 * T * ((3 if c["gate"] else 2) * NH * P + 2 * NG * N + NH), flops=5 * T * NH * P * N)


# ------------------------------------------------------------------ 64 bits
def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "q8":
        x = s["x"]
        amax = x.abs().max(1).values
        d = amax / 127.0
        codes = torch.zeros_like(x, dtype=torch.float64)
        live = amax > 0
        scaled = (x * torch.where(live, 1.0 / d, d)[:, None]).double()      # the binary32 product decides the code
        codes[live] = (torch.floor(scaled.abs() + 0.5) * torch.sign(scaled))[live]
        y = codes.clamp(-127, 127) @ s["w"][:, :c["K"]].double().t().contiguous()
        y = y * d.double()[:, None] * s["wd"].double()[None, :]
        return [y if s["bias"] is None else y + s["bias"].double()]
    n, ends = _lengths(c).tolist(), s["cu"].tolist()
    src, dst, pool = s["src"].tolist(), s["dst"].tolist(), s["state"].double()
    new, out = pool.clone(), []
    if c["op"] == "conv":
        W, w = c["W"], s["w"].double()
        for i in range(c["B"]):
            old = pool[src[i]] if src[i] >= 0 else torch.zeros_like(pool[0])
            rows = torch.cat([old, s["x"][ends[i]:ends[i + 1]].double()])
            y = sum(rows[k:k + n[i]] * w[k] for k in range(W))
            y = y if s["bias"] is None else y + s["bias"].double()
            out.append(y * torch.sigmoid(y) if c["silu"] else y)
            new[dst[i]] = rows[n[i]:]
        return [torch.cat(out), new]
    G = c["NH"] // c["NG"]
    f = lambda k: s[k].double()
    A, D = f("a"), f("d")
    for i in range(c["B"]):
        r = slice(ends[i], ends[i + 1])
        S = pool[src[i]].clone() if src[i] >= 0 else torch.zeros_like(pool[0])
        delta = torch.logaddexp(f("dt")[r] + f("dt_bias"), torch.zeros((), dtype=torch.float64, device="cuda"))
        x, keep = s["x"][r].double(), torch.exp(delta * A)
        b, cc = s["b"][r].double(), s["c"][r].double()
        y = torch.empty_like(x)
        for t in range(n[i]):
            u = (delta[t, :, None] * x[t]).unflatten(0, (c["NG"], G))
            S *= keep[t][:, None, None]
            S += (b[t][:, None, :, None] * u[:, :, None, :]).flatten(0, 1)
            y[t] = (S.unflatten(0, (c["NG"], G)) * cc[t][:, None, :, None]).sum(2).flatten(0, 1)
        y += D[:, None] * x
        if s["z"] is not None:
            z = s["z"][r].double()
            y *= z * torch.sigmoid(z)
        out.append(y)
        new[dst[i]] = S
    return [torch.cat(out), new]
