"""Cases of the linear-attention block's operators, for whole prompts and for single tokens.

Each case is a plain dict whose "kind" names the operator:

  attend  linear_attention: causal linear attention with a decay for each head,
          over whole sequences (a batch of them padded to one length)
  step    linear_attention_step: the same recurrence, one token a row, over a
          pool of states
  norm    residual_norm: norm after a block, gate and residual scale, and the
          next block's modulated norm
  w4      linear_w4: few rows times 4-bit weights with group scales

With own = False run() computes the operator from elementary torch operations
in 32 bits (64 where a decay is raised to a far position); with own = True it
calls the library.
"""
from __future__ import annotations

import math
from types import SimpleNamespace

import torch

own = False

DEV = "cuda"
CHUNK = 64  # tokens a chunk of the plain form


# ------------------------------------------------------------------ cases


def listed():
    return [
        # A whole 21 x 30 x 52 latent video as one causal sequence, from an
        # empty state; the final state is kept to go on from.
        dict(name="attend_video", kind="attend", dtype="bf16", seqs=1, heads=12, head_dim=128,
             tokens=21 * 30 * 52, ragged=False, carried=False),
        # Eight prompts of up to 512 tokens padded to one length, heads of 64.
        dict(name="attend_text_batch", kind="attend", dtype="bf16", seqs=8, heads=16, head_dim=64,
             tokens=512, ragged=True, carried=True),
        # The next latent frame of a stream, fp32 model, odd token count.
        dict(name="attend_frame_f32", kind="attend", dtype="f32", seqs=1, heads=4, head_dim=64,
             tokens=1559, ragged=False, carried=True),
        # A handful of tokens onto a carried state: latency.
        dict(name="attend_few_tokens", kind="attend", dtype="bf16", seqs=1, heads=12, head_dim=128,
             tokens=17, ragged=False, carried=True),
        # One token of one sequence: latency.
        dict(name="step_one", kind="step", dtype="bf16", rows=1, heads=12, head_dim=128,
             slots=0, padding=0),
        # A serving batch whose rows name their states in a larger pool, the
        # last rows padding.
        dict(name="step_pool", kind="step", dtype="bf16", rows=256, heads=12, head_dim=128,
             slots=320, padding=9),
        # Behind attention in a block over a whole video: RMS norm after,
        # adaLN gate, LayerNorm and modulation before the MLP.
        dict(name="norm_video", kind="norm", dtype="bf16", rows=21 * 30 * 52, hidden=1536,
             post="rms", pre="layer", mod_rows=0, res_scale=1.0),
        # fp32 model, every latent frame with its own noise level (one
        # modulation row each 250 tokens), deep-network residual scale.
        dict(name="norm_frames_f32", kind="norm", dtype="f32", rows=1000, hidden=1024,
             post="layer", pre="rms", mod_rows=250, res_scale=0.81),
        # A few tokens of a wide model: latency.
        dict(name="norm_tokens", kind="norm", dtype="bf16", rows=4, hidden=4096,
             post="rms", pre="rms", mod_rows=0, res_scale=1.0),
        # Q, K and V of one token at width 1536.
        dict(name="w4_one_token", kind="w4", dtype="bf16", out="bf16", rows=1, n=4608, k=1536,
             group=128, gelu=False),
        # The first MLP product of a wide model for a batch of eight tokens.
        dict(name="w4_wide_mlp", kind="w4", dtype="bf16", out="bf16", rows=8, n=28672, k=8192,
             group=128, gelu=True),
        # fp32 rows, small groups, an odd number of outputs.
        dict(name="w4_f32_odd", kind="w4", dtype="f32", out="f32", rows=3, n=5001, k=2048,
             group=32, gelu=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("attend", "attend", "step", "norm", "w4"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if kind == "attend":
        d, seqs = rng.choice((64, 128)), _log(rng, 1, 16)
        heads = rng.randint(1, 32)
        most = 12 * 32760 * 128 // (4 if dtype == "f32" else 1)
        tokens = _log(rng, 1, max(2, min(32760, most // (seqs * heads * d))))
        return dict(kind=kind, dtype=dtype, seqs=seqs, heads=heads, head_dim=d, tokens=tokens,
                    ragged=rng.random() < 0.5, carried=rng.random() < 0.5)
    if kind == "step":
        rows, d = _log(rng, 1, 256), rng.choice((64, 128))
        heads = rng.randint(1, 12 if d == 128 else 32)
        slots = rng.choice((0, rows + rng.randint(0, 64)))
        return dict(kind=kind, dtype=dtype, rows=rows, heads=heads, head_dim=d, slots=slots,
                    padding=rng.randint(0, rows // 4) if slots else 0)
    if kind == "norm":
        hidden = 4 * _log(rng, 16, 2048)
        rows = _log(rng, 1, max(2, min(60000, 32760 * 1536 // (2 * hidden))))
        return dict(kind=kind, dtype=dtype, rows=rows, hidden=hidden,
                    post=rng.choice(("none", "layer", "rms")), pre=rng.choice(("layer", "rms")),
                    mod_rows=rng.choice((0, rng.randint(1, rows))),
                    res_scale=rng.choice((1.0, 0.5, 1.7)))
    k = 128 * _log(rng, 1, 64)
    n = _log(rng, 16, max(17, min(28672, 28672 * 4096 // k)))
    return dict(kind="w4", dtype=dtype, out=rng.choice(("bf16", "f32")), rows=_log(rng, 1, 32), n=n,
                k=k, group=rng.choice((32, 64, 128)), gelu=rng.random() < 0.3)


# ----------------------------------------------------------------- inputs


def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _generator(seed, k):
    g = torch.Generator(device=DEV)
    g.manual_seed((seed * 1000003 + k * 7919 + 29) % (1 << 62))
    return g


def _normal(shape, seed, k, std=1.0, mean=0.0):
    t = torch.randn(shape, generator=_generator(seed, k), device=DEV, dtype=torch.float32)
    return t.mul_(std).add_(mean)


def _whole(lo, hi, shape, seed, k, dtype=torch.int32):
    return torch.randint(lo, hi, shape, generator=_generator(seed, k), device=DEV, dtype=dtype)


def _slopes(heads):
    """Decay rates in a geometric row from 1/2 down to 2^-8; the last head
    of several never forgets."""
    s = [2.0 ** (-8.0 * (h + 1) / heads) for h in range(heads)]
    if heads > 2:
        s[-1] = 0.0
    return torch.tensor(s, dtype=torch.float32, device=DEV)


def prepare(case, seed):
    c = case
    s = SimpleNamespace(c=c)
    if c["kind"] == "attend":
        n, h, t, d = c["seqs"], c["heads"], c["tokens"], c["head_dim"]
        dt = _dtype(c["dtype"])
        s.q, s.k = (_normal((n, h, t, d), seed, i).to(dt) for i in (1, 2))
        s.vt = torch.zeros((n, h, d, (t + 7) // 8 * 8), dtype=dt, device=DEV)
        s.vt[..., :t] = _normal((n, h, d, t), seed, 3).to(dt)
        s.slopes = _slopes(h)
        s.lengths = _whole(0, t + 1, (n,), seed, 4) if c["ragged"] else None
        s.state = _normal((n, h, d, d), seed, 5) if c["carried"] else None
        s.state_out = torch.zeros((n, h, d, d), dtype=torch.float32, device=DEV)
        s.o = torch.zeros((n, t, h * d), dtype=dt, device=DEV)
        s.scale = d ** -0.5
    elif c["kind"] == "step":
        n, h, d = c["rows"], c["heads"], c["head_dim"]
        pool = c["slots"] or n
        # Q | K | V side by side, as one projection leaves them
        qkv = _normal((n, 3 * h * d), seed, 1).to(_dtype(c["dtype"]))
        s.q, s.k, s.v = (qkv[:, i * h * d:(i + 1) * h * d] for i in range(3))
        s.slopes = _slopes(h)
        s.state = _normal((pool, h, d, d), seed, 2)
        s.state_out = torch.zeros_like(s.state)
        s.o = torch.zeros((n, h * d), dtype=qkv.dtype, device=DEV)
        s.slots = None
        if c["slots"]:
            s.slots = torch.randperm(pool, generator=_generator(seed, 3), device=DEV)[:n].to(torch.int32)
            s.slots[n - c["padding"]:] = -1
        s.scale = d ** -0.5
    elif c["kind"] == "norm":
        n, h = c["rows"], c["hidden"]
        mods = -(-n // c["mod_rows"]) if c["mod_rows"] else 1
        s.h = _normal((n, h), seed, 1, 2.0, 0.3)
        s.y = _normal((n, h), seed, 2, 1.5, 0.2).to(_dtype(c["dtype"]))
        s.gate, s.shift, s.mscale = (_normal((mods, h), seed, 3 + i, 0.3) for i in range(3))
        s.post_weight = _normal((h,), seed, 6, 0.1, 1.0) if c["post"] != "none" else None
        s.pre_weight = _normal((h,), seed, 7, 0.1, 1.0) if c["pre"] == "rms" else None
        s.h_out = torch.zeros_like(s.h)
        s.a = torch.zeros((n, h), dtype=_dtype(c["dtype"]), device=DEV)
    else:
        m, n, k, g = c["rows"], c["n"], c["k"], c["group"]
        tiles = (n + 15) // 16
        s.x = _normal((m, k), seed, 1).to(_dtype(c["dtype"]))
        # codes and scales as the library lays them out: any bytes are codes
        s.codes = _whole(0, 256, (tiles, k // 128, 64, 16), seed, 2, torch.uint8)
        s.scales = _normal((tiles, k // g, 16), seed, 3, 0.001, 0.005)
        s.bias = _normal((n,), seed, 4, 0.1)
        s.out = torch.zeros((m, n), dtype=_dtype(c["out"]), device=DEV)
    return s


# ------------------------------------------------------------- plain forms


def _plain_attend(s):
    n, h, t, d = s.q.shape
    chunks = -(-t // CHUNK)
    pad = chunks * CHUNK - t
    lengths = s.lengths if s.lengths is not None else torch.full((n,), t, dtype=torch.int32, device=DEV)
    at = torch.arange(chunks * CHUNK, device=DEV)
    live = (at[None, :] < lengths[:, None])[:, None, :, None]  # [n, 1, tokens, 1]

    def cut(x):  # [n, h, t, d] -> [n h, chunks, CHUNK, d], dead tokens 0
        x = torch.nn.functional.pad(x.float(), (0, 0, 0, pad))
        return torch.where(live, x, torch.zeros((), device=DEV)).reshape(n * h, chunks, CHUNK, d)

    q, k, v = cut(s.q), cut(s.k), cut(s.vt[..., :t].transpose(2, 3))
    rate = s.slopes.double().repeat(n)[:, None]                               # [n h, 1]
    count = (lengths[:, None] - at[None, ::CHUNK]).clamp(0, CHUNK)            # [n, chunks]
    count = count.repeat_interleave(h, 0)                                     # live tokens
    i = torch.arange(CHUNK, device=DEV)
    # each chunk's own part of the state, decayed to its last live token
    left = (count[:, :, None] - 1 - i).clamp(min=0)
    own_part = (k * torch.exp(-rate[:, :, None] * left).float()[..., None]).transpose(2, 3).contiguous() @ v
    # the state at each chunk's start: a sum over all earlier chunks and the
    # carried state, each decayed by the tokens since
    done = count.cumsum(1)
    since = torch.exp(-rate[:, :, None] * (torch.nn.functional.pad(done, (1, 0))[:, :, None] - done[:, None, :]))
    since = torch.where(torch.arange(chunks + 1, device=DEV)[:, None] > torch.arange(chunks, device=DEV)[None, :],
                        since, torch.zeros((), dtype=torch.float64, device=DEV)).float()
    states = (since @ own_part.reshape(n * h, chunks, d * d)).reshape(n * h, chunks + 1, d, d)
    if s.state is not None:
        gone = torch.exp(-rate * torch.nn.functional.pad(done, (1, 0))).float()
        states = states + gone[..., None, None] * s.state.reshape(n * h, 1, d, d)
    decay = torch.exp(-rate[:, :, None] * (i[:, None] - i[None, :]).clamp(min=0)).float()
    scores = (q @ k.transpose(2, 3).contiguous()) * torch.where(i[:, None] >= i[None, :], decay, torch.zeros((), device=DEV))[:, None]
    o = scores @ v + torch.exp(-rate * (i + 1)).float()[:, None, :, None] * (q @ states[:, :-1])
    o = (s.scale * o).reshape(n, h, chunks * CHUNK, d)[:, :, :t]
    o = torch.where(live[:, :, :t], o, torch.zeros((), device=DEV))
    return {"o": o.transpose(1, 2).reshape(n, t, h * d).to(s.o.dtype),
            "state": states[:, -1].reshape(n, h, d, d)}


def _plain_step(s):
    n, h, d = s.q.shape[0], s.slopes.numel(), s.state.shape[-1]
    q, k, v = (x.float().reshape(n, h, d) for x in (s.q, s.k, s.v))
    rows = torch.arange(n - s.c["padding"], device=DEV)
    at = s.slots[rows].long() if s.slots is not None else rows
    new = torch.exp(-s.slopes)[:, None, None] * s.state[at] + k[rows][..., :, None] * v[rows][..., None, :]
    s.state_out[at] = new
    s.o[rows] = (s.scale * (q[rows][..., :, None] * new).sum(2)).reshape(-1, h * d).to(s.o.dtype)
    return {"o": s.o, "state": s.state_out}


def _plain_normed(x, kind, weight):
    if kind == "layer":
        x = x - x.mean(1, keepdim=True)
    if kind != "none":
        x = x * torch.rsqrt((x * x).mean(1, keepdim=True) + 1e-6)
    return x if weight is None else x * weight


def _plain_norm(s):
    c = s.c
    row = torch.arange(c["rows"], device=DEV) // (c["mod_rows"] or c["rows"])
    h = c["res_scale"] * s.h + s.gate[row] * _plain_normed(s.y.float(), c["post"], s.post_weight)
    a = _plain_normed(h, c["pre"], s.pre_weight) * (1 + s.mscale[row]) + s.shift[row]
    return {"h": h, "a": a.to(s.a.dtype)}


def _gelu(y):
    return 0.5 * y * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)))


def _weights(codes, scales, n, dtype):
    """[n][k] weights from the library's layout: a tile of 16 outputs holds,
    for each 128 inputs, 64 runs of 16 bytes; run l is output l % 16, and its
    4-byte word j has inputs 32 j + 8 (l / 16) + (0, 2, 4, 6, 1, 3, 5, 7) in
    its nibbles from the lowest up."""
    tiles, blocks = codes.shape[:2]
    c = codes.reshape(tiles, blocks, 4, 16, 4, 4)                # tile, block, g, n, j, byte
    c = torch.stack((c & 15, c >> 4), -1).reshape(tiles, blocks, 4, 16, 4, 2, 4)  # ..., odd, half
    c = c.permute(0, 3, 1, 4, 2, 6, 5).reshape(tiles * 16, blocks * 128)  # j, g, half, odd
    w = scales.to(dtype).transpose(1, 2).reshape(tiles * 16, -1, 1) * (
        c.to(dtype) - 8).reshape(tiles * 16, scales.shape[1], -1)
    return w.reshape(tiles * 16, -1)[:n]


def _plain_w4(s):
    w = _weights(s.codes, s.scales, s.c["n"], torch.float32)
    y = s.x.float() @ w.t() + s.bias
    return {"out": (_gelu(y) if s.c["gelu"] else y).to(s.out.dtype)}


# -------------------------------------------------------------------- run


def run(s):
    c = s.c
    if not own:
        return {"attend": _plain_attend, "step": _plain_step, "norm": _plain_norm,
                "w4": _plain_w4}[c["kind"]](s)
    import paper_2607_12358_amd as A
    if c["kind"] == "attend":
        A.linear_attention(s.q, s.k, s.vt, s.slopes, s.o, state_in=s.state, state_out=s.state_out,
                           lengths=s.lengths, scale=s.scale)
        return {"o": s.o, "state": s.state_out}
    if c["kind"] == "step":
        A.linear_attention_step(s.q, s.k, s.v, s.slopes, s.o, s.state, state_out=s.state_out,
                                slots=s.slots, scale=s.scale)
        return {"o": s.o, "state": s.state_out}
    if c["kind"] == "norm":
        A.residual_norm(s.h, s.y, h_out=s.h_out, out=s.a, res_scale=c["res_scale"], post=c["post"],
                        post_weight=s.post_weight, gate=s.gate, pre=c["pre"],
                        pre_weight=s.pre_weight, shift=s.shift, scale=s.mscale,
                        rows_per_mod=c["mod_rows"])
        return {"h": s.h_out, "a": s.a}
    A.linear_w4(s.x, s.codes, s.scales, s.out, bias=s.bias, gelu=c["gelu"])
    return {"out": s.out}


def work(case):
    c = case
    size = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "attend":
        tokens, d = c["seqs"] * c["heads"] * c["tokens"], c["head_dim"]
        if c["ragged"]:
            tokens //= 2  # lengths are uniform in 0 .. tokens
        states = c["seqs"] * c["heads"] * d * d * (2 if c["carried"] else 1)
        return {"bytes": 4 * size * tokens * d + 4 * states, "flops": 4 * tokens * d * d}
    if c["kind"] == "step":
        live, d = (c["rows"] - c["padding"]) * c["heads"], c["head_dim"]
        return {"bytes": live * (8 * d * d + 4 * size * d), "flops": 5 * live * d * d}
    if c["kind"] == "norm":
        values = c["rows"] * c["hidden"]
        return {"bytes": values * (8 + 2 * size), "flops": 16 * values}
    m, n, k = c["rows"], c["n"], c["k"]
    return {"bytes": n * k // 2 + 4 * n * (k // c["group"]) + m * k * size
            + m * n * (2 if c["out"] == "bf16" else 4), "flops": 2 * m * n * k}


# ------------------------------------------------------------------ exact


def exact(case, seed):
    """run()'s outputs from the definitions, in 64 bits."""
    c = case
    s = prepare(c, seed)
    if c["kind"] == "attend":
        return _exact_attend(s)
    if c["kind"] == "step":
        h, d = c["heads"], c["head_dim"]
        o, state = torch.zeros(s.o.shape, dtype=torch.float64, device=DEV), s.state_out.double()
        for r in range(c["rows"] - c["padding"]):
            at = int(s.slots[r]) if s.slots is not None else r
            q, k, v = (x[r].double().reshape(h, d) for x in (s.q, s.k, s.v))
            was = s.state[at].double() * torch.exp(-s.slopes.double())[:, None, None]
            state[at] = was + k[:, :, None] * v[:, None, :]
            # q (lambda S + k v) = lambda (q S) + (q . k) v
            o[r] = s.scale * (torch.matmul(q[:, None, :], was)[:, 0] + (q * k).sum(1, keepdim=True) * v).reshape(-1)
        return {"o": o, "state": state}
    if c["kind"] == "norm":
        y, h = s.y.double(), s.h.double()
        per = c["mod_rows"] or c["rows"]
        gate, shift, scale = (m.double().repeat_interleave(per, 0)[: c["rows"]]
                              for m in (s.gate, s.shift, s.mscale))

        def normed(x, kind, w):
            if kind == "layer":
                x = (x - x.mean(1, keepdim=True)) / torch.sqrt(x.var(1, unbiased=False, keepdim=True) + 1e-6)
            elif kind == "rms":
                x = x / torch.sqrt(x.pow(2).sum(1, keepdim=True) / x.shape[1] + 1e-6)
            return x if w is None else w.double() * x

        h = h * c["res_scale"] + normed(y, c["post"], s.post_weight) * gate
        z = normed(h, c["pre"], s.pre_weight)
        return {"h": h, "a": z + z * scale + shift}
    # w4, from the layout's words: one output tile, word and nibble at a time
    x, g = s.x.double(), c["group"]
    tiles = s.codes.shape[0]
    y = torch.zeros((c["rows"], tiles, 16), dtype=torch.float64, device=DEV)
    for j in range(4):
        for run_ in range(4):
            part = s.codes.reshape(tiles, -1, 4, 16, 4, 4)[:, :, run_, :, j]    # tile, block, n, byte
            for e in range(8):
                nibble = (0, 4, 1, 5, 2, 6, 3, 7)[e]
                code = (part[..., nibble // 2] >> (4 * (nibble % 2))) & 15
                at = 128 * torch.arange(part.shape[1], device=DEV) + 32 * j + 8 * run_ + e
                w = (code.double() - 8) * s.scales.double()[:, at // g]          # tile, block, n
                y += torch.matmul(x[:, at], w.transpose(0, 1).reshape(len(at), -1)).reshape(y.shape)
    y = y.reshape(c["rows"], -1)[:, : c["n"]] + s.bias.double()
    if c["gelu"]:
        y = y / 2 * (1 + torch.tanh((y + 0.044715 * y * y * y) * (2 / math.pi) ** 0.5))
    return {"out": y}


def _exact_attend(s, rows=512):
    """o_i = scale sum_{j <= i} lambda^(i-j) (q_i k_j) v_j + scale lambda^(i+1) q_i S_0."""
    n, h, t, d = s.q.shape
    rate = s.slopes.double()[:, None, None]
    o = torch.zeros((n, t, h * d), dtype=torch.float64, device=DEV)
    state = torch.zeros((n, h, d, d), dtype=torch.float64, device=DEV)
    for b in range(n):
        live = t if s.lengths is None else int(s.lengths[b])
        was = s.state[b].double() if s.state is not None else state[b].clone()
        q, k, v = s.q[b].double(), s.k[b].double(), s.vt[b, :, :, :t].double().transpose(1, 2).contiguous()
        for i0 in range(0, live, rows):
            i1 = min(live, i0 + rows)
            far = torch.arange(i0, i1, device=DEV)[:, None] - torch.arange(i1, device=DEV)[None, :]
            p = torch.matmul(q[:, i0:i1], k[:, :i1].transpose(1, 2).contiguous())
            p *= torch.exp(-rate * far.clamp(min=0)) * (far >= 0)
            part = torch.matmul(p, v[:, :i1])
            part += torch.exp(-rate * torch.arange(i0 + 1, i1 + 1, device=DEV)[None, :, None]) * torch.matmul(q[:, i0:i1], was)
            o[b, i0:i1] = s.scale * part.transpose(0, 1).reshape(i1 - i0, h * d)
        fade = torch.exp(-rate * (live - 1 - torch.arange(live, device=DEV))[None, :, None])
        state[b] = torch.matmul((k[:, :live] * fade).transpose(1, 2).contiguous(), v[:, :live])
        state[b] += torch.exp(-rate * live) * was
    return {"o": o, "state": state}
