"""The operators around a layer's products that this framework is timed on.

Between two rounds every worker of a simulated training run computes a forward
and a backward pass with its own weights (the rows of x[n][d]).  The products
and the plain norm of such a pass are timed in operators.py; here are what
mixes the tokens and the norm that stands around a block:

  attention        out = softmax(scale * Q K^T) V of packed sequences, causal,
                   query heads in groups that share a key head, and the
                   gradients of Q, K and V
  recurrence       h_t = a_t * h_(t-1) + (1 - a_t) * x_t with a = sigmoid(gate),
                   channel by channel, over packed sequences with an initial
                   state each, and the gradients of gate, x and the states
  blocknorm        s = residual + scale * sigmoid(gate) * norm(z) * post_weight;
                   y = norm(s) * pre_weight: the norm behind a block with its
                   gate and residual scale and the norm in front of the next
                   block; y is held in 8 bits, in training s too
  blocknorm_backward   its gradients, from the s kept in 8 bits

Sequences are packed: starts[n][count + 1] has the row on which each of a
worker's sequences begins, and where the last one ends.  Rows behind that
belong to none; what an operator gives there is 0, and what it reads there has
no part in anything.

Sizes are generic: widths and heads of small to mid-sized transformers, odd
ones, one token to long batches, 1 to 64 workers.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6
GROUP = 128
DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
BYTES = {"float32": 4, "bfloat16": 2, "float16": 2}


def listed():
    return [
        # Evaluation: the next token of 16 workers' models against what each has read.
        dict(name="attention_token", op="attention", n=16, t=1, keys=1024, heads=12, kv=4, width=64,
             count=1, dtype="bfloat16", grad=False),
        # A few workers, odd sizes, texts of different lengths and padding behind them.
        dict(name="attention_odd", op="attention", n=3, t=777, keys=777, heads=6, kv=2, width=80,
             count=5, dtype="float16", grad=True),
        # A training batch of 16 workers, packed texts; evaluation of it.
        dict(name="attention_batch", op="attention", n=16, t=2048, keys=2048, heads=16, kv=4, width=64,
             count=3, dtype="bfloat16", grad=False),
        # The same batch's training step.
        dict(name="attention_back_batch", op="attention", n=16, t=2048, keys=2048, heads=16, kv=4,
             width=64, count=3, dtype="bfloat16", grad=True),
        # One worker with one long text.
        dict(name="attention_back_long", op="attention", n=1, t=16384, keys=16384, heads=8, kv=2,
             width=128, count=1, dtype="bfloat16", grad=True),
        # Evaluation: a token for each of 16 workers, from the states that they keep.
        dict(name="recurrence_token", op="recurrence", n=16, t=1, width=1024, count=1,
             dtype="bfloat16", grad=False),
        # A batch of 16 workers' packed texts.
        dict(name="recurrence_batch", op="recurrence", n=16, t=2048, width=1024, count=3,
             dtype="bfloat16", grad=False),
        # Its training step.
        dict(name="recurrence_back_batch", op="recurrence", n=16, t=2048, width=1024, count=3,
             dtype="bfloat16", grad=True),
        # One worker, a very long text and odd channels, in 32 bits.
        dict(name="recurrence_back_long", op="recurrence", n=1, t=65536, width=333, count=1,
             dtype="float32", grad=True),
        # A training batch of 16 workers, with what the backward pass needs.
        dict(name="blocknorm_batch", op="blocknorm", n=16, t=2048, width=1024, dtype="bfloat16",
             gated=True, keep=True),
        # A few workers with odd sizes, in 32 bits, without a gate.
        dict(name="blocknorm_back_odd", op="blocknorm_backward", n=5, t=777, width=1001, dtype="float32",
             gated=False),
        dict(name="blocknorm_back_batch", op="blocknorm_backward", n=16, t=2048, width=1024,
             dtype="bfloat16", gated=True),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A pass of 1 to 64 workers, 1 to 65,536 tokens, heads of 16 to 256 or
    channels of 16 to 8,192, that does at most what the largest listed do."""
    op = rng.choice(["attention"] * 5 + ["recurrence"] * 3 + ["blocknorm", "blocknorm_backward"])
    n = _logint(rng, 1, 64)
    case = dict(op=op, n=n, dtype=rng.choice(["bfloat16", "bfloat16", "float16", "float32"]))
    if op == "attention":
        kv = rng.choice([1, 2, 3, 4, 6, 8])
        heads = kv * rng.choice([1, 1, 2, 3, 4, 8])
        width = rng.choice([16, 32, 33, 48, 64, 64, 64, 80, 96, 100, 128, 128, 192, 256])
        grad = rng.random() < 0.6
        # What the scores of the plain form take, and the products.
        scores = min(2.0 ** 31, 2.7e11 / width)
        if case["dtype"] == "float32":
            scores /= 4
        if rng.random() < 0.2:
            # A few new tokens behind a text.
            t = _logint(rng, 1, 32)
            keys = _logint(rng, t, max(t, min(65536.0, scores / (n * heads * t), 1e8 / (n * kv * width))))
            case.update(t=t, keys=keys, count=1, grad=False)
        else:
            top = min(16384.0, math.sqrt(scores / (n * heads)), 1e8 / (n * heads * width))
            t = _logint(rng, 1, max(1.0, top))
            case.update(t=t, keys=t, count=_logint(rng, 1, max(1, min(64, t // 8))), grad=grad)
        case.update(heads=heads, kv=kv, width=width)
        return case
    k = _logint(rng, 16, 8192)
    if rng.random() < 0.6:
        k = -(-k // 32) * 32
    case["width"] = k
    top = min(65536.0, 1e8 / BYTES[case["dtype"]] / (n * k))
    # One in six a single token, the others spread over the lengths.
    case["t"] = t = 1 if rng.random() < 1 / 6 or top < 2 else _logint(rng, 1, top)
    if op == "recurrence":
        case["count"] = _logint(rng, 1, max(1, min(64, t // 4)))
        case["grad"] = rng.random() < 0.6
    else:
        case["gated"] = rng.random() < 0.7
        if op == "blocknorm":
            case["keep"] = rng.random() < 0.7
    return case


# ---- 8-bit rows in elementary operations ---------------------------------------


def _stride(width):
    return -(-width // GROUP) * GROUP


def _pack(v, group):
    """(codes, exponents) of float rows v[n][rows][width]: a group of entries
    (a whole row, or 128 of it) as rint(v / 2^e), the smallest e >= -126 that
    keeps the codes within 127."""
    n, rows, width = v.shape
    s = _stride(width)
    v = torch.nn.functional.pad(v, (0, s - width))
    v = v.view(n, rows, -1, group) if group else v.view(n, rows, 1, s)
    a = v.abs().amax(-1)
    m, p = torch.frexp(a)
    e = torch.where(a > 0, p - 7 + (m > 127 / 128), -126).clamp(min=-126)
    q = torch.round(torch.ldexp(v, -e.unsqueeze(-1)))
    return q.to(torch.int8).view(n, rows, s), e.to(torch.int8)


def _values(codes, exps, width):
    """What codes and exponents stand for."""
    n, rows, s = codes.shape
    v = codes.float().view(n, rows, exps.shape[2], -1)
    return torch.ldexp(v, exps.unsqueeze(-1).to(torch.int32)).view(n, rows, s)[..., :width]


# ---- inputs ----------------------------------------------------------------------


def _model_view(gen, dev, n, width, std, mean=0.0):
    """A vector [n][width] in the middle of model rows of odd length, 4 bytes
    off any wider alignment, as a parameter in a model is."""
    d = width + 7 if width % 2 == 0 else width + 8
    x = torch.empty(n, d, device=dev).normal_(mean, std, generator=gen)
    return x[:, 3:3 + width]


def _starts(gen, dev, n, t, count):
    """Where every worker's sequences begin, and the last one ends: about
    even lengths, and with several of them some rows of padding behind."""
    if count == 1:
        at = torch.tensor([0, t], device=dev).expand(n, 2)
    else:
        step = t / count
        at = torch.arange(1, count + 1, device=dev) * step
        at = at + (torch.rand(n, count, device=dev, generator=gen) - 0.5) * step
        at[:, -1] = t - torch.rand(n, device=dev, generator=gen) * step * 0.5
        at = torch.cat([torch.zeros(n, 1, device=dev), at], 1).floor().clamp(0, t)
    return at.to(torch.int32).contiguous()


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    n, t, k, dt = case["n"], case["t"], case["width"], DTYPES[case["dtype"]]
    st = dict(case=case, dt=dt)

    def normal(*shape, std=1.0):
        return torch.empty(*shape, device=dev).normal_(0.0, std, generator=gen)

    def stream(rows, width):
        # A residual stream: features of different sizes, a few of them large.
        size = torch.exp(normal(n, 1, width, std=0.5))
        return normal(n, rows, width).mul_(size)

    if case["op"] == "attention":
        heads, kv, keys = case["heads"], case["kv"], case["keys"]
        if keys == t:
            # Views into what one projection of the tokens gave.
            row = normal(n, t, (heads + 2 * kv) * k).to(dt)
            row = row.unflatten(2, (heads + 2 * kv, k))
            st["q"], st["k"], st["v"] = row.split([heads, kv, kv], 2)
        else:
            st["q"] = normal(n, t, heads, k).to(dt)
            st["k"], st["v"] = normal(n, keys, kv, k).to(dt), normal(n, keys, kv, k).to(dt)
        st["starts"] = _starts(gen, dev, n, t, case["count"])
        # With more keys than queries the queries are a text's last tokens.
        st["key_starts"] = st["starts"] if keys == t else _starts(gen, dev, n, keys, 1)
        if case["grad"]:
            st["dout"] = normal(n, t, heads, k, std=1e-2).to(dt)
    elif case["op"] == "recurrence":
        # Gates that keep between a token and a few hundred.
        st["gate"] = (normal(n, t, k, std=1.0) + 2.0 * normal(n, 1, k).abs()).to(dt)
        st["x"] = stream(t, k).to(dt)
        st["initial"] = normal(n, case["count"], k)
        st["starts"] = _starts(gen, dev, n, t, case["count"])
        if case["grad"]:
            st["dh"] = normal(n, t, k, std=1e-2).to(dt)
            st["dlast"] = normal(n, case["count"], k, std=1e-2)
    else:
        st["post"] = _model_view(gen, dev, n, k, 0.1, 1.0)
        st["pre"] = _model_view(gen, dev, n, k, 0.1, 1.0)
        st["scale"] = _model_view(gen, dev, n, 1, 0.05, 0.5)[:, 0]
        st["z"] = stream(t, k).to(dt)
        st["gate"] = normal(n, t, k).to(dt) if case["gated"] else None
        if case["op"] == "blocknorm":
            st["residual"] = stream(t, k).to(dt)
        else:
            s = stream(t, k)
            st["codes"], st["exps"] = _pack(s, GROUP)
            st["post_rstd"] = torch.rsqrt(st["z"].float().square().mean(-1) + EPS)
            st["rstd"] = torch.rsqrt(s.square().mean(-1) + EPS)
            st["dy"] = normal(n, t, k, std=1e-2).to(dt)
            st["dsum"] = normal(n, t, k, std=1e-2).to(dt)
            st["dpost"] = _model_view(gen, dev, n, k, 0.0)
            st["dpre"] = _model_view(gen, dev, n, k, 0.0)
            st["dscale"] = _model_view(gen, dev, n, 1, 0.0)[:, 0]
    return st


# ---- one pass, in elementary operations --------------------------------------------


def _sequence(starts, rows):
    """The sequence of every row [n][rows]: -1 or count where it is in none."""
    at = torch.arange(rows, device=starts.device, dtype=torch.int32).expand(starts.shape[0], rows)
    return torch.searchsorted(starts, at.contiguous(), right=True) - 1


def _hidden(starts, key_starts, t, keys):
    """[n][t][keys]: which keys a query does not see.  The last query of a
    sequence sees all of its keys, each one before it a key less."""
    count = starts.shape[1] - 1
    sq, sk = _sequence(starts, t), _sequence(key_starts, keys)
    inside = ((sq >= 0) & (sq < count)).unsqueeze(2)
    end = sq.clamp(0, count - 1) + 1
    left = starts.gather(1, end) - 1 - torch.arange(t, device=starts.device)
    last = key_starts.gather(1, end) - left
    seen = (sq.unsqueeze(2) == sk.unsqueeze(1)) & inside
    return ~(seen & (torch.arange(keys, device=starts.device) < last.unsqueeze(2)))


def _attention(st):
    case, dt = st["case"], st["dt"]
    n, t, keys, heads, kv, d = (case[i] for i in ("n", "t", "keys", "heads", "kv", "width"))
    scale = d ** -0.5

    def split(v):
        # [n][t][heads][d] -> [n][kv][heads / kv * t][d]
        return v.float().view(n, t, kv, heads // kv, d).permute(0, 2, 3, 1, 4).reshape(n, kv, -1, d)

    def join(v):
        return v.view(n, kv, heads // kv, t, d).permute(0, 3, 1, 2, 4).reshape(n, t, heads, d).to(dt)

    q = split(st["q"])
    k, v = (st[i].float().transpose(1, 2).contiguous() for i in ("k", "v"))
    hidden = _hidden(st["starts"], st["key_starts"], t, keys)
    p = torch.matmul(q, k.transpose(2, 3)).mul_(scale)
    p.view(n, kv, -1, t, keys).masked_fill_(hidden.view(n, 1, 1, t, keys), -math.inf)
    most = p.amax(-1, keepdim=True)
    p = p.sub_(torch.where(most == -math.inf, 0.0, most)).exp_()
    p = p.div_(p.sum(-1, keepdim=True).clamp(min=1e-38))
    out = join(torch.matmul(p, v))
    if not case["grad"]:
        return [out]
    dout = split(st["dout"])
    # Rows of no sequence have no gradient, whatever stands there.
    dv = torch.matmul(p.transpose(2, 3), dout)
    ds = torch.matmul(dout, v.transpose(2, 3))
    ds = ds.sub_((ds * p).sum(-1, keepdim=True)).mul_(p).mul_(scale)
    dq = join(torch.matmul(ds, k))
    dk = torch.matmul(ds.transpose(2, 3), q)
    return [out, dq, dk.transpose(1, 2).contiguous().to(dt), dv.transpose(1, 2).contiguous().to(dt)]


def _scan(a, b):
    """c_t = a_t * c_(t-1) + b_t along axis 1, in steps of doubled reach."""
    t, reach = a.shape[1], 1
    while reach < t:
        b = torch.cat([b[:, :reach], torch.addcmul(b[:, reach:], a[:, reach:], b[:, :-reach])], 1)
        a = torch.cat([a[:, :reach], a[:, reach:] * a[:, :-reach]], 1)
        reach *= 2
    return b


def _recurrence(st):
    case, dt = st["case"], st["dt"]
    n, t, w, count = case["n"], case["t"], case["width"], case["count"]
    seq = _sequence(st["starts"], t)
    inside = ((seq >= 0) & (seq < count)).unsqueeze(2)
    at = seq.clamp(0, count - 1)
    index = torch.arange(t, device=seq.device)
    first = (st["starts"].gather(1, at) == index).unsqueeze(2)
    final = (st["starts"].gather(1, at + 1) - 1 == index).unsqueeze(2)
    gate, x = st["gate"].float(), st["x"].float()
    a, c = torch.sigmoid(gate), torch.sigmoid(-gate)
    before = torch.gather(st["initial"], 1, at.unsqueeze(2).expand(n, t, w))
    keep = torch.where(inside & ~first, a, 0.0)
    new = torch.where(inside, c * x + torch.where(first, a * before, 0.0), 0.0)
    h = _scan(keep, new)
    ends = (st["starts"][:, 1:].long() - 1).unsqueeze(2).expand(n, count, w)
    empty = (st["starts"][:, 1:] == st["starts"][:, :-1]).unsqueeze(2)
    last = torch.where(empty, st["initial"], torch.gather(h, 1, ends.clamp(min=0)))
    if not case["grad"]:
        return [h.to(dt), last]
    dlast = torch.gather(st["dlast"], 1, at.unsqueeze(2).expand(n, t, w))
    dh = torch.where(inside, st["dh"].float() + torch.where(final, dlast, 0.0), 0.0)
    on = torch.cat([keep[:, 1:], torch.zeros_like(keep[:, :1])], 1)
    dh = _scan(on.flip(1), dh.flip(1)).flip(1)
    prior = torch.where(first, before, torch.cat([torch.zeros_like(h[:, :1]), h[:, :-1]], 1))
    dgate = torch.where(inside, dh * (prior - x) * (a * c), 0.0)
    begins = st["starts"][:, :-1].long().unsqueeze(2).expand(n, count, w).clamp(max=t - 1)
    dinitial = torch.where(empty, st["dlast"], torch.gather(dh * a, 1, begins))
    return [h.to(dt), last, dgate.to(dt), (dh * c).to(dt), dinitial]


def _blocknorm(st):
    case, dt, k = st["case"], st["dt"], st["case"]["width"]
    z = st["z"].float()
    post_rstd = torch.rsqrt(z.square().mean(-1) + EPS)
    u = z * post_rstd.unsqueeze(-1) * st["post"].unsqueeze(1)
    if st["gate"] is not None:
        u = u * torch.sigmoid(st["gate"].float())
    s = (st["residual"].float() + u * st["scale"].view(-1, 1, 1)).to(dt)
    f = s.float()
    rstd = torch.rsqrt(f.square().mean(-1) + EPS)
    y = f * rstd.unsqueeze(-1) * st["pre"].unsqueeze(1)
    out = [s, post_rstd, rstd, _values(*_pack(y, 0), k).to(torch.bfloat16)]
    if case["keep"]:
        out.append(_values(*_pack(f, GROUP), k).to(torch.bfloat16))
    return out


def _blocknorm_backward(st):
    dt, k = st["dt"], st["case"]["width"]
    rstd = st["rstd"].unsqueeze(-1)
    sh = _values(st["codes"], st["exps"], k) * rstd
    dy = st["dy"].float()
    st["dpre"].copy_((dy * sh).sum(1))
    u = dy * st["pre"].unsqueeze(1)
    ds = st["dsum"].float() + rstd * (u - sh * (u * sh).mean(-1, keepdim=True))
    post_rstd = st["post_rstd"].unsqueeze(-1)
    zh = st["z"].float() * post_rstd
    branch = ds * st["scale"].view(-1, 1, 1)
    g = torch.sigmoid(st["gate"].float()) if st["gate"] is not None else torch.ones_like(zh)
    un = zh * st["post"].unsqueeze(1)
    st["dscale"].copy_((ds * g * un).sum((1, 2)))
    du = branch * g
    st["dpost"].copy_((du * zh).sum(1))
    v = du * st["post"].unsqueeze(1)
    dz = post_rstd * (v - zh * (v * zh).mean(-1, keepdim=True))
    out = [ds.to(dt), dz.to(dt), st["dpre"], st["dpost"], st["dscale"]]
    if st["gate"] is not None:
        out.append((branch * un * g * torch.sigmoid(-st["gate"].float())).to(dt))
    return out


def _plain(st):
    op = st["case"]["op"]
    if op == "attention":
        return _attention(st)
    if op == "recurrence":
        return _recurrence(st)
    return _blocknorm(st) if op == "blocknorm" else _blocknorm_backward(st)


def _own(st):
    from paper_2110_04175_amd import layer
    case = st["case"]
    op = case["op"]
    if op == "attention":
        t, keys = case["t"], case["keys"]
        # One text of each worker needs no list of who sees what.
        ranges = None
        if case["count"] > 1:
            ranges = layer.attention_ranges(st["starts"], t, st["key_starts"], keys, causal=True)
        out, lse = layer.attention(st["q"], st["k"], st["v"], ranges, causal=True, keep=case["grad"])
        if not case["grad"]:
            return [out]
        return [out, *layer.attention_backward(st["dout"], st["q"], st["k"], st["v"], out, lse, ranges,
                                               causal=True)]
    if op == "recurrence":
        h, last, saved = layer.recurrence(st["gate"], st["x"], st["initial"], st["starts"], keep=case["grad"])
        if not case["grad"]:
            return [h, last]
        return [h, last, *layer.recurrence_backward(st["dh"], st["dlast"], st["gate"], st["x"], saved,
                                                    st["initial"], st["starts"])]
    if op == "blocknorm":
        s, y, post_rstd, rstd, saved = layer.blocknorm(st["z"], st["gate"], st["residual"], st["post"],
                                                       st["scale"], st["pre"], eps=EPS, keep=case["keep"])
        out = [s, post_rstd, rstd, layer.unpack(y, torch.bfloat16)]
        return out + [layer.unpack(saved, torch.bfloat16)] if case["keep"] else out
    saved = layer.Packed(st["codes"], st["exps"], case["width"])
    dz, dgate, ds = layer.blocknorm_backward(st["dy"], st["dsum"], st["z"], st["gate"], saved,
                                             st["post_rstd"], st["rstd"], st["post"], st["scale"],
                                             st["pre"], st["dpost"], st["dscale"], st["dpre"])
    out = [ds, dz, st["dpre"], st["dpost"], st["dscale"]]
    return out if dgate is None else out + [dgate]


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    n, t, w, a = case["n"], case["t"], case["width"], BYTES[case["dtype"]]
    op = case["op"]
    if op == "attention":
        heads, kv, keys, count = (case[i] for i in ("heads", "kv", "keys", "count"))
        # Pairs of a query and a key that it sees; lengths vary by a sixth in the square.
        length = t / count * (7 / 6 if count > 1 else 1)
        pairs = t * (length + 1) / 2 if keys == t else t * (keys - (t - 1) / 2)
        flops = 4 * w * n * heads * pairs
        size = n * w * a * (2 * t * heads + 2 * keys * kv)
        return {"bytes": 2 * size if case["grad"] else size, "flops": 3.5 * flops if case["grad"] else flops}
    if op == "recurrence":
        states = 8 * n * case["count"] * w
        if case["grad"]:
            return {"bytes": 6 * a * n * t * w + 2 * states, "flops": 20 * n * t * w}
        return {"bytes": 3 * a * n * t * w + states, "flops": 8 * n * t * w}
    gates = 1 if case["gated"] else 0
    if op == "blocknorm":
        # z, residual and gate in; the sum and the values held in 8 bits out.
        held = 2 if case["keep"] else 1
        return {"bytes": n * t * w * (a * (3 + gates) + 2 * held) + 8 * n * w + 8 * n * t,
                "flops": 16 * n * t * w}
    return {"bytes": n * t * w * (a * (5 + 2 * gates) + 1) + 16 * n * w + 8 * n * t,
            "flops": 30 * n * t * w}


# ---- in 64 bits ------------------------------------------------------------------


def _exact_attention(st):
    case, wide = st["case"], torch.float64
    n, t, keys, heads, kv, d = (case[i] for i in ("n", "t", "keys", "heads", "kv", "width"))
    grad = case["grad"]
    q, k, v = (st[i].to(wide) for i in ("q", "k", "v"))
    out = torch.zeros(n, t, heads, d, dtype=wide, device=q.device)
    dq = torch.zeros_like(out)
    dk, dv = torch.zeros(n, keys, kv, d, dtype=wide, device=q.device), \
        torch.zeros(n, keys, kv, d, dtype=wide, device=q.device)
    starts, key_starts = st["starts"].tolist(), st["key_starts"].tolist()
    for i in range(n):
        for (b, e), (kb, ke) in zip(zip(starts[i], starts[i][1:]), zip(key_starts[i], key_starts[i][1:])):
            if e <= b or ke <= kb:
                continue
            lq, lk = e - b, ke - kb
            row = torch.arange(lq, device=q.device).unsqueeze(1)
            seen = torch.arange(lk, device=q.device) <= row + (lk - lq)
            some = seen.any(1, keepdim=True)
            for h in range(heads):
                g = h // (heads // kv)
                qs, ks, vs = q[i, b:e, h], k[i, kb:ke, g], v[i, kb:ke, g]
                s = torch.mm(qs, ks.T.contiguous()) / math.sqrt(d)
                s = torch.where(seen, s, -math.inf)
                p = torch.where(some, torch.softmax(torch.where(some, s, 0.0), 1), 0.0)
                out[i, b:e, h] = torch.mm(p, vs)
                if not grad:
                    continue
                do = st["dout"][i, b:e, h].to(wide)
                dv[i, kb:ke, g] += torch.mm(p.T.contiguous(), do)
                dp = torch.mm(do, vs.T.contiguous())
                ds = p * (dp - (p * dp).sum(1, keepdim=True)) / math.sqrt(d)
                dq[i, b:e, h] = torch.mm(ds, ks)
                dk[i, kb:ke, g] += torch.mm(ds.T.contiguous(), qs)
    return [out, dq, dk, dv] if grad else [out]


def _exact_recurrence(st):
    """In blocks of tokens: within one, h_t = sum over s <= t of the product
    of a from s + 1 to t, written out one token at a time."""
    case, wide = st["case"], torch.float64
    n, t, w, count = case["n"], case["t"], case["width"], case["count"]
    gate, x, initial = (st[i].to(wide) for i in ("gate", "x", "initial"))
    starts = st["starts"].tolist()
    begins, ends = {}, {}
    for i in range(n):
        for j in range(count):
            if starts[i][j + 1] > starts[i][j]:
                begins.setdefault(starts[i][j], []).append((i, j))
                ends.setdefault(starts[i][j + 1] - 1, []).append((i, j))
    a = 1 / (1 + torch.exp(-gate))
    c = 1 / (1 + torch.exp(gate))
    behind = torch.tensor([s[-1] for s in starts], device=gate.device)
    live = (torch.arange(t, device=gate.device) < behind.unsqueeze(1)).unsqueeze(2).to(wide)
    h, prior = torch.zeros_like(x), torch.zeros_like(x)
    last = initial.clone()
    state = torch.zeros(n, w, dtype=wide, device=x.device)
    for step in range(t):
        for i, j in begins.get(step, ()):
            state[i] = initial[i, j]
        prior[:, step] = state
        state = (a[:, step] * state + c[:, step] * x[:, step]) * live[:, step]
        h[:, step] = state
        for i, j in ends.get(step, ()):
            last[i, j] = state[i]
    if not case["grad"]:
        return [h, last]
    dh, dlast = st["dh"].to(wide) * live, st["dlast"].to(wide)
    dinitial, back = dlast.clone(), torch.zeros_like(state)
    dstate = torch.zeros_like(x)
    for step in range(t - 1, -1, -1):
        for i, j in ends.get(step, ()):
            back[i] = dlast[i, j]
        d = (back + dh[:, step]) * live[:, step]
        dstate[:, step] = d
        back = a[:, step] * d
        for i, j in begins.get(step, ()):
            dinitial[i, j] = back[i]
            back[i] = 0
    return [h, last, dstate * (prior - x) * a * c, dstate * c, dinitial]


def _exact_held(v, group):
    """What 64-bit rows stand for when they are held in 8 bits."""
    n, rows, width = v.shape
    wide = torch.zeros(n, rows, _stride(width), dtype=v.dtype, device=v.device)
    wide[:, :, :width] = v
    parts = wide.unflatten(2, (-1, group or wide.shape[2]))
    most = parts.abs().amax(3, keepdim=True)
    quantum = torch.exp2(torch.floor(torch.log2(most.clamp(min=2.0 ** -119))) - 6)
    quantum = torch.where(most > 127 * quantum, 2 * quantum, quantum).clamp(min=2.0 ** -126)
    return (torch.round(parts / quantum) * quantum).flatten(2)[:, :, :width]


def exact(case, seed):
    """In 64 bits, what is held in 8 bits too until it is held."""
    st = prepare(case, seed)
    op, k, dt, wide = case["op"], case["width"], st["dt"], torch.float64
    if op == "attention":
        # One product a head of each sequence: thousands of them take too long.
        return None if case["n"] * case["count"] * case["heads"] > 6000 else _exact_attention(st)
    if op == "recurrence":
        # A token at a time.
        return None if case["t"] > 40000 else _exact_recurrence(st)
    z, w = st["z"].to(wide), st["post"].to(wide)[:, None, :]
    gate = 1 / (1 + torch.exp(-st["gate"].to(wide))) if case["gated"] else torch.ones_like(z)
    scale = st["scale"].to(wide)[:, None, None]
    if op == "blocknorm":
        rms = torch.sqrt((z * z).sum(2) / k + EPS)
        full = st["residual"].to(wide) + scale * gate * (z / rms[:, :, None] * w)
        s = full.to(dt).to(wide)
        rms_s = torch.sqrt((s * s).sum(2) / k + EPS)
        y = s / rms_s[:, :, None] * st["pre"].to(wide)[:, None, :]
        held = [_exact_held(y, 0)] + ([_exact_held(s, GROUP)] if case["keep"] else [])
        return [full, 1.0 / rms, 1.0 / rms_s, *held]
    # The Jacobian of v -> v / rms(v) at the kept rms, applied to a gradient.
    def through(dv, unit, inv):
        return inv * dv - inv * unit * ((dv * unit).sum(2, keepdim=True) / k)

    q, e = st["codes"], st["exps"]
    size = torch.pow(torch.tensor(2.0, dtype=wide, device=q.device), e.to(wide))
    s = (q.to(wide) * size.repeat_interleave(q.shape[2] // e.shape[2], dim=2))[:, :, :k]
    inv, post_inv = st["rstd"].to(wide)[:, :, None], st["post_rstd"].to(wide)[:, :, None]
    sh, zh, dy = s * inv, z * post_inv, st["dy"].to(wide)
    ds = st["dsum"].to(wide) + through(dy * st["pre"].to(wide)[:, None, :], sh, inv)
    dz = through(ds * scale * gate * w, zh, post_inv)
    out = [ds, dz, (dy * sh).sum(1), (ds * scale * gate * zh).sum(1), (ds * gate * zh * w).sum((1, 2))]
    if case["gated"]:
        out.append(ds * scale * zh * w * gate * (1 - gate))
    return out
