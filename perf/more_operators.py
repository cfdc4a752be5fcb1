"""Timed cases of what a sequence model does with the positions and heads of its tokens: linear attention whose memory of
earlier tokens fades at a rate of each head's own, and a learned bias of the distance between two tokens.

  attend       outputs of linear attention with a decay for each head, over whole prompts: one sequence, batches or packed
               sequences; with the memory a sequence begins with and the one it ends with where asked for
  attend_grad  its backward pass: gradients of queries, keys and values
  step         one new token of each running request: its memory is brought up to date and read
  bias         a bias for every pair of tokens and every head, looked up by buckets of their distance on each axis
  bias_grad    its backward pass: the gradient of the learned table

A case names an operator, its sizes and types:

  b, s             sequences of s tokens each, or (packed) b sequences of different lengths that hold s tokens on average
  hq, hk           heads of queries, and of keys and values
  dk, dv           size of a head of queries and keys, and of values
  state            the memory before is given and the one after is asked for
  slots            memories that the running requests' are among
  nq, nk           tokens across which a bias is laid; `grid`: patches of an image with rows and columns as axes, otherwise text
  axes, buckets    axes of the positions, buckets of a distance
  far              distances from here on share a bucket
  packed           several sequences side by side: pairs of tokens of two of them are masked
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"f16": 2, "bf16": 2, "f32": 4}
DEVICE = "cuda:0"
LARGEST = 32768 * 32 * 256           # elements of queries and values of the largest prompt
LARGEST_GRAD = 16384 * 16 * 256


def _attend(name, op, b, s, hq, hk, dk, dv, dtype, packed=False, state=False):
    return {"name": name, "op": op, "b": b, "s": s, "hq": hq, "hk": hk, "dk": dk, "dv": dv, "dtype": dtype, "packed": packed, "state": state}


def _step(name, b, hq, hk, dk, dv, dtype, slots):
    return {"name": name, "op": "step", "b": b, "hq": hq, "hk": hk, "dk": dk, "dv": dv, "dtype": dtype, "slots": slots}


def _bias(name, op, b, nq, nk, heads, axes, buckets, far, dtype, grid=False, packed=False):
    return {"name": name, "op": op, "b": b, "nq": nq, "nk": nk, "heads": heads, "axes": axes, "buckets": buckets, "far": far, "dtype": dtype,
            "grid": grid, "packed": packed}


def listed():
    return [
        # a few short prompts, packed: launch latency
        _attend("attend_short_4", "attend", 4, 61, 8, 8, 64, 64, "bf16", packed=True),
        # the patch tokens of a batch of images, an image a sequence, heads of 72
        _attend("attend_images_96_f16", "attend", 96, 729, 16, 16, 72, 72, "f16", packed=True),
        # a short batch in single precision that goes on from an earlier part and is gone on from
        _attend("attend_state_f32", "attend", 3, 1001, 12, 12, 64, 64, "f32", state=True),
        # a long prompt; the largest
        _attend("attend_prompt_32768", "attend", 1, 32768, 32, 32, 128, 128, "bf16", state=True),
        # a short training batch whose query heads share keys and values, in single precision
        _attend("attend_grad_257_f32", "attend_grad", 2, 257, 8, 2, 64, 64, "f32"),
        # a training batch
        _attend("attend_grad_16384", "attend_grad", 4, 4096, 16, 16, 128, 128, "bf16"),
        # a single request's new token
        _step("step_1", 1, 16, 16, 64, 64, "bf16", 1),
        # a new token of each running request; their memories are among many
        _step("step_200", 200, 32, 8, 128, 128, "bf16", 256),
        # one new token's row of biases before a long context
        _bias("bias_row_32768", "bias", 1, 1, 32768, 32, 1, 32, 128, "bf16"),
        # an image encoder's patches, rows and columns; an odd number of tokens
        _bias("bias_images_f16", "bias", 8, 729, 729, 16, 2, 32, 64, "f16", grid=True),
        # packed images of single precision: rows, columns and time
        _bias("bias_grad_packed_f32", "bias_grad", 1, 1001, 1001, 8, 3, 16, 32, "f32", grid=True, packed=True),
        # a training batch of text whose sequences share their positions
        _bias("bias_grad_4096", "bias_grad", 2, 4096, 4096, 16, 1, 32, 128, "bf16"),
    ]


def draw(rng: random.Random):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["attend", "attend", "attend_grad", "attend_grad", "step", "bias", "bias_grad"])
    dtype = rng.choice(["f16", "bf16", "bf16", "f32"])
    if op in ("attend", "attend_grad", "step"):
        dk = rng.choice([16, 32, 48, 64, 64, 72, 80, 96, 128, 128])
        dv = dk if rng.random() < 0.7 else rng.choice([32, 64, 128])
        hk = rng.choice([1, 2, 4, 8, 8, 16])
        hq = hk * (1 if rng.random() < 0.7 else rng.choice([2, 3, 4]))
        if op == "step":
            most = 256 * 32 * 128 * 128 // (hq * dk * dv)
            b = spread(1, min(256, most))
            c = _step("", b, hq, hk, dk, dv, dtype, b + rng.randint(0, 64))
        else:
            most = (LARGEST if op == "attend" else LARGEST_GRAD) // (hq * (dk + dv)) // (4 if dtype == "f32" else 1)
            s = spread(1, min(32768, most))
            b = spread(1, max(1, min(128, most // s)))
            c = _attend("", op, b, s, hq, hk, dk, dv, dtype, packed=b > 1 and rng.random() < 0.5, state=op == "attend" and rng.random() < 0.4)
    else:
        axes, grid = rng.choice([(1, False), (1, False), (2, True), (3, True)])
        heads = rng.choice([1, 4, 8, 12, 16, 16, 32])
        far = rng.choice([16, 32, 64, 128, 128, 256])
        most = 2 * 4096 * 4096 * 16 // heads // (2 if dtype == "f32" else 1)
        nk = spread(16, 4096)
        nq = nk if op == "bias_grad" or rng.random() < 0.7 else 1
        c = _bias("", op, spread(1, max(1, min(32, most // (nq * nk)))), nq, nk, heads, axes, rng.choice([16, 32, 32, 64]), far, dtype,
                  grid=grid, packed=grid and nq > 1 and rng.random() < 0.5)
    del c["name"]
    return c


# ---- sizes that belong to a case --------------------------------------------------------------------------------------


def _lengths(case):
    """Tokens of each sequence: their sum belongs to the case."""
    if not case["packed"]:
        return [case["s"]] * case["b"]
    rng, b, total = random.Random(7 * case["b"] + case["s"]), case["b"], case["b"] * case["s"]
    share = [math.exp(rng.gauss(0.0, 0.5)) for _ in range(b)]
    got = [max(1, int(total * x / sum(share))) for x in share]
    got[0] += max(0, total - sum(got))
    return got


def _buckets(n, far):
    """Bucket of the distances -far .. far (and all beyond): half of the n for either direction, half of those for single
    distances, the others for distances that grow by a factor."""
    half = n // 2
    single = half // 2
    got = []
    for d in range(-far, far + 1):
        a = abs(d)
        b = a if a < single else min(half - 1, single + int(math.log(a / single) / math.log(far / single) * (half - single) + 1e-9))
        got.append(b + (half if d > 0 else 0))
    return got


def _positions(case, rng):
    """Positions (axes, nk) of the keys' tokens and, where they are packed, whose sequence each is of."""
    n, axes = case["nk"], case["axes"]
    if not case["grid"]:
        return [list(range(n))] * axes, None
    rows, ids, seq = [[] for _ in range(axes)], [], 0
    while len(ids) < n:
        w = max(2, math.isqrt(n)) if not case["packed"] else rng.randint(6, 24)
        h = -(-n // w) if not case["packed"] else rng.randint(6, 24)
        for i in range(h * w):
            place = (i // w, i % w, seq)
            for a in range(axes):
                rows[a].append(place[a])
            ids.append(seq)
        seq += 1
    return [r[:n] for r in rows], ids[:n] if case["packed"] else None


# ---- inputs -----------------------------------------------------------------------------------------------------------


class _State:
    pass


def prepare(case, seed):
    s = _State()
    s.case = case
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    dtype = DTYPES[case["dtype"]]

    def randn(*shape, to=dtype):
        return torch.randn(*shape, device=DEVICE, generator=gen).to(to)

    if case["op"] in ("bias", "bias_grad"):
        n = case["buckets"]
        s.buckets = torch.tensor(_buckets(n, case["far"]), dtype=torch.int32, device=DEVICE)
        rows, ids = _positions(case, random.Random(case["nk"]))
        keys = torch.tensor(rows, dtype=torch.int32, device=DEVICE) + seed % 1000
        s.ids = None if ids is None else torch.tensor(ids, dtype=torch.int32, device=DEVICE)
        s.qpos = keys[:, case["nk"] - case["nq"]:]
        s.kpos = keys
        if case["op"] == "bias":
            s.table = randn(case["axes"], n, case["heads"])
            if case["b"] > 1:                                    # every image counts from a place of its own
                begin = torch.randint(0, 1000, (case["axes"], case["b"], 1), device=DEVICE, generator=gen, dtype=torch.int32)
                s.qpos, s.kpos = s.qpos[:, None] + begin, s.kpos[:, None] + begin
                s.ids = None if s.ids is None else s.ids.expand(case["b"], -1)
        else:
            s.grad = randn(case["b"], case["heads"], case["nq"], case["nk"])
        return s
    hq, hk, dk, dv = case["hq"], case["hk"], case["dk"], case["dv"]
    # rates from the fastest head's, about two tokens, to the slowest's, some hundred
    s.log_decay = -torch.exp2(-8.0 * torch.arange(1, hq + 1, device=DEVICE, dtype=torch.float32) / hq) * (0.9 + 0.2 * (seed % 97) / 97)
    if case["op"] == "step":
        b, n = case["b"], case["slots"]
        s.q, s.k, s.v = randn(b, hq, dk) * dk ** -0.5, randn(b, hk, dk), randn(b, hk, dv)
        s.memory = randn(n, hq, dk, dv, to=torch.float32)
        s.slots = torch.randperm(n, device=DEVICE, generator=gen)[:b].to(torch.int32)
        return s
    lengths = _lengths(case)
    shape = (sum(lengths),) if case["packed"] else (case["b"], case["s"])
    s.starts = None
    s.lengths = lengths
    if case["packed"]:
        at = [0]
        for n in lengths:
            at.append(at[-1] + n)
        s.starts = torch.tensor(at, dtype=torch.int32, device=DEVICE)
    s.q, s.k, s.v = randn(*shape, hq, dk) * dk ** -0.5, randn(*shape, hk, dk), randn(*shape, hk, dv)
    s.memory = randn(len(lengths), hq, dk, dv, to=torch.float32) if case["state"] else None
    s.g = randn(*shape, hq, dv) if case["op"] == "attend_grad" else None
    return s


# ---- plain forms ------------------------------------------------------------------------------------------------------


def _spread_out(x, s):
    """(sequences, tokens, ...) in 32 bits, zeros behind a packed sequence's last token."""
    if s.starts is None:
        return x.float()
    longest = max(s.lengths)
    at = s.starts[:-1, None].long() + torch.arange(longest, device=x.device)
    inside = at < s.starts[1:, None]
    return x.float()[at.clamp(max=x.shape[0] - 1)] * inside.view(*inside.shape, *(1,) * (x.dim() - 1))


def _together(x, s):
    if s.starts is None:
        return x
    inside = torch.arange(max(s.lengths), device=x.device) < (s.starts[1:, None] - s.starts[:-1, None])
    return x[inside]


def _walk(a, b, c, log_decay, memory=None, lengths=None, block=128):
    """Sum over j <= t of exp(log_decay (t - j)) (a_t . b_j) c_j, block by block: within a block as a product of matrices, from the
    blocks before through the memory they left, which rests behind a sequence's end.  All (n, tokens, heads, size)."""
    n, tokens, heads, _ = a.shape
    out = a.new_empty(n, tokens, heads, c.shape[-1])
    memory = a.new_zeros(n, heads, b.shape[-1], c.shape[-1]) if memory is None else memory
    i = torch.arange(min(block, tokens), device=a.device, dtype=torch.float32)
    fade = torch.where(i[:, None] >= i, torch.exp(log_decay[:, None, None] * (i[:, None] - i).clamp(min=0)), 0.0)
    for at in range(0, tokens, block):
        m = min(block, tokens - at)
        x, y, z = (v[:, at:at + m].transpose(1, 2) for v in (a, b, c))
        age = torch.exp(log_decay[:, None] * (i[:m] + 1))[..., None]
        got = (x @ y.transpose(-1, -2) * fade[:, :m, :m]) @ z + (x @ memory) * age
        out[:, at:at + m] = got.transpose(1, 2)
        steps = torch.full((n,), m, device=a.device) if lengths is None else (lengths - at).clamp(0, m)
        left = torch.exp(log_decay[:, None] * (steps[:, None, None] - 1 - i[:m]).clamp(min=0))[..., None]
        memory = memory * torch.exp(log_decay * steps[:, None])[..., None, None] + (y * left).transpose(-1, -2) @ z
    return out, memory


def _plain_attend(s):
    q, k, v = (_spread_out(x, s) for x in (s.q, s.k, s.v))
    k, v = (x.repeat_interleave(s.case["hq"] // s.case["hk"], 2) for x in (k, v))
    out, memory = _walk(q, k, v, s.log_decay, s.memory, None if s.starts is None else s.starts.diff())
    out = _together(out, s).to(s.v.dtype)
    return {"out": out, "state": memory} if s.case["state"] else {"out": out}


def _plain_attend_grad(s):
    group = s.case["hq"] // s.case["hk"]
    q, k, v, g = (_spread_out(x, s) for x in (s.q, s.k, s.v, s.g))
    k, v = (x.repeat_interleave(group, 2) for x in (k, v))

    def later(a, b, c):                                          # the same sum over j >= t; shared heads' gradients added up
        x = _walk(a.flip(1), b.flip(1), c.flip(1), s.log_decay)[0].flip(1)
        return x.unflatten(2, (-1, group)).sum(3)

    dq, dk, dv = _walk(g, v, k, s.log_decay)[0], later(v, g, q), later(k, q, g)
    return {n: _together(x, s).to(s.q.dtype) for n, x in (("dq", dq), ("dk", dk), ("dv", dv))}


def _plain_step(s):
    group, slots = s.case["hq"] // s.case["hk"], s.slots.long()
    k, v = (x.float().repeat_interleave(group, 1) for x in (s.k, s.v))
    now = s.memory[slots] * torch.exp(s.log_decay)[:, None, None] + k[..., None] * v[..., None, :]
    s.memory[slots] = now
    return {"out": (s.q.float()[..., None] * now).sum(-2).to(s.v.dtype), "state": s.memory}


def _plain_bias(s):
    far = s.case["far"]
    got = 0
    for a in range(s.case["axes"]):
        d = (s.kpos[a][..., None, :].long() - s.qpos[a][..., :, None].long()).clamp(-far, far) + far
        got = got + s.table[a].float()[s.buckets[d].long()]      # (..., nq, nk, heads)
    got = got.movedim(-1, -3)
    if s.ids is not None:
        got = got.masked_fill((s.ids[..., None, :] != s.ids[..., :, None]).unsqueeze(-3), -math.inf)
    return got.to(s.table.dtype).contiguous()


def _plain_bias_grad(s):
    c, far = s.case, s.case["far"]
    got = s.grad.new_zeros(c["axes"], c["buckets"], c["heads"], dtype=torch.float64)
    for h in range(c["heads"]):                                  # one head after the other: long sums, in 64 bits
        g = s.grad[:, h].double().sum(0)
        if s.ids is not None:
            g = g.masked_fill(s.ids[:, None] != s.ids, 0.0)
        for a in range(c["axes"]):
            d = (s.kpos[a][None].long() - s.qpos[a][:, None].long()).clamp(-far, far) + far
            by_distance = g.new_zeros(2 * far + 1).index_add_(0, d.flatten(), g.flatten())
            got[a, :, h].index_add_(0, s.buckets.long(), by_distance)
    return got.float()


# ---- the framework's operators ----------------------------------------------------------------------------------------


def _own(s):
    import paper_1911_00472_b200 as P
    c = s.case
    if c["op"] == "attend":
        out, state = P.decay_attention(s.q, s.k, s.v, s.log_decay, starts=s.starts, state=s.memory, final=c["state"])
        return {"out": out, "state": state} if c["state"] else {"out": out}
    if c["op"] == "attend_grad":
        dq, dk, dv, _ = P.decay_attention_backward(s.g, s.q, s.k, s.v, s.log_decay, starts=s.starts)
        return {"dq": dq, "dk": dk, "dv": dv}
    if c["op"] == "step":
        return {"out": P.decay_step(s.q, s.k, s.v, s.log_decay, s.memory, slots=s.slots), "state": s.memory}
    if c["op"] == "bias":
        return P.relative_bias(s.table, s.buckets, s.qpos, s.kpos, q_ids=s.ids, k_ids=s.ids)
    return P.relative_bias_backward(s.grad, c["buckets"], s.buckets, s.qpos, s.kpos, q_ids=s.ids, k_ids=s.ids)


def run(s):
    if own:
        return _own(s)
    return {"attend": _plain_attend, "attend_grad": _plain_attend_grad, "step": _plain_step, "bias": _plain_bias, "bias_grad": _plain_bias_grad}[s.case["op"]](s)


# ---- work and definition ----------------------------------------------------------------------------------------------


def work(case):
    """Each input read once, each output written once; attention as the recurrence has it: a product into the memory and one out of it."""
    size = BYTES[case["dtype"]]
    if case["op"] in ("bias", "bias_grad"):
        values = float(case["b"] * case["heads"] * case["nq"] * case["nk"])
        table = case["axes"] * case["buckets"] * case["heads"] * (size if case["op"] == "bias" else 4)
        places = 4.0 * case["axes"] * (case["nq"] + case["nk"]) * (case["b"] if case["op"] == "bias" else 1)
        return {"bytes": values * size + table + places, "flops": values * case["axes"]}
    hq, hk, dk, dv = case["hq"], case["hk"], case["dk"], case["dv"]
    tokens = case["b"] if case["op"] == "step" else sum(_lengths(case))
    memory = 4.0 * hq * dk * dv
    inputs, outputs = hq * dk + hk * dk + hk * dv, hq * dv
    flops = 4.0 * tokens * hq * dk * dv
    if case["op"] == "step":
        return {"bytes": tokens * (inputs + outputs) * size + 2.0 * tokens * memory, "flops": flops}
    if case["op"] == "attend":
        return {"bytes": float(tokens * (inputs + outputs) * size) + (2.0 * case["b"] * memory if case["state"] else 0.0), "flops": flops}
    return {"bytes": float(tokens * (2 * inputs + outputs) * size), "flops": 2.5 * flops}


def _weights(rate, at, to, tokens, device):
    """exp(rate (t - j)) for t in at .. to, j in 0 .. to, 0 where j > t."""
    d = torch.arange(at, to, device=device, dtype=torch.float64)[:, None] - torch.arange(to, device=device, dtype=torch.float64)
    return torch.where(d >= 0, torch.exp(rate * d.clamp(min=0)), torch.zeros((), device=device, dtype=torch.float64))


def _exact_attend(s):
    """Sequence by sequence and head by head, every pair of tokens."""
    c, group = s.case, s.case["hq"] // s.case["hk"]
    q, k, v = (x.flatten(0, -3) for x in (s.q, s.k, s.v))
    grad = c["op"] == "attend_grad"
    got = {n: torch.zeros_like(x, dtype=torch.float64) for n, x in ((("dq", q), ("dk", k), ("dv", v)) if grad else ())}
    if not grad:
        got["out"] = torch.empty(*q.shape[:-1], c["dv"], device=q.device, dtype=torch.float64)
        if c["state"]:
            got["state"] = torch.empty_like(s.memory, dtype=torch.float64)
    g = s.g.flatten(0, -3) if grad else None
    begin = 0
    for i, n in enumerate(s.lengths):
        end = begin + n
        for h in range(c["hq"]):
            rate = s.log_decay[h].double()
            x, y, z = q[begin:end, h].double(), k[begin:end, h // group].double(), v[begin:end, h // group].double()
            for at in range(0, n, 4096):
                to = min(n, at + 4096)
                w = _weights(rate, at, to, n, q.device)
                if grad:
                    o = g[begin + at:begin + to, h].double()
                    pair = (o @ z[:to].T) * w
                    got["dq"][begin + at:begin + to, h] = pair @ y[:to]
                    got["dk"][begin:begin + to, h // group] += pair.T @ x[at:to]
                    got["dv"][begin:begin + to, h // group] += ((x[at:to] @ y[:to].T) * w).T @ o
                else:
                    out = ((x[at:to] @ y[:to].T) * w) @ z[:to]
                    if c["state"]:
                        out += (x[at:to] @ s.memory[i, h].double()) * torch.exp(rate * torch.arange(at + 1, to + 1, device=q.device, dtype=torch.float64))[:, None]
                    got["out"][begin + at:begin + to, h] = out
            if c["state"]:
                left = torch.exp(rate * torch.arange(n - 1, -1, -1, device=q.device, dtype=torch.float64))[:, None]
                got["state"][i, h] = (y * left).T @ z + s.memory[i, h].double() * torch.exp(rate * n)
        begin = end
    like = {"dq": s.q, "dk": s.k, "dv": s.v}
    return {n: x if n == "state" else x.view(*(like.get(n, s.q)).shape[:-1], x.shape[-1]) for n, x in got.items()}


def _exact_step(s):
    group = s.case["hq"] // s.case["hk"]
    after, out = s.memory.double(), torch.empty(*s.q.shape[:-1], s.case["dv"], device=s.q.device, dtype=torch.float64)
    for i, slot in enumerate(s.slots.tolist()):
        for h in range(s.case["hq"]):
            after[slot, h] = after[slot, h] * math.exp(float(s.log_decay[h])) + torch.outer(s.k[i, h // group].double(), s.v[i, h // group].double())
            out[i, h] = s.q[i, h].double() @ after[slot, h]
    return {"out": out, "state": after}


def _distances(s, a, batch):
    """Buckets of all pairs on an axis, distance by distance from the ends."""
    kpos, qpos = (p[a] if p.dim() == 2 else p[a, batch] for p in (s.kpos, s.qpos))
    d = kpos.double()[None, :] - qpos.double()[:, None]
    far = s.case["far"]
    return s.buckets[torch.where(d < -far, -far, torch.where(d > far, far, d)).long() + far].long()


def _exact_bias(s):
    c = s.case
    got = []
    for batch in range(c["b"]):
        one = torch.zeros(c["heads"], c["nq"], c["nk"], device=DEVICE, dtype=torch.float64)
        for a in range(c["axes"]):
            bucket = _distances(s, a, batch)
            for h in range(c["heads"]):
                one[h] += s.table[a, :, h].double()[bucket]
        if s.ids is not None:
            ids = s.ids if s.ids.dim() == 1 else s.ids[batch]
            one[:, ids[:, None] != ids[None, :]] = -math.inf
        got.append(one)
    return torch.stack(got) if s.qpos.dim() == 3 else got[0]


def _exact_bias_grad(s):
    c = s.case
    g = s.grad.sum(0, dtype=torch.float64)
    if s.ids is not None:
        g = g * (s.ids[:, None] == s.ids[None, :])
    got = torch.zeros(c["axes"], c["buckets"], c["heads"], device=DEVICE, dtype=torch.float64)
    for a in range(c["axes"]):
        bucket = _distances(s, a, 0)
        for n in range(c["buckets"]):
            got[a, n] = (g * (bucket == n)).sum((-1, -2))
    return got


def exact(case, seed):
    s = prepare(case, seed)
    return {"attend": _exact_attend, "attend_grad": _exact_attend, "step": _exact_step, "bias": _exact_bias, "bias_grad": _exact_bias_grad}[case["op"]](s)
