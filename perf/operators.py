"""The operators a text-conditioned next-scale transformer needs beside the cache and its self-attention, as one pass each:
rotary positions of Q and K, appending to and attending over a cache held in 8 bits, and cross attention to an encoder's
states.

`own` false: the operators in plain torch, 32 bits inside; true: the library's calls.

A case is a dict of plain values; `op` names the operator:
  rotary   Q [rows, heads, T, head_dim] and K [rows, kv_heads, T, head_dim] rotated by a table of cosines and sines
  table    that table, from positions
  cross    queries of a scale of `side` x `side` tokens over each row's own encoder states: `keys` of them at most, `ragged`
           lengths, `packed` one behind the other or padded to the same length
  pass     one layer's whole schedule, appended to and attended over a cache held in 8 bits
  attend   the last scale's queries over such a cache
  store    a scale appended to such a cache and read back
"""
import math

import torch

own = False

S256 = "1,2,3,4,5,6,8,10,13,16"
S512 = "1,2,3,4,6,9,13,18,24,32"
S1024 = "1,2,4,6,8,12,16,20,24,32,40,48,64"

_ROTARY = {"op": "rotary", "rows": 2, "heads": 16, "kv_heads": 16, "head_dim": 64, "T": 1, "rotary_dim": 64, "axes": 1,
           "layout": "half", "scaling": "plain", "factor": 1.0, "base": 10000.0, "original": 0.0, "first": 0, "index": False,
           "views": False, "transposed": False}
_TABLE = {"op": "table", "count": 1, "rotary_dim": 64, "axes": 1, "scaling": "plain", "factor": 1.0, "base": 10000.0,
          "original": 0.0}
_CROSS = {"op": "cross", "rows": 2, "heads": 16, "kv_heads": 16, "head_dim": 128, "side": 1, "keys": 77, "ragged": True,
          "packed": False, "views": False}
_CACHE = {"op": "attend", "rows": 2, "heads": 16, "head_dim": 64, "sides": S256, "condensed": 2, "local": 2, "demanding": False}


def listed():
    return [
        # the first token of one image, guidance doubled: latency is all there is
        dict(_ROTARY, name="rotary_token"),
        # gradients of part of the head, in a batch of odd-sided scales taken out of one projection, every row with positions of
        # its own and some tokens without one, frequencies scaled by parts for four times the length
        dict(_ROTARY, name="rotary_part", rows=128, heads=30, kv_heads=30, T=169, rotary_dim=48, layout="interleaved",
             scaling="parts", factor=4.0, original=680.0, index=True, views=True, transposed=True),
        # the last scale of eight 1024 x 1024 images, rows and columns as two axes, from views of one projection
        dict(_ROTARY, name="rotary_last_scale", rows=16, head_dim=128, rotary_dim=128, T=4096, axes=2, first=6425, views=True),
        # a table for a long context, its base scaled: made once for a model
        dict(_TABLE, name="table_long", count=131071, rotary_dim=128, scaling="base", factor=16.0),
        # the first token of one image over its prompt and the empty prompt of guidance
        dict(_CROSS, name="cross_token"),
        # a coarse scale of eight images, four query heads to each head of the encoder's states, packed prompts
        dict(_CROSS, name="cross_coarse", rows=16, kv_heads=4, side=6, keys=512, packed=True),
        # a class-conditional batch's last scale over padded states of 64 images
        dict(_CROSS, name="cross_batch", rows=128, heads=30, kv_heads=30, head_dim=64, side=16, keys=133),
        # the last scale of eight 1024 x 1024 images over packed prompts, views of one projection
        dict(_CROSS, name="cross_last_scale", rows=16, side=64, keys=512, packed=True, views=True),
        # one layer of one image, every scale: interactive generation
        dict(_CACHE, name="cache_image", op="pass"),
        # the last scale of a serving batch of 64 images in a cache-efficient layer
        dict(_CACHE, name="cache_batch", rows=128, heads=30),
        # the last scale of two 1024 x 1024 images in a cache-demanding layer: 10 521 keys
        dict(_CACHE, name="cache_last_scale", rows=4, head_dim=128, sides=S1024, demanding=True),
        # a large scale of eight images into the cache, and out of it again
        dict(_CACHE, name="cache_store", op="store", rows=16, head_dim=128, sides="32"),
    ]


# ---------------------------------------------------------------- drawn cases
def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_sides(rng, last):
    s, growth = [1], rng.uniform(1.2, 1.8)
    while s[-1] < last and len(s) < 16:
        s.append(min(last, max(s[-1] + 1, int(s[-1] * growth * rng.uniform(0.9, 1.1)))))
    return ",".join(str(x) for x in s)


def _heads(rng):
    kv = rng.choice([1, 2, 4, 5, 8, 10, 16])
    return kv, kv * rng.choice([1, 1, 2, 3, 4])


def _draw_once(rng):
    op = rng.choice(["rotary", "rotary", "table", "cross", "cross", "cross", "pass", "attend", "attend", "store"])
    head_dim = rng.choice([64, 128])
    if op == "table":
        axes = rng.choice([1, 2])
        return dict(_TABLE, count=_log_int(rng, 1, 131071), axes=axes, rotary_dim=4 * axes * rng.randint(1, 32 // axes),
                    scaling=rng.choice(["plain", "linear", "base", "parts"]), factor=rng.choice([1.0, 2.0, 3.5, 8.0]),
                    base=rng.choice([10000.0, 500000.0]), original=4096.0)
    if op == "rotary":
        kv, heads = _heads(rng)
        axes = rng.choice([1, 2])
        return dict(_ROTARY, rows=_log_int(rng, 1, 128), heads=heads, kv_heads=kv, head_dim=head_dim, T=_log_int(rng, 1, 4096),
                    rotary_dim=rng.choice([head_dim, head_dim, 4 * axes * rng.randint(1, head_dim // 4 // axes)]), axes=axes,
                    layout=rng.choice(["half", "interleaved"]), scaling=rng.choice(["plain", "linear", "base", "parts"]),
                    factor=rng.choice([1.0, 2.0, 3.5, 8.0]), original=4096.0, first=_log_int(rng, 1, 100000) - 1,
                    index=rng.random() < 0.3, views=rng.random() < 0.5, transposed=rng.random() < 0.3)
    if op == "cross":
        kv, heads = _heads(rng)
        return dict(_CROSS, rows=_log_int(rng, 1, 128), heads=heads, kv_heads=kv, head_dim=head_dim, side=_log_int(rng, 1, 64),
                    keys=_log_int(rng, 1, 1100), ragged=rng.random() < 0.8, packed=rng.random() < 0.5, views=rng.random() < 0.5)
    sides = rng.choice([S256, S512 if head_dim == 64 else S1024, _draw_sides(rng, _log_int(rng, 4, 48))])
    if op == "store":
        sides = str(_log_int(rng, 1, 64))
    return dict(_CACHE, op=op, rows=_log_int(rng, 1, 128), heads=rng.choice([1, 4, 8, 15, 16, 30]), head_dim=head_dim, sides=sides,
                condensed=rng.randint(0, 3), local=rng.randint(1, 3), demanding=rng.random() < 0.4)


def _state_bytes(case):
    if case["op"] in ("rotary", "table"):
        return work(case)["bytes"]
    if case["op"] == "cross":
        t = case["side"] ** 2
        return case["rows"] * case["head_dim"] * (4 * case["heads"] * t + 4 * case["kv_heads"] * case["keys"])
    return sum(s * s for s in _sides(case)) * case["rows"] * case["heads"] * case["head_dim"] * 12


def draw(rng):
    top = [work(c) for c in listed()]
    max_bytes, max_flops = max(w["bytes"] for w in top), max(w["flops"] for w in top)
    while True:
        c = _draw_once(rng)
        while True:
            w = work(c)
            if w["bytes"] <= max_bytes and w["flops"] <= max_flops and _state_bytes(c) <= 4e9:
                return c
            if c.get("rows", 1) == 1:
                break
            c["rows"] = max(1, c["rows"] * 2 // 3)


# ---------------------------------------------------------------- what a case is
def _sides(case):
    return [int(s) for s in case["sides"].split(",")]


def _kept(case, k):
    """Scales the queries of scale k attend to."""
    if case["demanding"]:
        return list(range(k + 1))
    return [s for s in range(k + 1) if s < case["condensed"] or s > k - case["local"]]


def _lengths(case):
    """Keys of each row: from none to all of them, the first row with all, and (guidance) the second half short."""
    rows, keys = case["rows"], case["keys"]
    if not case["ragged"]:
        return [keys] * rows
    out = []
    for r in range(rows):
        if r == 0:
            out.append(keys)
        elif r >= (rows + 1) // 2 and r % 4 != 3:
            out.append(min(keys, 1 + r % 3))
        else:
            out.append((keys * ((r * 37) % 64) + 32) // 64)
    return out


def work(case):
    """Inputs read once, outputs written once; flops of the two products over the keys that are attended."""
    op = case["op"]
    if op == "table":
        n = case["count"]
        return {"bytes": n * (4 * case["axes"] + 4 * case["rotary_dim"]), "flops": 2 * n * case["rotary_dim"]}
    if op == "rotary":
        values = case["rows"] * (case["heads"] + case["kv_heads"]) * case["T"]
        nbytes = values * case["head_dim"] * 4 + case["T"] * case["rotary_dim"] * 4 * (case["rows"] if case["index"] else 1)
        return {"bytes": nbytes + (4 * case["rows"] * case["T"] if case["index"] else 0), "flops": 3 * values * case["rotary_dim"]}
    d, rows, heads = case["head_dim"], case["rows"], case["heads"]
    if op == "cross":
        t, keys = case["side"] ** 2, sum(_lengths(case))
        return {"bytes": 4 * rows * heads * t * d + 4 * case["kv_heads"] * keys * d, "flops": 4 * heads * t * keys * d}
    tok = [s * s for s in _sides(case)]
    per = rows * heads * d
    held = [per * (2 * t) + rows * heads * 2 * ((t + 15) // 16) for t in tok]   # codes and scales of a scale
    if op == "store":
        return {"bytes": 4 * per * tok[-1] * 2 + 2 * held[-1], "flops": 6 * per * tok[-1]}
    nbytes = flops = 0
    for k, t in enumerate(tok):
        if op == "attend" and k < len(tok) - 1:
            continue
        keys = _kept(case, k)
        nbytes += 4 * per * t + sum(held[s] for s in keys)
        flops += 4 * per * t * sum(tok[s] for s in keys)
        if op == "pass":
            nbytes += 4 * per * t   # K and V of the scale; their codes are written once and counted as read above
    return {"bytes": nbytes, "flops": flops}


# ---------------------------------------------------------------- inputs
class _State:
    pass


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, *shape):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, 1.0, generator=g)


def _bf16(g, *shape):
    return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0.0, 1.0, generator=g)


def _positions(count, axes, first):
    """One axis: token numbers.  Two: rows and columns of the finest grid, scaled, so fractions."""
    n = torch.arange(count, dtype=torch.float64, device="cuda") + first
    if axes == 1:
        return n.float()[:, None].contiguous()
    side = max(1, math.isqrt(count - 1) + 1)
    y, x = torch.div(n - first, side, rounding_mode="floor"), torch.remainder(n - first, side)
    return (torch.stack([y, x], 1) * (64.0 / side)).float().contiguous()


def _frequencies(case):
    """Per axis, in 64 bits, and the amplitude of the table."""
    p = case["rotary_dim"] // case["axes"]
    i = torch.arange(p // 2, dtype=torch.float64, device="cuda")
    base, f, scaling = case["base"], case["factor"], case["scaling"]
    if scaling == "base":
        base = base * f ** (p / (p - 2.0))
    inv = torch.pow(torch.tensor(base, dtype=torch.float64, device="cuda"), -2.0 * i / p)
    if scaling == "linear":
        inv = inv / f
    if scaling != "parts":
        return inv, 1.0

    def at(beta):
        return p * math.log(case["original"] / (2.0 * math.pi * beta)) / (2.0 * math.log(case["base"]))

    lo, hi = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), p - 1)
    ramp = torch.clamp((i - lo) / (hi - lo if hi > lo else 1e-3), 0.0, 1.0)
    return inv * (1.0 - ramp) + inv / f * ramp, 0.1 * math.log(f) + 1.0


def _plain_table(case, positions):
    inv, amp = _frequencies(case)
    angle = positions.double()[:, :, None] * inv
    return torch.stack([torch.cos(angle) * amp, torch.sin(angle) * amp], -1).flatten(1, 2).float()


def _spec(case):
    from paper_2511_16047_b200 import binding as B
    return B.make_rotary(case["rotary_dim"], axes=case["axes"],
                         layout=B.ROTARY_INTERLEAVED if case.get("layout") == "interleaved" else B.ROTARY_HALF, base=case["base"],
                         scaling={"plain": B.ROTARY_PLAIN, "linear": B.ROTARY_LINEAR, "base": B.ROTARY_BASE,
                                  "parts": B.ROTARY_BY_PARTS}[case["scaling"]],
                         factor=case["factor"], original_length=case["original"])


class _Cache:
    """A cache of one layer over an arena of the caller's."""

    def __init__(self, case, sides, flags):
        from paper_2511_16047_b200 import binding as B
        self.B = B
        desc, _keep = B.make_desc(1, case["heads"], case["head_dim"], case["rows"], sides,
                                  [(case.get("condensed", 0), case.get("local", 1), case.get("demanding", False))], flags=flags)
        n = B.amskv_cache_required_bytes(desc)
        self.arena = torch.empty(n, dtype=torch.uint8, device="cuda")
        self.handle = B.amskv_cache_create(desc, self.arena, n)

    def __del__(self):
        if getattr(self, "handle", None):
            self.B.amskv_cache_destroy(self.handle)


def _rotary_inputs(case, seed):
    g = _generator(seed)
    rows, t, d, h, kh = case["rows"], case["T"], case["head_dim"], case["heads"], case["kv_heads"]
    if case["views"]:
        x = _bf16(g, rows, t, h + 2 * kh, d).transpose(1, 2)   # one projection's result: Q, K and V heads
        q, k = x[:, :h], x[:, h:h + kh]
    else:
        q, k = _bf16(g, rows, h, t, d), _bf16(g, rows, kh, t, d)
    index = None
    if case["index"]:
        index = torch.randint(0, t, (rows, t), generator=g, device="cuda", dtype=torch.int32)
        index[:, ::11] = -1   # tokens without a position
    return q, k, _positions(t, case["axes"], case["first"]), index


def _cross_inputs(case, seed):
    g = _generator(seed)
    rows, h, kh, d, s, t = (case[x] for x in ("rows", "heads", "kv_heads", "head_dim", "keys", "side"))
    t *= t
    q = _bf16(g, rows, t, h, d).transpose(1, 2) if case["views"] else _bf16(g, rows, h, t, d)
    lengths = _lengths(case)
    n, total = (1, max(1, sum(lengths))) if case["packed"] else (rows, s)
    if case["views"]:
        kv = _bf16(g, n, total, 2, kh, d)
        k, v = kv[:, :, 0].transpose(1, 2), kv[:, :, 1].transpose(1, 2)
    else:
        k, v = _bf16(g, n, kh, total, d), _bf16(g, n, kh, total, d)
    return q, k, v, lengths


def _cache_inputs(case, seed):
    """Q, K, V of every scale.  Keys have a few large channels, as trained ones do, and heads differ in size."""
    g = _generator(seed)
    rows, h, d = case["rows"], case["heads"], case["head_dim"]
    size = torch.exp2(_normal(g, 1, h, 1, 1))
    channel = torch.where(_normal(g, 1, h, 1, d) > 1.8, 6.0, 1.0)
    steps = []
    for s in _sides(case):
        q = _bf16(g, rows, h, s * s, d)
        k = (_normal(g, rows, h, s * s, d) * channel).bfloat16()
        v = (_normal(g, rows, h, s * s, d) * size).bfloat16()
        steps.append((q, k, v))
    return steps


def prepare(case, seed):
    st = _State()
    st.case, op = case, case["op"]
    if own:
        from paper_2511_16047_b200 import binding as B
        st.B = B
    if op == "table":
        st.positions = _positions(case["count"], case["axes"], int(seed) % 1000)
        if own:
            st.spec = _spec(case)
            st.table = torch.empty((case["count"], case["rotary_dim"] // 2, 2), dtype=torch.float32, device="cuda")
    elif op == "rotary":
        st.q, st.k, positions, st.index = _rotary_inputs(case, seed)
        if own:
            st.spec = _spec(case)
            st.table = torch.empty((case["T"], case["rotary_dim"] // 2, 2), dtype=torch.float32, device="cuda")
            st.B.amskv_rotary_table(st.spec, positions, case["T"], st.table, torch.cuda.current_stream())
            st.q_out, st.k_out = (torch.empty(x.shape, dtype=x.dtype, device="cuda") for x in (st.q, st.k))
        else:
            st.table = _plain_table(case, positions)
    elif op == "cross":
        st.q, st.k, st.v, lengths = _cross_inputs(case, seed)
        st.lengths = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        st.offsets = torch.zeros(case["rows"] + 1, dtype=torch.int32, device="cuda")
        st.offsets[1:] = torch.cumsum(st.lengths, 0)
        if own:
            st.cache = _Cache(case, [case["side"]], 0)
            st.out = torch.empty(st.q.shape, dtype=st.q.dtype, device="cuda")
    else:
        st.steps = _cache_inputs(case, seed)
        if own:
            st.cache = _Cache(case, _sides(case), st.B.FLAG_KV_E4M3)
            st.outs = [torch.empty_like(q) for q, _, _ in st.steps]
            if op == "store":
                st.back = [torch.empty_like(x) for x in st.steps[-1][1:]]
            if op == "attend":
                for k, (_, kk, v) in enumerate(st.steps):
                    st.B.amskv_append(st.cache.handle, 0, k, kk, v, torch.cuda.current_stream())
        if op == "attend":   # the cache is there before the call
            held = None if own else [(_plain_codes(kk), _plain_codes(v)) for _, kk, v in st.steps]
            st.q, st.steps = st.steps[-1][0], None
            if not own:
                st.held = [held[s] for s in _kept(case, len(held) - 1)]
    return st


# ---------------------------------------------------------------- plain forms
def _plain_rotary(case, table, x, index):
    """x [rows, heads, T, head_dim]; the table's rows in token order, or by index."""
    half = case["rotary_dim"] // 2
    if index is None:
        c, s = table[:, :, 0][None, None], table[:, :, 1][None, None]
    else:
        idle = (index < 0)[:, :, None]
        rows = table[index.clamp(min=0).long()]
        c = torch.where(idle, 1.0, rows[..., 0])[:, None]
        s = torch.where(idle, 0.0, rows[..., 1])[:, None]
    if case["transposed"]:
        s = -s
    part = x[..., :2 * half].float()
    shape = part.shape[:3]
    if case["layout"] == "interleaved":
        pairs = part.reshape(*shape, half, 2)
        u, w = pairs[..., 0], pairs[..., 1]
        turned = torch.stack([u * c - w * s, w * c + u * s], -1).reshape(part.shape)
    else:
        pairs = part.reshape(*shape, case["axes"], 2, half // case["axes"])
        u, w = pairs[..., 0, :].reshape(*shape, half), pairs[..., 1, :].reshape(*shape, half)
        a, b = u * c - w * s, w * c + u * s
        cut = (*shape, case["axes"], half // case["axes"])
        turned = torch.stack([a.reshape(cut), b.reshape(cut)], -2).reshape(part.shape)
    return torch.cat([turned.to(x.dtype), x[..., 2 * half:]], -1)


def _power(e):
    """2^e, exactly."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _plain_codes(x):
    """Codes in e4m3 and a power of two for every 16 tokens of a (row, head)."""
    rows, heads, t, d = x.shape
    blocks = (t + 15) // 16
    f = torch.zeros((rows, heads, blocks * 16, d), dtype=torch.float32, device=x.device)
    f[:, :, :t] = x.float()
    f = f.view(rows, heads, blocks, 16 * d)
    mant, exp = torch.frexp(f.abs().amax(-1, keepdim=True))
    e = (exp - 9 + (mant > 0.875)).clamp(min=-100)
    e = torch.where(mant == 0, 0, e)
    codes = (f * _power(-e)).to(torch.float8_e4m3fn)
    return codes.view(rows, heads, blocks * 16, d)[:, :, :t].contiguous(), e.to(torch.int8)


def _plain_values(held):
    codes, e = held
    rows, heads, t, d = codes.shape
    scale = _power(e).expand(rows, heads, e.shape[2], 16).reshape(rows, heads, -1, 1)[:, :, :t]
    return codes.float() * scale


def _plain_attention(q, k, v, lengths=None):
    """q [rows, heads, T, D], k and v [rows, kv_heads, S, D] in 32 bits; lengths: keys of each row.  A few rows or heads at a
    time where the scores would not fit."""
    rows, heads, t, d = q.shape
    n = k.shape[2]
    group = heads // k.shape[1]
    out = torch.empty((rows, heads, t, d), dtype=torch.bfloat16, device=q.device)
    step = max(1, int(5e8 // (t * n)))
    for r0 in range(0, rows, max(1, step // heads)):
        r1 = min(rows, r0 + max(1, step // heads))
        for h0 in range(0, heads, min(heads, step)):
            h1 = min(heads, h0 + min(heads, step))
            kv = torch.arange(h0, h1, device=q.device) // group
            kk, vv = k[r0:r1][:, kv], v[r0:r1][:, kv]
            scores = torch.matmul(q[r0:r1, h0:h1].float() * (1.0 / math.sqrt(d)), kk.transpose(2, 3))
            if lengths is not None:
                alive = (torch.arange(n, device=q.device)[None] < lengths[r0:r1, None])[:, None, None]
                scores = torch.where(alive, scores, float("-inf"))
            top = scores.amax(-1, keepdim=True)
            p = torch.exp(scores - torch.where(top == float("-inf"), 0.0, top))
            total = p.sum(-1, keepdim=True)
            out[r0:r1, h0:h1] = (torch.matmul(p, vv) / torch.where(total == 0, 1.0, total)).to(torch.bfloat16)
    return out


def _padded(case, x, lengths, offsets):
    """Packed states as padded ones."""
    n = case["keys"]
    at = offsets[:-1].long()[:, None] + torch.arange(n, device=x.device)[None]
    alive = torch.arange(n, device=x.device)[None] < lengths[:, None]
    at = torch.where(alive, at, 0)
    return torch.where(alive[:, None, :, None], x[0][:, at].transpose(0, 1).float(), 0.0)


def _run_plain(st):
    case, op = st.case, st.case["op"]
    if op == "table":
        return _plain_table(case, st.positions)
    if op == "rotary":
        return [_plain_rotary(case, st.table, x, st.index) for x in (st.q, st.k)]
    if op == "cross":
        if case["packed"]:
            k, v = (_padded(case, x, st.lengths, st.offsets) for x in (st.k, st.v))
        else:
            k, v = st.k.float(), st.v.float()
        return _plain_attention(st.q, k, v, st.lengths)
    if op == "store":
        return [_plain_values(_plain_codes(x)).to(torch.bfloat16) for x in st.steps[-1][1:]]
    if op == "attend":
        k, v = (torch.cat([_plain_values(s[i]) for s in st.held], 2) for i in range(2))
        return _plain_attention(st.q, k, v)
    held, outs = [], []
    for i, (q, kk, vv) in enumerate(st.steps):
        held.append((_plain_codes(kk), _plain_codes(vv)))
        k, v = (torch.cat([_plain_values(held[s][j]) for s in _kept(case, i)], 2) for j in range(2))
        outs.append(_plain_attention(q, k, v))
    return outs


# ---------------------------------------------------------------- the library's calls
def _run_own(st):
    B, case, op, stream = st.B, st.case, st.case["op"], torch.cuda.current_stream()
    if op == "table":
        B.amskv_rotary_table(st.spec, st.positions, case["count"], st.table, stream)
        return st.table
    if op == "rotary":
        B.amskv_rotary(st.spec, st.table, case["T"], 0, st.index, case["rows"], case["T"], case["head_dim"], case["heads"], st.q,
                       st.q_out, case["kv_heads"], st.k, st.k_out, transposed=case["transposed"], stream=stream)
        return [st.q_out, st.k_out]
    if op == "cross":
        keys = st.k.shape[2]
        where = {"offsets": st.offsets} if case["packed"] else {"lengths": st.lengths}
        B.amskv_cross_attend(st.cache.handle, 0, case["kv_heads"], keys, st.k, st.v, st.q, st.out, max_keys=case["keys"],
                             stream=stream, **where)
        return st.out
    cache = st.cache.handle
    if op == "attend":
        last = len(_sides(case)) - 1
        B.amskv_attend(cache, 0, last, st.q, st.outs[last], stream)
        return st.outs[last]
    B.amskv_cache_reset(cache)
    if op == "store":
        B.amskv_append(cache, 0, 0, st.steps[0][1], st.steps[0][2], stream)
        B.amskv_read_segment(cache, 0, 0, st.back[0], st.back[1], stream)
        return st.back
    for k, (q, kk, v) in enumerate(st.steps):
        B.amskv_append_attend(cache, 0, k, kk, v, q, st.outs[k], stream)
    return st.outs


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------- 64 bits, from the definitions
def _exact_angles(case, pos):
    p = case["rotary_dim"] // case["axes"]
    f, freqs, amp = case["factor"], [], 1.0
    for i in range(p // 2):
        w = math.exp(-2.0 * i / p * math.log(case["base"]))
        if case["scaling"] == "base":
            w = math.exp(-2.0 * i / p * (math.log(case["base"]) + p / (p - 2.0) * math.log(f)))
        elif case["scaling"] == "linear":
            w /= f
        elif case["scaling"] == "parts":
            # a channel that turns beta times over the original length sits at index d(beta)
            lo, hi = (p / 2.0 * (math.log(case["original"]) - math.log(2.0 * math.pi * b)) / math.log(case["base"]) for b in (32.0, 1.0))
            lo, hi = max(0, math.floor(lo)), min(p - 1, math.ceil(hi))
            share = min(1.0, max(0.0, (i - lo) / (hi - lo if hi > lo else 1e-3)))
            w, amp = w * (1.0 - share + share / f), 1.0 + 0.1 * math.log(f)
        freqs.append(w)
    w = torch.tensor(freqs, dtype=torch.float64, device=pos.device)
    return torch.cat([pos[:, a:a + 1].double() * w[None] for a in range(case["axes"])], 1), amp


def _exact_attention(q, k, v, chunk=1 << 27):
    """One (row, head): [T, D], [S, D], [S, D], all 64 bits."""
    if k.shape[0] == 0:
        return torch.zeros_like(q)
    out, step = torch.empty_like(q), max(1, chunk // k.shape[0])
    for t in range(0, q.shape[0], step):
        out[t:t + step] = torch.softmax(q[t:t + step] @ k.T / math.sqrt(q.shape[1]), -1) @ v
    return out


def _exact_held(x):
    """[rows, heads, T, D] -> the values an 8-bit cache holds, in 64 bits."""
    out = x.double()
    for b in range(0, x.shape[2], 16):
        block = out[:, :, b:b + 16]
        top = block.abs().amax((2, 3), keepdim=True)
        e = torch.ceil(torch.log2(top.clamp(min=1e-300) / 448.0)).clamp(min=-100.0)
        e = torch.where(top <= 448.0 * torch.exp2(e - 1.0), e - 1.0, e)   # (a logarithm may be off by a rounding)
        e = torch.where(top > 448.0 * torch.exp2(e), e + 1.0, e).clamp(min=-100.0)
        out[:, :, b:b + 16] = _exact_round(block * torch.exp2(-e)) * torch.exp2(e)
    return out


def _exact_round(y):
    """To the nearest number of 4 significant bits (steps of 2^-9 below 2^-6), ties to even."""
    low = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6)))
    low = torch.where(torch.exp2(low) > y.abs().clamp(min=2.0 ** -6), low - 1, low)
    step = torch.exp2(low - 3)
    return torch.round(y / step) * step


def exact(case, seed):
    op, w = case["op"], work(case)
    if op == "table":
        angle, amp = _exact_angles(case, _positions(case["count"], case["axes"], int(seed) % 1000))
        return torch.stack([angle.cos(), angle.sin()], -1) * amp
    if op == "rotary":
        q, k, pos, index = _rotary_inputs(case, seed)
        angle, amp = _exact_angles(case, pos)
        z = torch.polar(torch.full_like(angle, amp), -angle if case["transposed"] else angle)
        half, part = case["rotary_dim"] // 2, case["rotary_dim"] // case["axes"]
        i = torch.arange(half, device="cuda")
        if case["layout"] == "interleaved":
            first, second = 2 * i, 2 * i + 1
        else:
            first = torch.div(i, part // 2, rounding_mode="floor") * part + i % (part // 2)
            second = first + part // 2
        outs = []
        for x in (q, k):
            y = torch.empty(x.shape, dtype=torch.float64, device="cuda")
            for r in range(x.shape[0]):
                y[r] = x[r].double()
                turn = z if index is None else torch.where((index[r] >= 0)[:, None], z[index[r].long().clamp(min=0)], 1.0 + 0.0j)
                u = torch.complex(y[r][..., first], y[r][..., second]) * turn
                y[r][..., first], y[r][..., second] = u.real.clone(), u.imag.clone()
            outs.append(y)
        return outs
    if w["flops"] > 3e12 or w["bytes"] > 4e9:
        return None
    if op == "cross":
        q, k, v, lengths = _cross_inputs(case, seed)
        if case["rows"] * case["heads"] > 20000:
            return None
        out = torch.empty(q.shape, dtype=torch.float64, device="cuda")
        at = 0
        for r, n in enumerate(lengths):
            src, lo = (0, at) if case["packed"] else (r, 0)
            for h in range(case["heads"]):
                kh = h * case["kv_heads"] // case["heads"]
                out[r, h] = _exact_attention(q[r, h].double(), k[src, kh, lo:lo + n].double(), v[src, kh, lo:lo + n].double())
            at += n
        return out
    steps, sides = _cache_inputs(case, seed), _sides(case)
    if op != "store" and case["rows"] * case["heads"] * (1 if op == "attend" else len(sides)) > 20000:
        return None
    held = [[_exact_held(x) for x in (kk, v)] for _, kk, v in steps]
    if op == "store":
        return held[-1]
    outs = []
    for i, (q, _, _) in enumerate(steps):
        if op == "attend" and i < len(steps) - 1:
            continue
        out = torch.empty(q.shape, dtype=torch.float64, device="cuda")
        for r in range(case["rows"]):
            for h in range(case["heads"]):
                k, v = (torch.cat([held[s][j][r, h] for s in _kept(case, i)], 0) for j in range(2))
                out[r, h] = _exact_attention(q[r, h].double(), k, v)
        outs.append(out)
    return outs[-1] if op == "attend" else outs
