"""The operators in front of a compression, as cases to be timed and compared:
rotary positions and a paged 16-bit cache, into which a prompt is prefilled
chunk by chunk until its K and V are compressed.  A case is one call:

  rotate  rotary positions of Q and K rows (or the gradient: the rotation back)
  append  rows of new tokens into the pages, K rotated on the way, and Q with it
  gather  the rows of whole prompts out of the pages, packed for the compression
  attend  causal attention of a sequence's newest tokens (one, or a chunk) over
          its pages, with the log-sum-exp that the compression takes

A cache is a pool of pages of `page` slots; row s of its table lists the pages
of sequence s, whose slot j is row j % page of page table[s][j // page].  The
pool is [pages][heads][page][128] ("head") or [pages][page][heads][128]
("token").  Heads are those of the package's workloads (GQA 32/8, 28/4 and 64/8
heads, head_dim 128).

Keys have a few wide channels and values are N(0, 0.5); the queries of a KV
group share a direction and give scaled logits of standard deviation about 1.5,
and the first four slots of a sequence are attention sinks.
"""
import math

import numpy as np
import torch

own = False

D = 128   # head_dim
SHAPES = {"llama8b": (32, 8), "qwen7b": (28, 4), "llama70b": (64, 8)}
# rotary settings: channels rotated, layout, base, scaling
ROPES = {
    # the whole head, channel i with i + 64
    "half": (128, False, 500000.0, None),
    # ... frequencies scaled for a context eight times as long, long waves only
    "half_long": (128, False, 500000.0, ("waves", 8.0, 8192.0, 1.0, 4.0)),
    # neighbouring channels of the first half of a head, positions scaled by 4
    "part": (64, True, 10000.0, ("linear", 4.0)),
    # the whole head, neighbouring channels
    "pairs": (128, True, 10000.0, None),
}
LARGEST = 4 * D * 32 * 4096 * (131072 + 2048)  # flops of the largest attention


def _case(name, op, shape, batch, lo, hi, rows=1, dtype="bf16", page=64, layout="head", rope="half",
          backward=False, far=0, config=1):
    """`lo`..`hi`: slots of a sequence before the call (attend: besides the new
    ones; gather: prompt lengths; rotate: none); `rows`: new tokens of a
    sequence; `far`: the positions start about there; `config`: seed of the
    lengths."""
    return {"name": name, "op": op, "shape": shape, "batch": batch, "lo": lo, "hi": hi, "rows": rows,
            "dtype": dtype, "page": page, "layout": layout, "rope": rope, "backward": backward,
            "far": far, "config": config}


def listed():
    return [
        # the new tokens of a small serving batch, far into their contexts
        _case("rotate_token_b8", "rotate", "llama8b", 8, 0, 0, rope="half_long", far=100000),
        # gradients of a long training sequence's Q and K, part of each head
        _case("rotate_back_8191", "rotate", "qwen7b", 1, 0, 0, rows=8191, dtype="f16", rope="part",
              backward=True),
        # one new token for each of sixteen sequences
        _case("append_token_b16", "append", "llama8b", 16, 300, 1000, page=16),
        # a chunk of one prompt, an odd number of rows
        _case("append_chunk_8191", "append", "qwen7b", 1, 1001, 1001, rows=8191, dtype="f16", page=32,
              layout="token", rope="pairs"),
        # a short prompt, and a long one in small pages, packed for the compression
        _case("gather_777", "gather", "llama8b", 1, 777, 777),
        _case("gather_32k", "gather", "llama8b", 1, 32768, 32768, page=16),
        # one request's decode step over a short prompt
        _case("decode_777", "attend", "llama8b", 1, 776, 776),
        # a serving batch of a 70B-shaped model, eight query heads a group
        _case("decode_70b_b32", "attend", "llama70b", 32, 1000, 8000, dtype="f16", page=16, layout="token"),
        # the longest contexts
        _case("decode_128k_b4", "attend", "llama8b", 4, 131071, 131071),
        # a prompt's chunk between others, an odd number of tokens
        _case("chunk_501_at_16k", "attend", "qwen7b", 2, 9000, 16000, rows=501, dtype="f16", page=32),
        # a whole prompt from its first token on
        _case("prompt_8191", "attend", "llama8b", 1, 0, 0, rows=8191, page=128),
        # a large chunk late in the longest prompt
        _case("chunk_4k_at_128k", "attend", "llama8b", 1, 131072, 131072, rows=4096),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "attend", "append", "gather", "rotate"])
    shape = rng.choice(["llama8b", "llama8b", "qwen7b", "llama70b"])
    hq, h = SHAPES[shape]
    more = {"dtype": rng.choice(["bf16", "bf16", "f16"]), "page": rng.choice([16, 32, 64, 128, 256]),
            "layout": rng.choice(["head", "head", "token"]), "rope": rng.choice(sorted(ROPES)),
            "config": rng.randint(1, 1 << 20)}
    if op == "rotate":
        batch, rows = _log(rng, 1, 64), _log(rng, 1, 8192)
        while batch * rows * (hq + h) > 8192 * 40:
            rows = max(1, rows // 2)
        c = _case("", op, shape, batch, 0, 0, rows=rows, backward=rng.random() < 0.5,
                  far=rng.choice([0, 0, 1000, 100000, 1000000]), **more)
    elif op == "append":
        batch, rows = _log(rng, 1, 64), _log(rng, 1, 8192)
        while batch * rows * (hq + h) > 8192 * 40:
            rows = max(1, rows // 2)
        hi = _log(rng, 1, 2000)
        c = _case("", op, shape, batch, max(0, hi - rng.randint(0, 500)), hi, rows=rows, **more)
    elif op == "gather":
        batch, hi = _log(rng, 1, 32), _log(rng, 1, 32768)
        while batch * hi * h > 32768 * 8:
            batch, hi = max(1, batch // 2), hi if batch > 1 else hi // 2
        c = _case("", op, shape, batch, max(1, int(hi * rng.uniform(0.3, 1.0))), hi, **more)
    else:
        rows = rng.choice([1, 1, rng.randint(2, 8), _log(rng, 8, 8192), _log(rng, 8, 8192)])
        batch, hi = _log(rng, 1, 64), rng.choice([0, _log(rng, 1, 131072), _log(rng, 1, 131072)])
        # slots of all units, query tokens and flops within those of the listed cases
        while (batch > 1 or hi > 1) and (batch * h * (hi + rows) > 32 * 131072 or batch * rows > 16384
                                         or 4 * D * hq * batch * rows * (hi + rows) > LARGEST):
            batch, hi = max(1, batch // 2), hi if batch > 1 else hi // 2
        lo = hi if rng.random() < 0.4 else int(hi * rng.uniform(0.05, 0.9))
        c = _case("", op, shape, batch, lo, hi, rows=rows, **more)
    del c["name"]
    return c


# ------------------------------------------------------------- configuration
def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float16


def _before(c):
    """Slots of each sequence in use before the call."""
    rng = np.random.default_rng(c["config"])
    return rng.integers(c["lo"], c["hi"] + 1, size=c["batch"]).astype(np.int64)


def _after(c):
    return _before(c) + (0 if c["op"] == "gather" else c["rows"])


def _frequencies(rope):
    """Radians a position, in 64 bits."""
    rot, _, base, scaling = ROPES[rope]
    f = base ** -(np.arange(0, rot, 2, dtype=np.float64) / rot)
    if scaling is None:
        return f
    if scaling[0] == "linear":
        return f / scaling[1]
    # waves longer than length / low are stretched, those shorter than length /
    # high stay, those between are blended
    _, factor, length, low, high = scaling
    turns = length * f / (2 * math.pi)
    keep = np.clip((turns - low) / (high - low), 0.0, 1.0)
    return f * keep + f / factor * (1 - keep)


# ------------------------------------------------------------ the plain form
def _plain_rotate(x, positions, rope, backward=False):
    """Rows x [T, heads, 128] at int positions [T]; angles in 64 bits."""
    rot, interleaved, _, _ = ROPES[rope]
    f = torch.from_numpy(_frequencies(rope)).to(x.device)
    angle = positions.double()[:, None] * f * (-1 if backward else 1)
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    y = x.float().clone()
    if interleaved:
        a, b = y[..., 0:rot:2].clone(), y[..., 1:rot:2].clone()
        y[..., 0:rot:2], y[..., 1:rot:2] = a * cos - b * sin, a * sin + b * cos
    else:
        a, b = y[..., :rot // 2].clone(), y[..., rot // 2:rot].clone()
        y[..., :rot // 2], y[..., rot // 2:rot] = a * cos - b * sin, a * sin + b * cos
    return y.to(x.dtype)


def _plain_append(st):
    b, n, page = st["b"], st["rows"], st["page"]
    slot = (st["start"].long()[:, None] + torch.arange(n, device="cuda")).view(-1)
    seq = torch.arange(b, device="cuda").repeat_interleave(n)
    at = st["table"].long()[seq, slot // page]
    st["k_pages"][at, slot % page] = _plain_rotate(st["k"], slot, st["rope"])
    st["v_pages"][at, slot % page] = st["v"]
    st["lengths"].copy_(st["start"] + n)
    return _plain_rotate(st["q"], slot, st["rope"])


def _rows_of(st, part, s, n):
    """The first n slots of sequence s, [n, heads, 128]."""
    pages = st["table"][s, :-(-n // st["page"])].long()
    return st[part + "_pages"][pages].flatten(0, 1)[:n]


def _plain_gather(st):
    return [torch.cat([_rows_of(st, part, s, int(n)) for s, n in enumerate(st["lens"])])
            for part in ("k", "v")]


def _plain_attend(st):
    n, hq, h, q = st["rows"], st["hq"], st["h"], st["q"]
    group = hq // h
    out = torch.empty_like(q)
    lse = torch.empty((hq, q.shape[0]), dtype=torch.float32, device="cuda")
    for s, length in enumerate(st["lens"]):
        length = int(length)
        k = _rows_of(st, "k", s, length).transpose(0, 1).float()  # [h, length, D]
        v = _rows_of(st, "v", s, length).transpose(0, 1).float()
        step = max(1, min(n, (1 << 28) // (hq * length)))  # query tokens at a time
        for t in range(0, n, step):
            rows = slice(s * n + t, s * n + min(t + step, n))
            m = rows.stop - rows.start
            x = q[rows].float().view(m, h, group, D).permute(1, 0, 2, 3).reshape(h, m * group, D)
            z = (x @ k.transpose(1, 2) / math.sqrt(D)).view(h, m, group, length)
            last = length - n + t + torch.arange(m, device="cuda")
            hidden = torch.arange(length, device="cuda") > last[:, None]
            z = z.masked_fill(hidden[None, :, None], -math.inf)
            top = z.amax(-1, keepdim=True)
            e = torch.exp(z - top)
            total = e.sum(-1, keepdim=True)
            o = (e / total).view(h, m * group, length) @ v
            out[rows] = o.view(h, m, group, D).permute(1, 0, 2, 3).reshape(m, hq, D).to(q.dtype)
            lse[:, rows] = (top + total.log()).squeeze(-1).permute(0, 2, 1).reshape(hq, m)
    return out, lse


# ------------------------------------------------------------------ the calls
def _rows(gen, shape, dt, values):
    x = torch.randn(shape, generator=gen, device="cuda")
    if values:
        return (x * 0.5).to(dt)
    wide = torch.ones(D, device="cuda")
    wide[torch.randperm(D, generator=gen, device="cuda")[:4]] = 3.0
    return (x * wide).to(dt)


def prepare(case, seed):
    c, dev, dt = case, "cuda", _dtype(case)
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed))
    hq, h = SHAPES[c["shape"]]
    b, n, page = c["batch"], c["rows"], c["page"]
    st = {"op": c["op"], "b": b, "h": h, "hq": hq, "rows": n, "page": page, "rope": c["rope"],
          "backward": c["backward"]}
    if c["op"] == "rotate":
        first = c["far"] + torch.randint(0, 2000, (b, 1), generator=gen, device=dev)
        st["positions"] = (first + torch.arange(n, device=dev)).int().view(-1)
        st["q"] = _rows(gen, (b * n, hq, D), dt, False)
        st["k"] = _rows(gen, (b * n, h, D), dt, False)
        return st
    before, lens = _before(c), _after(c)
    st["lens"] = lens
    # the pool: somewhat more pages than are used, in no order
    used = -(-lens // page)
    pool = int(used.sum()) + b
    width = int(used.max()) + 1
    order = torch.randperm(pool, generator=gen, device=dev).int()
    table = np.full((b, width), -1, np.int64)
    at = 0
    for s in range(b):
        table[s, :used[s]] = np.arange(at, at + used[s])
        at += int(used[s])
    table = torch.from_numpy(table).to(dev)
    st["table"] = torch.where(table >= 0, order[table.clamp_min(0)], -1).int()
    lengths = lens if c["op"] != "append" else before
    st["lengths"] = torch.from_numpy(lengths).to(dev).int()
    for part in ("k", "v"):
        shape = (pool, h, page, D) if c["layout"] == "head" else (pool, page, h, D)
        x = torch.empty(shape, dtype=dt, device=dev)
        for i in range(0, pool, 4096):
            x[i:i + 4096] = _rows(gen, x[i:i + 4096].shape, dt, part == "v")
        st[part + "_pages"] = x.transpose(1, 2) if c["layout"] == "head" else x
    if c["op"] == "attend":
        common = torch.randn((b, 1, h, 1, D), generator=gen, device=dev)
        each = torch.randn((b, n, h, hq // h, D), generator=gen, device=dev)
        st["q"] = (1.1 * (0.8 * common + 0.6 * each)).view(b * n, hq, D).to(dt)
        for s in range(b):  # the first slots draw every query of their group
            sinks = torch.arange(min(4, int(lens[s])), device=dev)
            st["k_pages"][st["table"][s, 0].long(), sinks] += common[s, 0, :, 0].to(dt) * 0.35
    elif c["op"] == "append":
        st["start"] = st["lengths"].clone()
        st["q"] = _rows(gen, (b * n, hq, D), dt, False)
        st["k"] = _rows(gen, (b * n, h, D), dt, False)
        st["v"] = _rows(gen, (b * n, h, D), dt, True)
    return st


def _handle(st):
    """What a program makes once and keeps: its cache, rotary table, workspace
    and output buffers."""
    import paper_2606_24467_gb300 as ckv

    if "ready" not in st:
        if st["op"] in ("rotate", "append"):
            rot, interleaved, base, scaling = ROPES[st["rope"]]
            more = {}
            if scaling is not None and scaling[0] == "linear":
                more = {"scaling": "linear", "factor": scaling[1]}
            elif scaling is not None:
                more = {"scaling": "waves", "factor": scaling[1], "original_length": scaling[2],
                        "low": scaling[3], "high": scaling[4]}
            st["table_of_angles"] = ckv.Rope(rot, base=base, interleaved=interleaved, **more)
            st["q_out"] = torch.empty_like(st["q"])
        if st["op"] == "rotate":
            st["k_out"] = torch.empty_like(st["k"])
        else:
            st["cache"] = ckv.PagedCache(st["k_pages"], st["v_pages"], st["table"], st["lengths"])
        if st["op"] == "gather":
            st["cu"] = np.concatenate([[0], np.cumsum(st["lens"])]).astype(np.int32)
            shape = (int(st["cu"][-1]), st["h"], D)
            st["k_out"] = torch.empty(shape, dtype=st["k_pages"].dtype, device="cuda")
            st["v_out"] = torch.empty_like(st["k_out"])
        if st["op"] == "attend":
            st["ws"] = ckv.paged_workspace(st["cache"], st["hq"], st["rows"])
            st["out"] = torch.empty_like(st["q"])
            st["lse"] = torch.empty((st["hq"], st["q"].shape[0]), dtype=torch.float32, device="cuda")
        st["ready"] = True
    return ckv


def run(st):
    op = st["op"]
    ckv = _handle(st) if own else None
    if op == "rotate":
        if own:
            ckv.rope_apply(st["table_of_angles"], st["positions"], st["q"], st["k"], q_out=st["q_out"],
                           k_out=st["k_out"], backward=st["backward"])
            return {"q": st["q_out"], "k": st["k_out"]}
        return {part: _plain_rotate(st[part], st["positions"], st["rope"], st["backward"])
                for part in ("q", "k")}
    if op == "append":
        if own:
            ckv.paged_append(st["cache"], st["k"], st["v"], start=st["start"], rope=st["table_of_angles"],
                             q=st["q"], q_out=st["q_out"])
            q = st["q_out"]
        else:
            q = _plain_append(st)
        return {"q": q, "k_pages": st["k_pages"], "v_pages": st["v_pages"], "lengths": st["lengths"]}
    if op == "gather":
        if own:
            ckv.paged_gather(st["cache"], st["k_out"], st["v_out"], st["cu"])
            return {"k": st["k_out"], "v": st["v_out"]}
        k, v = _plain_gather(st)
        return {"k": k, "v": v}
    if own:
        ckv.paged_attend(st["cache"], st["q"], st["out"], st["ws"], lse=st["lse"])
        return {"out": st["out"], "lse": st["lse"]}
    out, lse = _plain_attend(st)
    return {"out": out, "lse": lse}


def work(case):
    """Bytes: input rows and slots in use read once, outputs written once.  Four
    products and two sums a rotated pair; two products and sums a channel of a
    visible slot and query head."""
    c, dt = case, 2
    hq, h = SHAPES[c["shape"]]
    b, n = c["batch"], c["rows"]
    rot = ROPES[c["rope"]][0]
    if c["op"] == "rotate":
        return {"bytes": b * n * ((hq + h) * D * dt * 2 + 4), "flops": b * n * (hq + h) * rot // 2 * 6}
    if c["op"] == "append":
        return {"bytes": b * n * (hq + 2 * h) * D * dt * 2 + 8 * b, "flops": b * n * (hq + h) * rot // 2 * 6}
    lens = _after(c)
    pages = int((-(-lens // c["page"])).sum())
    if c["op"] == "gather":
        rows = int(lens.sum())
        return {"bytes": rows * h * D * dt * 4 + 4 * pages, "flops": rows * h * D * 2}
    seen = int((n * (lens - n)).sum()) + b * n * (n + 1) // 2
    return {"bytes": int(lens.sum()) * h * D * dt * 2 + b * n * hq * (2 * D * dt + 4) + 4 * pages,
            "flops": 4 * D * hq * seen}


def exact(case, seed):
    """In 64 bits: rotations as products of complex numbers, attention a head
    and a few query tokens at a time."""
    c = case
    if c["op"] == "attend" and work(c)["flops"] > 6e12:
        return None
    st = prepare(case, seed)
    n, page = st["rows"], st["page"]

    def turned(x, pos, sign):
        rot, interleaved, _, _ = ROPES[c["rope"]]
        w = torch.from_numpy(_frequencies(c["rope"])).cuda()
        unit = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), sign * torch.outer(pos.double(), w))
        y = x.double()
        head, tail = y[..., :rot], y[..., rot:]
        pairs = head.unflatten(-1, (-1, 2)) if interleaved else head.unflatten(-1, (2, -1)).transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * unit[:, None])
        back = z.flatten(-2) if interleaved else z.transpose(-1, -2).flatten(-2)
        return torch.cat([back, tail], -1)

    if c["op"] == "rotate":
        sign = -1.0 if c["backward"] else 1.0
        return {part: turned(st[part], st["positions"], sign) for part in ("q", "k")}
    if c["op"] == "append":
        k, v = st["k_pages"].double(), st["v_pages"].double()
        first = st["start"].cpu().numpy()
        pos = np.concatenate([first[s] + np.arange(n) for s in range(st["b"])])
        table = st["table"].cpu().numpy()
        where = np.concatenate([table[s, (first[s] + np.arange(n)) // page] for s in range(st["b"])])
        where, pos = torch.from_numpy(where.astype(np.int64)).cuda(), torch.from_numpy(pos).cuda().long()
        k[where, pos % page], v[where, pos % page] = turned(st["k"], pos, 1.0), st["v"].double()
        return {"q": turned(st["q"], pos, 1.0), "k_pages": k, "v_pages": v, "lengths": None}

    def rows(part, s, head, length):
        slot = torch.arange(length, device="cuda")
        at = st["table"][s].long()[torch.div(slot, page, rounding_mode="floor")]
        return st[part + "_pages"][at, slot % page, head].double()

    if c["op"] == "gather":
        every = range(st["h"])
        return {part: torch.cat([torch.stack([rows(part, s, g, int(m)) for g in every], 1)
                                 for s, m in enumerate(st["lens"])]) for part in ("k", "v")}
    q = st["q"].double()
    out = torch.zeros_like(q)
    lse = torch.zeros(q.shape[1], q.shape[0], dtype=torch.float64, device="cuda")
    for s, length in enumerate(st["lens"]):
        length = int(length)
        place = torch.arange(length, device="cuda")
        for head in range(st["h"]):
            kk, vv = rows("k", s, head, length), rows("v", s, head, length)
            for i in range(head * (st["hq"] // st["h"]), (head + 1) * (st["hq"] // st["h"])):
                for t in range(0, n, 1024):
                    m = min(1024, n - t)
                    at = slice(s * n + t, s * n + t + m)
                    z = (q[at, i] @ kk.T) * D ** -0.5
                    z += torch.where(place > length - n + t + torch.arange(m, device="cuda")[:, None], -math.inf, 0.0)
                    lse[i, at] = torch.logsumexp(z, -1)
                    out[at, i] = torch.exp(z - lse[i, at, None]) @ vv
    return {"out": out, "lse": lse}
