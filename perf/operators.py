"""The operators of the 4-bit KV cache, as cases to be timed and compared.

After the compression of a prompt the kept rows live in a cache of 4-bit
codes; every decode step appends rows to it, attends over it and, from time to
time, evicts the slots that gathered the least attention.  A case is one call:

  append   rows of new tokens into the cache, with the values that it then holds
  gather   a prompt's retained rows into the cache by index lists, likewise
  attend   attention of one or a few query tokens a sequence over the cache
  evict    eviction down to a budget by accumulated attention weight, in place

A unit is a (sequence, KV group); a cache has `capacity` slots a unit.  A slot
has 128 codes of 4 bits for K and for V (byte b: channel 2b in the low bits,
2b + 1 in the high ones) and, for every 32 channels, a bf16 scale s and minimum
m (rows of 8: 4 scales, 4 minima): code n stands for s n + m.  Shapes are those
of the package's workloads (GQA 32/8, 28/4 and 64/8 heads, head_dim 128).

Keys have a few wide channels and values are N(0, 0.5); the queries of a KV
group share a direction and give scaled logits of standard deviation about 1.5;
accumulated weights are log-normal, some of them zero.
"""
import math

import numpy as np
import torch

own = False

D = 128   # head_dim
GR = 32   # channels that share a scale
SHAPES = {"llama8b": (32, 8), "qwen7b": (28, 4), "llama70b": (64, 8)}


def _case(name, op, shape, batch, lo, hi, queries=1, causal=False, weights=False, dtype="bf16",
          rows=1, budget=0, layers=1, sinks=4, recent=32, config=1):
    """`lo`..`hi`: slots in use (attend, evict: before the call; append: rows
    before it; gather: prompt lengths); `rows`: rows appended a sequence;
    `queries`: query tokens a sequence; `causal`: slots are seen by position;
    `weights`: attention weights are accumulated; `budget`: slots kept (a share
    of the slots in use below 1); `config`: seed of the lengths."""
    return {"name": name, "op": op, "shape": shape, "batch": batch, "lo": lo, "hi": hi,
            "queries": queries, "causal": causal, "weights": weights, "dtype": dtype, "rows": rows,
            "budget": budget, "layers": layers, "sinks": sinks, "recent": recent, "config": config}


def listed():
    return [
        # one request's decode step over a short prompt
        _case("decode_777", "attend", "llama8b", 1, 777, 777),
        # a serving batch of compressed prompts that evicts by weight later
        _case("decode_b8_weights", "attend", "llama8b", 8, 200, 1100, weights=True),
        # one long prompt, kept whole in 4 bits
        _case("decode_32k", "attend", "llama8b", 1, 32768, 32768),
        # speculative tokens verified in one call over a ragged batch
        _case("verify_4_ragged", "attend", "qwen7b", 8, 2000, 16000, queries=4, causal=True,
              weights=True, dtype="f16"),
        # the longest contexts, the largest cache
        _case("decode_128k_b4", "attend", "llama8b", 4, 131072, 131072),
        # a large serving batch of a 70B-shaped model, eight query heads a group
        _case("decode_70b_b64", "attend", "llama70b", 64, 1000, 8000, weights=True, dtype="f16"),
        # one new token for each of sixteen sequences
        _case("append_token_b16", "append", "llama8b", 16, 300, 1000),
        # a chunk of one prompt, an odd number of rows
        _case("append_chunk_8191", "append", "qwen7b", 1, 1001, 1001, rows=8191, dtype="f16"),
        # the kept rows of one layer of a short prompt
        _case("fill_layer_4k", "gather", "llama8b", 1, 4096, 4096, budget=128),
        # ... of all layers of a long prompt
        _case("fill_32layers_32k", "gather", "llama8b", 1, 32768, 32768, budget=917, layers=32),
        # every decode step drops one slot of each unit of a layer
        _case("evict_step_b8", "evict", "llama8b", 8, 1025, 1025, budget=1024),
        # ... or all layers drop 128 slots at once
        _case("evict_32layers_b8", "evict", "llama8b", 8, 1100, 1200, budget=1024, layers=32),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "append", "gather", "evict"])
    shape = rng.choice(["llama8b", "llama8b", "qwen7b", "llama70b"])
    heads = SHAPES[shape][1]
    dtype = rng.choice(["bf16", "bf16", "f16"])
    config = rng.randint(1, 1 << 20)
    more = {"sinks": rng.choice([0, 1, 4, 16]), "recent": rng.choice([0, 8, 32, 100])}
    room = 4 * 8 * 131072  # (sequence, group, slot)s of the largest listed case
    if op == "attend":
        batch, hi = _log(rng, 1, 64), _log(rng, 1, 131072)
        queries = rng.choice([1, 1, 1, 2, 3, 5, 8])
        while batch * heads * hi * queries > room:
            batch, hi = max(1, batch // 2), hi if batch > 1 else hi // 2
        lo = hi if rng.random() < 0.4 else max(1, int(hi * rng.uniform(0.05, 0.9)))
        c = _case("", op, shape, batch, max(lo, queries), max(hi, queries), queries=queries,
                  causal=queries > 1 or rng.random() < 0.3, weights=rng.random() < 0.5, dtype=dtype,
                  config=config)
    elif op == "append":
        batch, rows = _log(rng, 1, 64), _log(rng, 1, 8192)
        while batch * rows > 16384:
            rows = max(1, rows // 2)
        hi = _log(rng, 1, 2000)
        c = _case("", op, shape, batch, max(0, hi - rng.randint(0, 500)), hi, rows=rows, dtype=dtype,
                  config=config)
    elif op == "gather":
        layers, batch, hi = rng.choice([1, 1, 4, 16, 32]), rng.choice([1, 2, 4]), _log(rng, 100, 32768)
        budget = rng.choice([64, 128, 500, 917, 0.1, 0.5])
        most = budget if budget >= 1 else budget * hi  # rows kept of the longest prompt
        while layers * batch * heads * max(most, hi / 16) > 32 * 8 * 2048:
            layers, batch = max(1, layers // 2), max(1, batch // 2)
        c = _case("", op, shape, batch, max(20, int(hi * rng.uniform(0.3, 1.0))), hi, budget=budget,
                  layers=layers, dtype=dtype, config=config)
    else:
        layers, batch, hi = rng.choice([1, 1, 4, 16, 32]), _log(rng, 1, 16), _log(rng, 200, 40000)
        while layers * batch * heads * hi > 32 * 8 * 8 * 2000:
            layers, batch = max(1, layers // 2), max(1, batch // 2)
            hi = hi // 2 if layers * batch == 1 else hi
        c = _case("", op, shape, batch, max(150, int(hi * rng.uniform(0.5, 1.0))), hi,
                  budget=rng.choice([0.3, 0.5, 0.8, 0.95, 0.99, max(140, hi - 1)]), layers=layers,
                  config=config, **more)
    del c["name"]
    return c


# ------------------------------------------------------------- configuration
def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float16


def _lengths(c):
    """Slots in use (or prompt lengths) of each packed sequence."""
    rng = np.random.default_rng(c["config"])
    return np.tile(rng.integers(c["lo"], c["hi"] + 1, size=c["batch"]), c["layers"]).astype(np.int64)


def _kept(c):
    n = _lengths(c)
    b = np.full_like(n, int(c["budget"])) if c["budget"] >= 1 else (n * c["budget"]).astype(np.int64)
    if c["op"] == "evict":
        b = np.maximum(b, c["sinks"] + c["recent"])
    return np.minimum(b, n)


def _capacity(c):
    if c["op"] == "gather":
        most = int(_kept(c).max())
    else:
        most = int(_lengths(c).max()) + (c["rows"] if c["op"] == "append" else 0)
    return -(-max(most, 1) // 32) * 32


# ------------------------------------------------------------ the plain form
def _quantise(x):
    """Codes [.., 128] (uint8) and params [.., 8] (bf16) of rows x [.., 128]:
    the minimum rounded down to bf16, the smallest bf16 scale s with
    15 s >= max - minimum, and codes by the exact quotient, ties to even."""
    g = x.unflatten(-1, (D // GR, GR))
    lo = g.amin(-1).float()
    m = lo.bfloat16()
    m = torch.where(m.float() > lo, _step(m, -1), m)
    top = g.amax(-1).float() - m.float()
    s = (top / 15).bfloat16()
    s = torch.where(s.double() * 15 < top.double(), _step(s, 1), s)
    under = _step(s, -1)
    s = torch.where((s > 0) & (under.double() * 15 >= top.double()), under, s)
    d = g.float() - m.float()[..., None]
    n = (d.double() / torch.where(s > 0, s, torch.ones_like(s)).double()[..., None]).round()
    return n.to(torch.uint8).flatten(-2), torch.cat([s, m], -1)


def _step(x, up):
    """The next bf16 above (up = 1) or below (up = -1) x."""
    bits = x.view(torch.int16).to(torch.int32)
    line = torch.where(bits < 0, -(bits & 0x7FFF), bits) + up  # -0 and +0 are one place
    return torch.where(line < 0, (-line) - 32768, line).to(torch.int16).view(torch.bfloat16)


def _pack(codes):
    return codes[..., 0::2] | (codes[..., 1::2] << 4)


def _values(packed, params):
    """The values that codes stand for, in 32 bits."""
    n = torch.stack([packed & 15, packed >> 4], -1).flatten(-2).unflatten(-1, (D // GR, GR))
    s, m = params.float().split(4, -1)
    return (n.float() * s[..., None] + m[..., None]).flatten(-2)


def _plain_write(st, k, v, positions, weights, unit, slot):
    """Rows [R, 128] of units and slots [R] into the cache; their values."""
    back = []
    for x, part in ((k, "k"), (v, "v")):
        codes, params = _quantise(x)
        packed = _pack(codes)
        st[part + "_codes"].view(-1, st["cap"], D // 2)[unit, slot] = packed
        st[part + "_params"].view(-1, st["cap"], 8)[unit, slot] = params
        back.append(_values(packed, params).to(x.dtype))
    st["positions"].view(-1, st["cap"])[unit, slot] = positions
    st["weights"].view(-1, st["cap"])[unit, slot] = weights
    return back


def _plain_append(st):
    b, h, n = st["b"], st["h"], st["rows"]
    seq = torch.arange(b, device="cuda")[:, None, None]
    head = torch.arange(h, device="cuda")
    row = torch.arange(n, device="cuda")[:, None]
    unit = (seq * h + head).expand(b, n, h).reshape(-1)
    slot = (st["start"].view(b, 1, h) + row).reshape(-1).long()
    pos = st["new_positions"].view(b, n, 1).expand(b, n, h).reshape(-1)
    kb, vb = _plain_write(st, st["k"].reshape(-1, D), st["v"].reshape(-1, D), pos, 0.0, unit, slot)
    st["lengths"].copy_(st["start"] + n)
    return kb.view(st["k"].shape), vb.view(st["v"].shape)


def _plain_gather(st):
    b, h, cu = st["b"], st["h"], st["cu_out_dev"]
    rows = st["indices"].shape[1]
    row = torch.arange(rows, device="cuda")
    seq = torch.searchsorted(cu[1:], row, right=True)
    head = torch.arange(h, device="cuda")
    at = st["cu_dev"][seq][:, None] + st["indices"].T.long()
    unit = (seq[:, None] * h + head).reshape(-1)
    slot = (row - cu[seq])[:, None].expand(rows, h).reshape(-1)
    k, v = st["k"][at, head].reshape(-1, D), st["v"][at, head].reshape(-1, D)
    kb, vb = _plain_write(st, k, v, st["indices"].T.reshape(-1), 0.0, unit, slot)
    st["lengths"].copy_((cu[1:] - cu[:-1])[:, None].expand(b, h))
    return kb.view(rows, h, D), vb.view(rows, h, D)


def _plain_attend(st):
    b, h, cap, q = st["b"], st["h"], st["cap"], st["q"]
    n = q.shape[2]
    rows = q.view(b, h, -1, D).float()  # the group's heads, each with its query tokens
    group = rows.shape[2] // n
    z = rows @ _values(st["k_codes"], st["k_params"]).transpose(-1, -2) / math.sqrt(D)
    seen = (torch.arange(cap, device="cuda") < st["lengths"][..., None])[:, :, None]
    if "q_positions" in st:
        at = st["q_positions"].repeat(1, group)[:, None, :, None]  # row = (head, token)
        seen = seen & (st["positions"][:, :, None] <= at)
    z = z.masked_fill(~seen, -math.inf)
    top = z.amax(-1, keepdim=True)
    e = torch.exp(z - top.clamp_min(-1e30))
    total = e.sum(-1, keepdim=True)
    p = e / total.clamp_min(1e-30)
    out = (p @ _values(st["v_codes"], st["v_params"])).to(q.dtype).view_as(q)
    lse = (top + total.log()).squeeze(-1).view(b, -1, n)
    if st["accumulate"]:
        st["weights"] += p.sum(2)
    return out, lse


def _plain_evict(st):
    cap, n = st["cap"], st["lengths"].view(-1, 1).clone()
    pos, wt = st["positions"].view(-1, cap), st["weights"].view(-1, cap)
    slot = torch.arange(cap, device="cuda")
    used = slot < n
    newest = pos.masked_fill(~used, -1).amax(1, keepdim=True)
    forced = (pos < st["sinks"]) | (pos > newest - st["recent"])
    rank = torch.where(forced, math.inf, wt).masked_fill(~used, -math.inf)
    order = torch.sort(rank, dim=1, descending=True, stable=True).indices
    left = torch.minimum(n, st["budgets"].view(-1, 1))
    keep = torch.zeros_like(used).scatter_(1, order, slot < left)
    holes, movers = used & ~keep & (slot < left), keep & (slot >= left)
    # nonzero() lists unit by unit in slot order: the j-th hole takes the j-th mover
    (unit, to), (_, frm) = holes.nonzero().T, movers.nonzero().T
    for name in ("k_codes", "v_codes", "k_params", "v_params", "positions", "weights"):
        a = st[name].view(-1, cap, *st[name].shape[3:])
        a[unit, to] = a[unit, frm]
    st["lengths"].copy_(left.view_as(st["lengths"]))


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
    lens, cap = _lengths(c), _capacity(c)
    b = len(lens)
    st = {"op": c["op"], "b": b, "h": h, "hq": hq, "cap": cap}
    # the cache: metadata in one buffer, which an eviction changes
    u = b * h
    meta = torch.zeros(2 * u * cap + u, dtype=torch.int32, device=dev)
    st["meta"] = meta
    st["positions"] = meta[:u * cap].view(b, h, cap)
    st["weights"] = meta[u * cap:2 * u * cap].view(torch.float32).view(b, h, cap)
    st["lengths"] = meta[2 * u * cap:].view(b, h)
    st["lengths"].copy_(torch.from_numpy(lens).to(dev)[:, None].expand(b, h))
    for part in ("k", "v"):
        st[part + "_codes"] = torch.zeros((b, h, cap, D // 2), dtype=torch.uint8, device=dev)
        st[part + "_params"] = torch.zeros((b, h, cap, 8), dtype=torch.bfloat16, device=dev)
    if c["op"] in ("attend", "evict"):
        for part in ("k", "v"):
            for s in range(b):  # a sequence at a time: the codes are made in 64 bits
                codes, params = _quantise(_rows(gen, (h, cap, D), torch.bfloat16, part == "v"))
                st[part + "_codes"][s] = _pack(codes)
                st[part + "_params"][s] = params
        # positions with gaps, in the order of no sort once slots were evicted
        step = torch.randint(1, 4, (b, h, cap), generator=gen, device=dev)
        pos = step.cumsum(-1).int()
        if c["op"] == "evict":
            mixed = torch.rand((b, h, cap), generator=gen, device=dev)
            mixed.masked_fill_(torch.arange(cap, device=dev) >= st["lengths"][..., None], 2.0)
            pos = pos.gather(-1, mixed.argsort(-1))
        st["positions"].copy_(pos - pos.amin(-1, keepdim=True))
        w = torch.exp(2 * torch.randn((b, h, cap), generator=gen, device=dev))
        w.masked_fill_(torch.rand((b, h, cap), generator=gen, device=dev) < 0.02, 0.0)
        st["weights"].copy_(w)
    if c["op"] == "attend":
        n = c["queries"]
        common = torch.randn((b, h, 1, 1, D), generator=gen, device=dev)
        each = torch.randn((b, h, hq // h, n, D), generator=gen, device=dev)
        st["q"] = (1.1 * (0.8 * common + 0.6 * each)).view(b, hq, n, D).to(dt)
        st["accumulate"] = c["weights"]
        if c["causal"]:
            # the query tokens are the newest of their sequence: slots of the same
            # positions in every group
            st["positions"].copy_(st["positions"][:, :1].expand(b, h, cap).clone())
            last = st["positions"][:, 0].gather(1, st["lengths"][:, :1].long() - 1)
            back = torch.arange(n, device=dev, dtype=torch.int32) - (n - 1)
            st["q_positions"] = (last + 2 * back).contiguous()
    elif c["op"] == "append":
        n = st["rows"] = c["rows"]
        st["start"] = st["lengths"].clone()
        st["k"] = _rows(gen, (b * n, h, D), dt, False)
        st["v"] = _rows(gen, (b * n, h, D), dt, True)
        first = torch.from_numpy(lens).to(dev)[:, None]
        st["new_positions"] = (first + torch.arange(n, device=dev)).int().view(-1)
    elif c["op"] == "gather":
        kept = _kept(c)
        st["cu"] = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        st["cu_out"] = np.concatenate([[0], np.cumsum(kept)]).astype(np.int32)
        st["cu_dev"] = torch.from_numpy(st["cu"]).to(dev).long()
        st["cu_out_dev"] = torch.from_numpy(st["cu_out"]).to(dev).long()
        st["k"] = _rows(gen, (int(st["cu"][-1]), h, D), dt, False)
        st["v"] = torch.empty_like(st["k"]).normal_(generator=gen) * 0.5
        # a compression's choice: ascending positions, all over the prompt
        st["indices"] = torch.empty((h, int(st["cu_out"][-1])), dtype=torch.int32, device=dev)
        for s in range(b):
            pick = torch.rand((h, int(lens[s])), generator=gen, device=dev).argsort(-1)[:, :int(kept[s])]
            st["indices"][:, int(st["cu_out"][s]):int(st["cu_out"][s + 1])] = pick.sort(-1).values.int()
        # window queries of the compression call: its problem description is kept
        st["q_win"] = torch.empty((b, hq, 32, D), dtype=dt, device=dev)
    else:
        st["before"] = meta.clone()
        st["sinks"], st["recent"] = c["sinks"], c["recent"]
        kept = torch.from_numpy(_kept(c)).to(dev)
        st["budgets"] = kept[:, None].expand(b, h).int().contiguous()
    return st


def _cache(st):
    import paper_2606_24467_gb300 as ckv

    if "cache" not in st:  # a program's handle on its cache, kept like the cache itself
        st["cache"] = ckv.Q4Cache(st["k_codes"], st["v_codes"], st["k_params"], st["v_params"],
                                  st["positions"], st["lengths"], st["weights"])
        if st["op"] in ("attend", "evict"):
            n = st["q"].shape[2] if st["op"] == "attend" else 1
            st["ws"] = ckv.q4_workspace(st["cache"], st["hq"], n)
        if st["op"] == "attend":
            st["out"] = torch.empty_like(st["q"])
            st["lse"] = torch.empty(st["q"].shape[:3], dtype=torch.float32, device="cuda")
        elif st["op"] == "append":
            st["k_back"], st["v_back"] = torch.empty_like(st["k"]), torch.empty_like(st["v"])
        elif st["op"] == "gather":
            shape = (st["indices"].shape[1], st["h"], D)
            st["k_back"] = torch.empty(shape, dtype=st["k"].dtype, device="cuda")
            st["v_back"] = torch.empty_like(st["k_back"])
            st["problem"] = ckv.Problem(st["q_win"], st["k"], st["cu"], 32, 7)
    return ckv, st["cache"]


def run(st):
    op = st["op"]
    if op == "evict":
        # between two evictions a program's decode steps write new weights and
        # lengths; here they are set back to what they were
        st["meta"].copy_(st["before"])
    if own:
        ckv, cache = _cache(st)
        if op == "attend":
            ckv.q4_attend(cache, st["q"], st["out"], st["ws"], q_positions=st.get("q_positions"),
                          lse=st["lse"], accumulate=st["accumulate"])
            out, lse = st["out"], st["lse"]
        elif op == "append":
            ckv.q4_append(cache, st["k"], st["v"], st["new_positions"], start=st["start"],
                          k_values=st["k_back"], v_values=st["v_back"])
            kb, vb = st["k_back"], st["v_back"]
        elif op == "gather":
            ckv.q4_gather(st["problem"], cache, st["indices"], st["cu_out"], st["k"], st["v"],
                          k_values=st["k_back"], v_values=st["v_back"])
            kb, vb = st["k_back"], st["v_back"]
        else:
            ckv.q4_evict(cache, st["budgets"], st["ws"], sinks=st["sinks"], recent=st["recent"])
    elif op == "attend":
        out, lse = _plain_attend(st)
    elif op == "append":
        kb, vb = _plain_append(st)
    elif op == "gather":
        kb, vb = _plain_gather(st)
    else:
        _plain_evict(st)
    if op == "attend":
        got = {"out": out, "lse": lse}
        if st["accumulate"]:
            got["weights"] = st["weights"]
        return got
    if op in ("append", "gather"):
        # the values that the cache holds, and the words that hold them
        return {"k": kb, "v": vb, "k_words": st["k_codes"].view(torch.int64),
                "v_words": st["v_codes"].view(torch.int64), "k_params": st["k_params"],
                "v_params": st["v_params"], "positions": st["positions"], "lengths": st["lengths"]}
    # rows that moved are copies: compared as the words they are
    return {"k_words": st["k_codes"].view(torch.int64), "v_words": st["v_codes"].view(torch.int64),
            "k_params": st["k_params"].view(torch.int64), "v_params": st["v_params"].view(torch.int64),
            "positions": st["positions"], "lengths": st["lengths"], "weights": st["weights"]}


def work(case):
    """Bytes: every slot in use, index and input row read once, every output
    and every slot that changes written once.  An eviction reads a weight and
    a position a slot; of the slots below the budget the share that is evicted
    on average is filled again."""
    c, dt = case, 2
    hq, h = SHAPES[c["shape"]]
    lens = _lengths(c)
    b = len(lens)
    slot = 2 * (D // 2 + 16)  # codes and params of K and V
    if c["op"] == "attend":
        rows = hq * c["queries"]
        per = slot + (4 if c["causal"] else 0) + (8 if c["weights"] else 0)
        bytes_ = int(lens.sum()) * h * per + b * rows * (2 * D * dt + 4)
        return {"bytes": bytes_, "flops": int(lens.sum()) * rows * 4 * D}
    if c["op"] == "evict":
        kept = _kept(c)
        moved = (lens - kept) * kept / np.maximum(lens, 1)
        return {"bytes": int(h * (8 * lens.sum() + 2 * (slot + 8) * moved.sum()) + 8 * b * h),
                "flops": int(h * lens.sum())}
    rows = b * c["rows"] if c["op"] == "append" else int(_kept(c).sum())
    bytes_ = rows * h * (2 * D * dt * 2 + slot + 8 + 4)
    return {"bytes": bytes_, "flops": rows * h * 2 * D * 6}


def exact(case, seed):
    """In 64 bits: the attention over the values that the codes stand for, a
    unit at a time; the values of quantised rows; the weights that an eviction
    leaves, by a full sort of each unit."""
    c = case
    st = prepare(case, seed)
    b, h, cap = st["b"], st["h"], st["cap"]

    def stored(part, s, g, n):
        raw = st[part + "_codes"][s, g, :n].to(torch.int64)
        nib = torch.empty((n, D), dtype=torch.float64, device="cuda")
        nib[:, 0::2], nib[:, 1::2] = (raw % 16).double(), (raw // 16).double()
        par = st[part + "_params"][s, g, :n].double()
        return nib * par[:, :4].repeat_interleave(GR, 1) + par[:, 4:].repeat_interleave(GR, 1)

    if c["op"] == "attend":
        q = st["q"].double()
        n, group = q.shape[2], st["hq"] // h
        out = torch.zeros_like(q)
        lse = torch.full(q.shape[:3], -math.inf, dtype=torch.float64, device="cuda")
        wt = st["weights"].double()
        for s in range(b):
            for g in range(h):
                used = int(st["lengths"][s, g])
                kk, vv = stored("k", s, g, used), stored("v", s, g, used)
                for i in range(g * group, (g + 1) * group):
                    z = (q[s, i] @ kk.T) * D ** -0.5
                    if "q_positions" in st:
                        late = st["positions"][s, g, :used][None, :] > st["q_positions"][s][:, None]
                        z[late] = -math.inf
                    lse[s, i] = torch.logsumexp(z, -1)
                    p = torch.nan_to_num(torch.exp(z - lse[s, i][:, None]), nan=0.0)
                    out[s, i] = p @ vv
                    wt[s, g, :used] += p.sum(0)
        return {"out": out, "lse": lse, "weights": wt} if c["weights"] else {"out": out, "lse": lse}
    if c["op"] == "evict":
        wt = st["weights"].double().cpu().numpy()
        pos, lens = st["positions"].cpu().numpy(), st["lengths"].cpu().numpy()
        left = st["budgets"].cpu().numpy()
        for s in range(b):
            for g in range(h):
                n, k = int(lens[s, g]), int(left[s, g])
                p, w = pos[s, g, :n], wt[s, g, :n].copy()
                w[(p < c["sinks"]) | (p > p.max() - c["recent"])] = np.inf
                keep = np.zeros(n, bool)
                keep[np.argsort(-w, kind="stable")[:k]] = True
                to = np.flatnonzero(~keep[:k])
                wt[s, g, to] = wt[s, g, k + np.flatnonzero(keep[k:])]
        return {"k_words": None, "v_words": None, "k_params": None, "v_params": None,
                "positions": None, "lengths": None, "weights": torch.from_numpy(wt)}

    def quantised(x):
        y = x.double().reshape(-1, D // GR, GR)
        least = y.amin(-1, keepdim=True)
        m = least.float().view(torch.int32)  # bf16 inputs are their own; f16 round down
        cut = m & -65536
        cut = torch.where((m < 0) & (cut != m), cut + 65536, cut).view(torch.float32)
        spread = y.amax(-1, keepdim=True).float() - cut
        # a bf16 number close below the scale, then up to it in single steps
        s = (spread / 15 * 0.99).view(torch.int32) & -65536
        for _ in range(6):
            s = torch.where(s.view(torch.float32).double() * 15 < spread.double(), s + 65536, s)
        s = s.view(torch.float32).double()
        n = torch.round((y.float() - cut).double() / torch.where(s > 0, s, 1.0))
        return (n * s + cut.double()).view(x.shape)

    k, v = st["k"], st["v"]
    if c["op"] == "gather":
        row = np.arange(st["indices"].shape[1])
        seq = np.searchsorted(st["cu_out"], row, side="right") - 1
        at = torch.from_numpy(st["cu"][seq].astype(np.int64)).cuda()[:, None] + st["indices"].T.long()
        head = torch.arange(h, device="cuda")
        k, v = k[at, head], v[at, head]
    return {"k": quantised(k), "v": quantised(v), "k_words": None, "v_words": None, "k_params": None,
            "v_params": None, "positions": None, "lengths": None}
