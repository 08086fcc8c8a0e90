"""Timed cases of the paged-cache operators: what a serving program calls between the compressed
prompt and its answer, over the range of sizes it calls it with.

Five calls, all on one page pool (``[n_pages, page_size, n_kv_heads, 128]`` keys and values, block
tables, ragged batches):

* ``rope``        rotary positions of a tensor of heads (``rope``);
* ``append``      rotary positions of new queries and keys, and the new rows' way into the cache
                  (``PagedCache.append``);
* ``attention``   new tokens over the cache, chunks and single tokens (``PagedCache.attention``);
* ``accumulate``  the attention weight that each cached row receives (``PagedCache.accumulate``);
* ``evict``       the rows of the largest weight kept, the cache compacted (``PagedCache.evict``).

Inputs are made on the GPU from the seed: N(0, 1) rows, one in fifty keys along a direction that
the queries of its head group lean to (so that some rows gather weight), pages in random order.
"""
from __future__ import annotations

import math
import random

import torch

own = False

D = 128                                   # head dimension
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
ROPES = {                                 # theta, rotary_dim, interleaved, scaling, factor, orig_len, low, high
    "plain": (500000.0, 128, False, "none", 1.0, 0, 0.0, 0.0),
    "banded": (500000.0, 128, False, "banded", 8.0, 8192, 1.0, 4.0),
    "yarn": (10000.0, 128, False, "yarn", 32.0, 4096, 1.0, 32.0),
    "part": (10000.0, 64, True, "yarn", 16.0, 4096, 1.0, 32.0),
}


def _case(name, **kw):
    return dict(kw, name=name) if name else kw


def _rope(name, tokens, heads, spec, dtype="bf16", transposed=False):
    return _case(name, op="rope", tokens=tokens, n_q=heads, spec=spec, dtype=dtype, transposed=transposed)


def _batch(name, op, seqs, q_lo, q_hi, kv_lo, kv_hi, page, n_kv=8, n_q=32, dtype="bf16", **more):
    """q_lo..q_hi new tokens per sequence and kv_lo..kv_hi cached rows before them."""
    return _case(name, op=op, seqs=seqs, q_lo=q_lo, q_hi=q_hi, kv_lo=kv_lo, kv_hi=kv_hi, page=page, n_kv=n_kv,
                 n_q=n_q, dtype=dtype, **more)


def listed():
    return [
        # One decoding step of 32 requests: a few hundred KB, the launch counts.
        _rope("rope_step", 32, 32, "plain"),
        # Queries of a 16384-token chunk, half of the head rotated, scaled for a long context; the
        # transposed form is the gradient's.
        _rope("rope_chunk_16k", 16384, 32, "part", dtype="fp16", transposed=True),
        # The same step with the new rows' way into the cache, behind compressed prompts of some 4100 rows.
        _batch("append_step", "append", 32, 1, 1, 4100, 4700, 64, spec="banded"),
        # A ragged prefill of four compressed prompts.
        _batch("append_prompts", "append", 4, 3500, 4416, 0, 0, 16, spec="yarn"),
        # One request decodes behind its compressed prompt (4096 recalled positions, a 64-token question).
        _batch("attend_step", "attention", 1, 1, 1, 4160, 4160, 64),
        # 64 requests decode, each behind its own length.
        _batch("attend_step_64", "attention", 64, 1, 1, 1500, 16000, 16),
        # A 1024-token chunk of a prompt behind 32768 cached rows.
        _batch("attend_chunk_32k", "attention", 1, 1024, 1024, 31744, 31744, 128),
        # Compressed prompts come in while others decode; another head layout, the other type.
        _batch("attend_mixed", "attention", 12, 1, 700, 0, 4400, 32, 4, 28, "fp16"),
        # The weights of a decoding step of eight long requests, and of a whole compressed prompt.
        _batch("weigh_step_8", "accumulate", 8, 1, 1, 20000, 32768, 64),
        _batch("weigh_prompt", "accumulate", 1, 4160, 4160, 0, 0, 64),
        # One request back to its budget after 512 decoded tokens, every kv head on its own; a batch of
        # prompts cut to 4096 rows each, the heads together.
        _batch("evict_one", "evict", 1, 1, 1, 4607, 4607, 64, budget=4096, sink=4, recent=512, per_head=True),
        _batch("evict_prompts_16", "evict", 16, 1, 1, 6000, 14000, 16, budget=4096, sink=4, recent=64, per_head=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "append", "attention", "attention", "accumulate", "evict"])
    n_kv, n_q = rng.choice([(8, 32), (8, 32), (4, 28), (2, 16), (8, 8)])
    page = rng.choice([16, 32, 64, 128])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    if op == "rope":
        return _rope(None, _log_int(rng, 1, 16384), n_q, rng.choice(list(ROPES)), dtype, rng.random() < 0.5)
    if op == "append":
        hi = _log_int(rng, 1, 4000)
        return _batch(None, op, rng.randint(1, max(1, min(64, 16000 // hi))), rng.choice([1, hi]), hi, 0,
                      _log_int(rng, 1, 6000), page, n_kv, n_q, dtype, spec=rng.choice(list(ROPES)))
    if op == "evict":
        hi, budget = _log_int(rng, 600, 14000), _log_int(rng, 64, 4096)
        return _batch(None, op, rng.randint(1, 16), 1, 1, max(1, hi // 2), hi, page, n_kv, n_q, dtype, budget=budget,
                      sink=rng.choice([0, 4]), recent=min(budget - 4, rng.choice([0, 32, 512])),
                      per_head=rng.random() < 0.5)
    if rng.random() < 0.5:                                  # a decoding step
        hi = _log_int(rng, 1, 32000)
        return _batch(None, op, rng.randint(1, max(1, min(64, 500000 // hi))), 1, rng.choice([1, 1, 2, 4]), hi // 3, hi,
                      page, n_kv, n_q, dtype)
    hi, kv = _log_int(rng, 2, 2048), _log_int(rng, 1, 16000)
    seqs = rng.randint(1, max(1, min(12, 6000000 // (hi * (hi + kv)))))
    return _batch(None, op, seqs, rng.choice([1, hi]), hi, rng.choice([0, kv]), kv, page, n_kv, n_q, dtype)


def _lengths(case):
    """(new tokens, cached rows with them) of each sequence: of the sizes alone, whatever the seed."""
    r = random.Random(1234)
    q = [r.randint(case["q_lo"], case["q_hi"]) for _ in range(case["seqs"])]
    q[0] = case["q_hi"]
    return q, [n + r.randint(case["kv_lo"], case["kv_hi"]) for n in q]


def _inv_freq(spec):
    theta, R, _, scaling, factor, orig, low, high = ROPES[spec]
    f = [theta ** (-2.0 * i / R) for i in range(R // 2)]
    if scaling == "none":
        return f, 1.0
    if scaling == "banded":
        g = []
        for x in f:
            wave = 2 * math.pi / x
            t = min(1.0, max(0.0, (orig / wave - low) / (high - low)))
            g.append((1 - t) * x / factor + t * x)
        return g, 1.0
    d = [R * math.log(orig / (2 * math.pi * b)) / (2 * math.log(theta)) for b in (high, low)]
    lo, hi = max(math.floor(d[0]), 0), min(math.ceil(d[1]), R - 1)
    ramp = [min(1.0, max(0.0, (i - lo) / max(hi - lo, 0.001))) for i in range(R // 2)]
    return [x / factor * t + x * (1 - t) for x, t in zip(f, ramp)], 0.1 * math.log(factor) + 1.0


def prepare(case, seed):
    dev = torch.device("cuda", 0)
    g = torch.Generator(device=dev).manual_seed(seed)
    r = random.Random(seed)
    dt = DTYPES[case["dtype"]]
    randn = lambda *n: torch.randn(*n, generator=g, device=dev)  # noqa: E731
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    s = {"case": case}
    if case["op"] in ("rope", "append"):
        f, s["m"] = _inv_freq(case["spec"])
        s["freq"] = torch.tensor(f, dtype=torch.float64, device=dev)
        if own:
            from paper_2508_17892_b200 import RopeSpec
            theta, R, inter, scaling, factor, orig, low, high = ROPES[case["spec"]]
            s["spec"] = RopeSpec(theta=theta, rotary_dim=R, interleaved=inter, scaling=scaling, factor=factor,
                                 orig_len=orig, low=low, high=high)
    if case["op"] == "rope":
        n = case["tokens"]
        s["x"] = randn(n, case["n_q"], D).to(dt)
        s["pos"] = ints(sorted(r.sample(range(131072), n)))
        s["out"] = torch.empty_like(s["x"])
        return s
    q_len, kv_len = _lengths(case)
    n, n_kv, n_q, page = case["seqs"], case["n_kv"], case["n_q"], case["page"]
    blocks = [-(-k // page) for k in kv_len]
    width = max(blocks)
    budget = case.get("budget", 0)
    dst_width = -(-budget // page)
    n_pages = sum(blocks) + n * dst_width
    order = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)
    at, table = 0, torch.zeros(n, width, dtype=torch.int32, device=dev)
    for i, b in enumerate(blocks):
        table[i, :b] = order[at:at + b]
        at += b
    s["table"] = table
    if budget:
        s["dst"] = order[at:].view(n, dst_width).contiguous()
    starts = [0]
    for v in q_len:
        starts.append(starts[-1] + v)
    s["q_start"], s["kv_len"], s["n_tokens"], s["max_q"] = ints(starts), ints(kv_len), starts[-1], max(q_len)
    lean = randn(n_kv, D)
    lean = lean / lean.norm(dim=-1, keepdim=True)
    s["k_pool"] = torch.empty(n_pages, page, n_kv, D, dtype=dt, device=dev)
    s["v_pool"] = torch.empty_like(s["k_pool"])
    step = max(1, 65536 // page)
    for p0 in range(0, n_pages, step):                      # in pieces: 32-bit normals of a large pool take room
        m = min(step, n_pages - p0)
        hot = (torch.rand(m, page, n_kv, 1, generator=g, device=dev) < 0.02).float()
        s["k_pool"][p0:p0 + m] = (randn(m, page, n_kv, D) + 8.0 * hot * lean).to(dt)
        s["v_pool"][p0:p0 + m] = randn(m, page, n_kv, D).to(dt)
    q = randn(s["n_tokens"], n_kv, n_q // n_kv, D) + 4.0 * lean[:, None]
    s["q"] = q.view(s["n_tokens"], n_q, D).to(dt)
    if case["op"] == "append":
        s["k"], s["v"] = randn(s["n_tokens"], n_kv, D).to(dt), randn(s["n_tokens"], n_kv, D).to(dt)
        s["pos"] = torch.cat([torch.arange(k - m, k, device=dev) for m, k in zip(q_len, kv_len)]).to(torch.int32)
        s["q_out"] = torch.empty_like(s["q"])
    if case["op"] == "attention":
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros(s["n_tokens"], n_q, device=dev)
    if case["op"] in ("accumulate", "evict"):
        w = torch.rand(n_pages, n_kv, page, generator=g, device=dev)
        s["w_pool"] = w * w * w * w                         # few rows with much, many with little
    if case["op"] == "accumulate":
        s["lse"] = _attend(s, weights=False)[1]
    if own:
        from paper_2508_17892_b200 import PagedCache
        s["engine"] = PagedCache(n_kv_heads=n_kv, n_q_heads=n_q, page_size=page, dtype=dt, max_seqs=n)
        s["batch"] = s["engine"].batch(s["q_start"], s["kv_len"], s["table"], s["n_tokens"], s["max_q"])
    return s


def run(s):
    case = s["case"]
    return (_own if own else _plain)[case["op"]](s)


# -- the framework's calls ---------------------------------------------------------------

def _own_rope(s):
    from paper_2508_17892_b200 import rope
    return rope(s["x"], s["pos"], s["spec"], transposed=s["case"]["transposed"], out=s["out"])


def _own_append(s):
    q = s["engine"].append(s["batch"], s["q"], s["k"], s["v"], s["pos"], s["spec"], s["k_pool"], s["v_pool"],
                           q_out=s["q_out"])
    return {"q": q, "k": s["k_pool"], "v": s["v_pool"]}


def _own_attention(s):
    out, lse = s["engine"].attention(s["batch"], s["q"], s["k_pool"], s["v_pool"], out=s["out"], lse=s["lse"])
    return {"out": out, "lse": lse}


def _own_accumulate(s):
    return s["engine"].accumulate(s["batch"], s["q"], s["lse"], s["k_pool"], s["w_pool"])


def _own_evict(s):
    c = s["case"]
    kept, new_len = s["engine"].evict(s["batch"], c["budget"], c["sink"], c["recent"], s["k_pool"], s["v_pool"],
                                      s["w_pool"], per_head=c["per_head"], dst_table=s["dst"])
    return {"kept": kept, "len": new_len, "k": s["k_pool"], "v": s["v_pool"], "w": s["w_pool"]}


_own = {"rope": _own_rope, "append": _own_append, "attention": _own_attention, "accumulate": _own_accumulate,
        "evict": _own_evict}


# -- the plain forms ---------------------------------------------------------------------

def _rotate(x, pos, freq, m, spec, transposed=False):
    R, inter = ROPES[spec][1], ROPES[spec][2]
    ang = pos.double()[:, None] * freq                      # far positions: the angle needs 64 bits
    cos, sin = (m * torch.cos(ang)).float()[:, None], (m * torch.sin(ang)).float()[:, None]
    sin = -sin if transposed else sin
    y = x.float()
    a, b = (y[..., 0:R:2], y[..., 1:R:2]) if inter else (y[..., :R // 2], y[..., R // 2:R])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([a, b], dim=-1).flatten(-2) if inter else torch.cat([a, b], dim=-1)
    return torch.cat([turned, y[..., R:]], dim=-1).to(x.dtype)


def _token_seq(s):
    """The sequence of each token and its place among the sequence's new ones."""
    t = torch.arange(s["n_tokens"], device=s["q_start"].device)
    seq = torch.searchsorted(s["q_start"][1:].long(), t, right=True)
    return seq, t - s["q_start"].long()[seq]


def _plain_rope(s):
    c = s["case"]
    return _rotate(s["x"], s["pos"], s["freq"], s["m"], c["spec"], c["transposed"])


def _plain_append(s):
    c = s["case"]
    seq, j = _token_seq(s)
    n_new = (s["q_start"][1:] - s["q_start"][:-1]).long()
    slot = s["kv_len"].long()[seq] - n_new[seq] + j
    page, row = s["table"].long()[seq, slot // c["page"]], slot % c["page"]
    s["k_pool"][page, row] = _rotate(s["k"], s["pos"], s["freq"], s["m"], c["spec"])
    s["v_pool"][page, row] = s["v"]
    return {"q": _rotate(s["q"], s["pos"], s["freq"], s["m"], c["spec"]), "k": s["k_pool"], "v": s["v_pool"]}


def _padded(s):
    """Queries [n, h_kv, group * max_q, D], keys of each sequence [n, kv, h_kv, D], who sees what [n, max_q, kv]."""
    c, n = s["case"], s["case"]["seqs"]
    n_kv, group, max_q = c["n_kv"], c["n_q"] // c["n_kv"], s["max_q"]
    seq, j = _token_seq(s)
    q = torch.zeros(n, max_q, n_kv, group, D, device=s["q"].device)
    q[seq, j] = s["q"].float().view(-1, n_kv, group, D)
    k = s["k_pool"][s["table"].long()].view(n, -1, n_kv, D)
    n_new = (s["q_start"][1:] - s["q_start"][:-1]).long()
    limit = (s["kv_len"].long() - n_new)[:, None] + torch.arange(max_q, device=q.device)
    sees = torch.arange(k.shape[1], device=q.device) <= limit[..., None]
    return q, k.float(), sees, seq, j


def _attend(s, weights):
    """(output or the probabilities' column sums, lse) of the batch."""
    c, n = s["case"], s["case"]["seqs"]
    n_kv, group = c["n_kv"], c["n_q"] // c["n_kv"]
    q, k, sees, seq, j = _padded(s)
    x = torch.einsum("njghd,nkgd->ngjhk", q, k)
    x = x.mul_(1.0 / math.sqrt(D)).masked_fill_(~sees[:, None, :, None], -math.inf)
    if weights:
        lse = torch.full((n, s["max_q"], c["n_q"]), math.inf, device=q.device)
        lse[seq, j] = torch.where(s["lse"] == -math.inf, math.inf, s["lse"])
        x = x.sub_(lse.view(n, s["max_q"], n_kv, group).transpose(1, 2)[..., None]).exp_()
        return x.sum(dim=(2, 3)), s["lse"]
    top = x.amax(dim=-1, keepdim=True).clamp_min_(torch.finfo(torch.float32).min)
    p = x.sub_(top).exp_()
    total = p.sum(dim=-1, keepdim=True)
    lse = (top + total.log())[..., 0].transpose(1, 2).reshape(n, s["max_q"], c["n_q"])[seq, j]
    if "out" not in s:
        return None, lse
    v = s["v_pool"][s["table"].long()].view(n, -1, n_kv, D).float()
    o = torch.einsum("ngjhk,nkgd->njghd", p, v)
    o = o / total.clamp_min(1e-38).squeeze(-1).transpose(1, 2)[..., None]
    return o.reshape(n, s["max_q"], c["n_q"], D)[seq, j], lse


def _plain_attention(s):
    out, lse = _attend(s, weights=False)
    return {"out": out.to(s["q"].dtype), "lse": lse}


def _plain_accumulate(s):
    c = s["case"]
    sums, _ = _attend(s, weights=True)                      # [n, n_kv, kv]
    n, width = s["table"].shape
    held = torch.arange(width, device=sums.device) * c["page"] < s["kv_len"][:, None]
    pages = s["table"].long()[held]
    s["w_pool"][pages] += sums.view(n, c["n_kv"], width, c["page"]).transpose(1, 2)[held]
    return s["w_pool"]


def _plain_evict(s):
    c, n, B = s["case"], s["case"]["seqs"], s["case"]["budget"]
    table, dev = s["table"].long(), s["table"].device
    w = s["w_pool"][table].transpose(1, 2).reshape(n, c["n_kv"], -1)
    key = w if c["per_head"] else w.double().sum(dim=1, keepdim=True).float()
    t = torch.arange(key.shape[2], device=dev)
    kv = s["kv_len"].long()[:, None, None]
    key = torch.where((t < c["sink"]) | (t >= kv - c["recent"]), math.inf, key)
    key = torch.where(t < kv, key, -math.inf)
    new_len = s["kv_len"].clamp(max=B)
    order = torch.sort(key, dim=-1, descending=True, stable=True).indices[..., :B]
    valid = torch.arange(B, device=dev) < new_len[:, None, None]
    if order.shape[2] < B:
        order = torch.cat([order, order.new_zeros(n, order.shape[1], B - order.shape[2])], dim=2)
    kept = torch.where(valid, order, key.shape[2]).sort(dim=-1).values
    from_slot = torch.where(valid, kept, 0).expand(n, c["n_kv"], B)
    i, h, b = torch.nonzero(valid.expand(n, c["n_kv"], B), as_tuple=True)
    src = from_slot[i, h, b]
    sp, sr = table[i, src // c["page"]], src % c["page"]
    dp, dr = s["dst"].long()[i, b // c["page"]], b % c["page"]
    s["k_pool"][dp, dr, h] = s["k_pool"][sp, sr, h]
    s["v_pool"][dp, dr, h] = s["v_pool"][sp, sr, h]
    s["w_pool"][dp, h, dr] = s["w_pool"][sp, h, sr]
    return {"kept": torch.where(valid, kept, -1).to(torch.int32), "len": new_len, "k": s["k_pool"], "v": s["v_pool"],
            "w": s["w_pool"]}


_plain = {"rope": _plain_rope, "append": _plain_append, "attention": _plain_attention,
          "accumulate": _plain_accumulate, "evict": _plain_evict}


# -- from the definitions, in 64 bits -----------------------------------------------------

def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if case["op"] == "evict":
        return None                                         # positions and moved rows: nothing is computed
    if case["op"] in ("rope", "append"):
        R, inter = ROPES[case["spec"]][1], ROPES[case["spec"]][2]
        f, m = _inv_freq(case["spec"])
        first = [2 * i if inter else i for i in range(R // 2)]
        second = [2 * i + 1 if inter else i + R // 2 for i in range(R // 2)]

        def turn(x, sign=1.0):
            ang = s["pos"].double()[:, None, None] * torch.tensor(f, dtype=torch.float64, device=x.device)
            y = x.double()
            a, b = y[..., first], y[..., second]
            y[..., first] = m * (a * torch.cos(ang) - sign * b * torch.sin(ang))
            y[..., second] = m * (b * torch.cos(ang) + sign * a * torch.sin(ang))
            return y

        if case["op"] == "rope":
            return turn(s["x"], -1.0 if case["transposed"] else 1.0)
    q_len, kv_len = _lengths(case)
    starts, table, page = s["q_start"].tolist(), s["table"].long(), case["page"]
    n_kv, group = case["n_kv"], case["n_q"] // case["n_kv"]
    if case["op"] == "append":
        k, v, kr, vr = s["k_pool"].double(), s["v_pool"].double(), turn(s["k"]), s["v"].double()
        for i, (m_new, kv) in enumerate(zip(q_len, kv_len)):
            slot = torch.arange(kv - m_new, kv, device=k.device)
            k[table[i, slot // page], slot % page] = kr[starts[i]:starts[i + 1]]
            v[table[i, slot // page], slot % page] = vr[starts[i]:starts[i + 1]]
        return {"q": turn(s["q"]), "k": k, "v": v}
    lse = torch.full((s["n_tokens"], case["n_q"]), -math.inf, dtype=torch.float64, device=table.device)
    out = torch.zeros(s["n_tokens"], case["n_q"], D, dtype=torch.float64, device=table.device)
    w = s["w_pool"].double() if case["op"] == "accumulate" else None
    for i, (m_new, kv) in enumerate(zip(q_len, kv_len)):
        slot = torch.arange(kv, device=table.device)
        pg, row = table[i, slot // page], slot % page
        for h in range(n_kv):
            k, heads = s["k_pool"][pg, row, h].double(), slice(h * group, (h + 1) * group)
            x = torch.einsum("jhd,kd->jhk", s["q"][starts[i]:starts[i + 1], heads].double(), k) / math.sqrt(D)
            hidden = slot[None, :] > torch.arange(kv - m_new, kv, device=slot.device)[:, None]
            x.masked_fill_(hidden[:, None], -math.inf)
            if w is not None:
                given = s["lse"][starts[i]:starts[i + 1], heads].double()[..., None]
                w[pg, h, row] += torch.exp(x - given).sum(dim=(0, 1))
                continue
            z = torch.logsumexp(x, dim=-1)
            lse[starts[i]:starts[i + 1], heads] = z
            out[starts[i]:starts[i + 1], heads] = torch.exp(x - z[..., None]) @ s["v_pool"][pg, row, h].double()
    return w if w is not None else {"out": out, "lse": lse}


def work(case):
    n_q = case["n_q"]
    if case["op"] == "rope":
        return {"bytes": case["tokens"] * (4 * n_q * D + 4), "flops": 3 * case["tokens"] * n_q * ROPES[case["spec"]][1]}
    q_len, kv_len = _lengths(case)
    n_kv, new, kv = case["n_kv"], sum(q_len), sum(kv_len)
    pairs = sum(m * (k - m) + m * (m + 1) // 2 for m, k in zip(q_len, kv_len))
    if case["op"] == "append":
        return {"bytes": new * (4 * n_q * D + 8 * n_kv * D + 4), "flops": 3 * new * (n_q + n_kv) * ROPES[case["spec"]][1]}
    if case["op"] == "attention":
        return {"bytes": new * n_q * (4 * D + 4) + 4 * kv * n_kv * D, "flops": 4 * pairs * n_q * D}
    if case["op"] == "accumulate":
        return {"bytes": new * n_q * (2 * D + 4) + kv * n_kv * (2 * D + 8), "flops": 2 * pairs * n_q * D}
    kept = sum(min(k, case["budget"]) for k in kv_len)
    rows = n_kv if case["per_head"] else 1
    return {"bytes": 4 * kv * n_kv + kept * n_kv * (8 * D + 8) + 4 * kept * rows, "flops": 0}
