"""The paged-cache operators written out in 64 bits on the CPU, one sequence and head at a time, and makers of
batches whose pages lie anywhere."""
import math
import random

import torch

D = 128


def inv_freq(spec):
    R = spec.rotary_dim
    out = []
    for i in range(R // 2):
        b = spec.theta ** (-2.0 * i / R)
        if spec.scaling == "linear":
            b = b / spec.factor
        elif spec.scaling == "banded":
            wave = 2 * math.pi / b
            if wave < spec.orig_len / spec.high:
                pass
            elif wave > spec.orig_len / spec.low:
                b = b / spec.factor
            else:
                t = (spec.orig_len / wave - spec.low) / (spec.high - spec.low)
                b = (1 - t) * b / spec.factor + t * b
        elif spec.scaling == "yarn":
            d = lambda n: R * math.log(spec.orig_len / (2 * math.pi * n)) / (2 * math.log(spec.theta))  # noqa: E731
            lo, hi = max(math.floor(d(spec.high)), 0), min(math.ceil(d(spec.low)), R - 1)
            r = min(1.0, max(0.0, (i - lo) / max(hi - lo, 0.001)))
            b = r * b / spec.factor + (1 - r) * b
        out.append(b)
    return out


def attn_factor(spec):
    if spec.attn_factor > 0:
        return spec.attn_factor
    return 0.1 * math.log(spec.factor) + 1.0 if spec.scaling == "yarn" else 1.0


def rope(x, positions, spec, transposed=False):
    """(turned x in 64 bits, bound on what 32-bit arithmetic may be off by before the rounding)."""
    x = x.double()
    out, slack = x.clone(), torch.zeros_like(x)
    m, R = attn_factor(spec), spec.rotary_dim
    for i, f in enumerate(inv_freq(spec)):
        a, b = (2 * i, 2 * i + 1) if spec.interleaved else (i, i + R // 2)
        ang = positions.double()[:, None] * f
        c, s = torch.cos(ang), torch.sin(ang) * (-1 if transposed else 1)
        out[..., a] = m * (x[..., a] * c - x[..., b] * s)
        out[..., b] = m * (x[..., b] * c + x[..., a] * s)
        # cosine and sine: the turn's fraction rounded to 32 bits (2^-25 of a turn: 2^-22.3), the function's and the
        # factor's roundings (2^-22), two products and a sum (2^-23): together below 2^-20 of |a| + |b|
        slack[..., a] = slack[..., b] = m * (x[..., a].abs() + x[..., b].abs()) * 2.0 ** -20
    return out, slack


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def assert_rounded(got, want, slack, what=""):
    u = half_step(got.dtype)
    tiny = torch.finfo(got.dtype).tiny * u                  # subnormal results: half a step of the least one
    bound = u * (want.abs() + slack) + slack + tiny
    err = (got.double().cpu() - want).abs()
    assert bool((err <= bound).all()), (what, float((err / bound).max()))


class Batch:
    """Random lengths, tables and pools on the CPU; .gpu() gives the tensors and the library's batch."""

    def __init__(self, q_len, kv_len, page, n_kv, n_q, dtype=torch.bfloat16, seed=0, spare=3, wide=0, garbage=True,
                 tail_tokens=0, joint=False):
        g = torch.Generator().manual_seed(seed)
        r = random.Random(seed)
        self.q_len, self.kv_len_list, self.page, self.n_kv, self.n_q, self.dtype = q_len, kv_len, page, n_kv, n_q, dtype
        n = len(q_len)
        blocks = [-(-k // page) for k in kv_len]
        self.n_pages = sum(blocks) + spare
        pages = list(range(self.n_pages))
        r.shuffle(pages)
        width = max(blocks + [1]) + wide
        self.table = torch.full((n, width), 2 ** 30 if garbage else 0, dtype=torch.int32)   # entries behind the rows: anything
        at = 0
        for i, b in enumerate(blocks):
            self.table[i, :b] = torch.tensor(pages[at:at + b], dtype=torch.int32)
            at += b
        self.free = pages[at:]
        starts = [0]
        for m in q_len:
            starts.append(starts[-1] + m)
        self.starts = starts
        self.n_tokens = starts[-1] + tail_tokens
        self.max_q = max(q_len + [0])
        self.q_start = torch.tensor(starts, dtype=torch.int32)
        self.kv_len = torch.tensor(kv_len, dtype=torch.int32)
        if joint:                                            # keys and values of a page next to each other
            kv = torch.randn(self.n_pages, 2, page, n_kv, D, generator=g).to(dtype)
            self.k_pool, self.v_pool = kv[:, 0], kv[:, 1]
        else:
            self.k_pool = torch.randn(self.n_pages, page, n_kv, D, generator=g).to(dtype)
            self.v_pool = torch.randn(self.n_pages, page, n_kv, D, generator=g).to(dtype)
        self.w_pool = torch.rand(self.n_pages, n_kv, page, generator=g)
        self.q = torch.randn(self.n_tokens, n_q, D, generator=g).to(dtype)
        self.k = torch.randn(self.n_tokens, n_kv, D, generator=g).to(dtype)
        self.v = torch.randn(self.n_tokens, n_kv, D, generator=g).to(dtype)
        self.pos = torch.randint(0, 1 << 20, (self.n_tokens,), generator=g, dtype=torch.int32)
        self.joint = joint

    def slots(self, i):
        t = torch.arange(self.kv_len_list[i])
        return self.table[i, t // self.page].long(), t % self.page

    def poison(self):
        """NaN and infinities wherever no sequence has a row."""
        held = torch.zeros(self.n_pages, self.page, dtype=torch.bool)
        for i in range(len(self.q_len)):
            held[self.slots(i)] = True
        for pool, bad in ((self.k_pool, math.nan), (self.v_pool, math.inf)):
            pool[~held] = bad
        self.v_pool[:, ::2][~held[:, ::2]] = math.nan
        return self

    def gpu(self, engine):
        out = {n: getattr(self, n).cuda() for n in ("q_start", "kv_len", "table", "w_pool", "q", "k", "v", "pos")}
        if self.joint:
            kv = torch.stack([self.k_pool, self.v_pool], dim=1).cuda()
            out["k_pool"], out["v_pool"] = kv[:, 0], kv[:, 1]
        else:
            out["k_pool"], out["v_pool"] = self.k_pool.cuda(), self.v_pool.cuda()
        out["batch"] = engine.batch(out["q_start"], out["kv_len"], out["table"], self.n_tokens, self.max_q)
        return out


def _logits(b, i, h, q):
    """(logits [new, kv] with -inf where hidden, bound on a 32-bit logit's error)."""
    pg, row = b.slots(i)
    g = h // (b.n_q // b.n_kv)
    k = b.k_pool[pg, row, g].double()
    x = q[b.starts[i]:b.starts[i + 1], h].double()
    s = x @ k.T / math.sqrt(D)
    m, kv = x.shape[0], k.shape[0]
    hidden = torch.arange(kv)[None, :] > torch.arange(kv - m, kv)[:, None]
    # 128 products summed in 32 bits: each partial sum is off by at most 2^-24 of the sum of their sizes, the scale
    # and the conversion to powers of two add a few more steps
    size = (x.abs() @ k.abs().T / math.sqrt(D))
    slack = size.amax(dim=1) * 136 * 2.0 ** -24 if kv else torch.zeros(m, dtype=torch.float64)
    return s.masked_fill(hidden, -math.inf), slack, (pg, row, g)


def attention(b, q=None):
    """out, lse in 64 bits and the bounds on their errors; tokens of no sequence: NaN in `out`'s place."""
    q = b.q if q is None else q
    u = half_step(b.dtype)
    out = torch.full((b.n_tokens, b.n_q, D), math.nan, dtype=torch.float64)
    lse = torch.full((b.n_tokens, b.n_q), math.nan, dtype=torch.float64)
    tol_o, tol_l = torch.zeros_like(out), torch.zeros_like(lse)
    for i in range(len(b.q_len)):
        rows = slice(b.starts[i], b.starts[i + 1])
        for h in range(b.n_q):
            s, slack, (pg, row, g) = _logits(b, i, h, q)
            z = torch.logsumexp(s, dim=1) if s.shape[1] else torch.full((s.shape[0],), -math.inf, dtype=torch.float64)
            p = torch.where(torch.isneginf(z)[:, None], 0.0, torch.exp(s - z[:, None]))
            v = b.v_pool[pg, row, g].double()
            o = p @ v if s.shape[1] else torch.zeros(s.shape[0], D, dtype=torch.float64)
            out[rows, h], lse[rows, h] = o, z
            # probabilities: rounded once (u), logits off by `slack` in numerator and denominator, exponentials by
            # 2^-21; the output rounded once (u).  In fp16 a probability below its normal range is off by up to 2^-25
            # of the running maximum's, whose own is at least 2^-8.
            pv = p @ v.abs() if s.shape[1] else torch.zeros_like(o)
            rel = u + 2 * (slack + 2.0 ** -21) + 2.0 ** -20
            tol_o[rows, h] = u * o.abs() + rel[:, None] * pv * (1 + u) + 1e-30
            if b.dtype == torch.float16 and s.shape[1]:
                tol_o[rows, h] += 2.0 ** -25 * v.abs().sum(dim=0)[None, :] * p.amax(dim=1, keepdim=True)
                tol_o[rows, h] += 2.0 ** -25
            tol_l[rows, h] = slack + 2.0 ** -20 * (1 + torch.where(torch.isfinite(z), z.abs(), 0.0))
    return out, lse, tol_o, tol_l


def accumulate(b, lse, q=None):
    """w_pool after the call and the bound on its error; lse: 32-bit values as given."""
    q = b.q if q is None else q
    w, tol = b.w_pool.double().clone(), torch.zeros(b.w_pool.shape, dtype=torch.float64)
    tol += 2.0 ** -23 * w
    for i in range(len(b.q_len)):
        for h in range(b.n_q):
            s, slack, (pg, row, g) = _logits(b, i, h, q)
            given = lse[b.starts[i]:b.starts[i + 1], h].double()[:, None]
            p = torch.where(torch.isneginf(given) | torch.isneginf(s), 0.0, torch.exp(s - given))
            # logits off by `slack`, the exponent's rounding 2^-24 of its parts, the exponential 2^-21; then a sum of
            # up to (new tokens x heads) terms in 32 bits
            part = torch.where(torch.isfinite(given), given.abs(), 0.0) + torch.where(torch.isfinite(s), s.abs(), 0.0)
            rel = slack[:, None] + 2.0 ** -22 * part + 2.0 ** -20
            rel = rel + 2.0 ** -24 * (s.shape[0] * (b.n_q // b.n_kv) + 8)
            w.index_put_((pg, torch.full_like(pg, g), row), p.sum(dim=0), accumulate=True)
            tol.index_put_((pg, torch.full_like(pg, g), row), (p * rel).sum(dim=0) + 2.0 ** -23 * p.sum(dim=0), accumulate=True)
    return w, tol


def evict_choice(b, budget, n_sink, n_recent, per_head):
    """Kept rows [seq][list] ascending."""
    kept = []
    for i in range(len(b.kv_len_list)):
        kv = b.kv_len_list[i]
        pg, row = b.slots(i)
        w = b.w_pool[pg, :, row]                             # [kv, n_kv]
        lists = [w[:, g] for g in range(b.n_kv)] if per_head else [w.double().sum(dim=1).float()]
        mine = []
        for key in lists:
            if kv <= budget:
                mine.append(list(range(kv)))
                continue
            mid = sorted(range(n_sink, kv - n_recent), key=lambda t: (-float(key[t]), t))[:budget - n_sink - n_recent]
            mine.append(list(range(n_sink)) + sorted(mid) + list(range(kv - n_recent, kv)))
        kept.append(mine)
    return kept
