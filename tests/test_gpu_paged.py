"""The paged-cache operators on the GPU against their definitions in 64 bits, through the Python entry points."""
import ctypes
import math

import pytest
import torch

import paged_reference as ref

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float16


def _engine(b, **kw):
    from paper_2508_17892_b200 import PagedCache
    return PagedCache(n_kv_heads=b.n_kv, n_q_heads=b.n_q, page_size=b.page, dtype=b.dtype,
                      max_seqs=max(1, len(b.q_len)), **kw)


def _close(eng):
    torch.cuda.synchronize()
    eng.check_status()
    assert eng.check_guards() == 0, "a kernel wrote past the end of a workspace buffer"
    eng.close()


# ---- rotary positions ---------------------------------------------------------------------------

def _spec(**kw):
    from paper_2508_17892_b200 import RopeSpec
    return RopeSpec(**kw)


SPECS = {
    "half": dict(),
    "interleaved": dict(interleaved=True, theta=10000.0),
    "part_half": dict(rotary_dim=64, theta=10000.0),
    "part_interleaved": dict(rotary_dim=32, interleaved=True),
    "linear": dict(scaling="linear", factor=4.0, theta=10000.0),
    "banded": dict(scaling="banded", factor=8.0, orig_len=8192, low=1.0, high=4.0),
    "yarn": dict(scaling="yarn", factor=32.0, orig_len=4096, low=1.0, high=32.0, theta=10000.0),
    "yarn_given": dict(scaling="yarn", factor=16.0, orig_len=4096, low=1.0, high=32.0, attn_factor=1.25, interleaved=True),
}


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("name", SPECS)
def test_rope_matches_64_bits(name, dtype, transposed):
    from paper_2508_17892_b200 import rope
    spec = _spec(**SPECS[name])
    g = torch.Generator().manual_seed(3)
    for n, heads in ((1, 1), (7, 5), (300, 8)):
        x = torch.randn(n, heads, 128, generator=g).to(dtype)
        pos = torch.randint(0, 1 << 21, (n,), generator=g, dtype=torch.int32)
        pos[0] = -5 if n > 1 else 2 ** 31 - 1
        got = rope(x.cuda(), pos.cuda(), spec, transposed=transposed)
        want, slack = ref.rope(x, pos, spec, transposed)
        ref.assert_rounded(got.cpu(), want, slack, name)


@pytest.mark.parametrize("dim,rotary", [(16, 16), (48, 32), (80, 80), (256, 256), (576, 64), (1024, 128)])
def test_rope_head_sizes_strides_and_in_place(dim, rotary):
    from paper_2508_17892_b200 import rope
    g = torch.Generator().manual_seed(dim)
    # 6000 tokens: more than one token to a CTA; a slice of a wider tensor, the rest left as it was
    for n in (1, 33, 6000 if dim <= 80 else 100):
        wide = torch.randn(n, 5, dim, generator=g).to(BF)
        pos = torch.randint(0, 100000, (n,), generator=g, dtype=torch.int32)
        spec = _spec(rotary_dim=rotary, interleaved=dim % 32 == 0)
        buf = wide.cuda()
        out = rope(buf[:, 1:4], pos.cuda(), spec, out=buf[:, 1:4])
        assert out.data_ptr() == buf[:, 1:4].data_ptr()
        want, slack = ref.rope(wide[:, 1:4], pos, spec)
        ref.assert_rounded(buf[:, 1:4].cpu(), want, slack)
        assert torch.equal(buf[:, 0].cpu(), wide[:, 0]) and torch.equal(buf[:, 4].cpu(), wide[:, 4])


def test_rope_transposed_is_the_gradient():
    """<y, rope(x)> is linear in x: its derivative by x is rope(y, transposed), by the formula and by differences."""
    from paper_2508_17892_b200 import rope
    g = torch.Generator().manual_seed(9)
    spec = _spec(**SPECS["yarn_given"])
    x, y = (torch.randn(5, 3, 128, generator=g).to(FP) for _ in range(2))
    pos = torch.arange(5, dtype=torch.int32) * 1000
    grad = rope(y.cuda(), pos.cuda(), spec, transposed=True).double().cpu()
    xd = x.double().requires_grad_()
    a, b = xd[..., 0::2], xd[..., 1::2]
    ang = pos.double()[:, None, None] * torch.tensor(ref.inv_freq(spec), dtype=torch.float64)
    turned = 1.25 * torch.stack([a * ang.cos() - b * ang.sin(), b * ang.cos() + a * ang.sin()], dim=-1).flatten(-2)
    (turned * y.double()).sum().backward()
    want, slack = ref.rope(y, pos, spec, True)
    assert torch.allclose(want, xd.grad, rtol=0, atol=1e-12)
    ref.assert_rounded(grad.to(FP), want, slack)
    step = torch.zeros_like(x)
    step[2, 1, 7] = 0.5
    # the outputs carry half a step each: 128 of them, sizes below 8
    diff = (rope((x + step).cuda(), pos.cuda(), spec).double() - rope(x.cuda(), pos.cuda(), spec).double()).cpu()
    fd = (diff * y.double()).sum() / float((x + step).double()[2, 1, 7] - x.double()[2, 1, 7])
    assert abs(float(fd) - float(want[2, 1, 7])) <= 2 * 2 * 2 * 8 * 2.0 ** -11 * float(y[2, 1, 6:8].double().abs().sum()) / 0.5


# ---- append -----------------------------------------------------------------------------------

APPEND = [
    # q_len, kv_len, page, n_kv, n_q, dtype, options
    ([1], [1], 16, 1, 1, BF, {}),
    ([3, 0, 1, 40], [70, 5, 1, 40], 16, 8, 32, BF, dict(tail_tokens=5)),
    ([130, 2], [200, 1030], 64, 4, 28, FP, dict(joint=True)),
    ([17], [17], 1024, 2, 8, BF, {}),
    ([5000, 300], [5200, 300], 128, 2, 4, BF, {}),
]


@pytest.mark.parametrize("case", APPEND, ids=range(len(APPEND)))
@pytest.mark.parametrize("name", ["banded", "part_interleaved", None])
def test_append_writes_the_new_rows_and_nothing_else(case, name):
    q_len, kv_len, page, n_kv, n_q, dtype, opt = case
    b = ref.Batch(q_len, kv_len, page, n_kv, n_q, dtype, seed=len(q_len), **opt)
    eng = _engine(b)
    t = b.gpu(eng)
    spec = _spec(**SPECS[name]) if name else None
    q_out = torch.full_like(t["q"], 7.0)
    eng.append(t["batch"], t["q"], t["k"], t["v"], t["pos"] if spec else None, spec, t["k_pool"], t["v_pool"], t["w_pool"],
               q_out=q_out)
    k_want, k_slack = ref.rope(b.k, b.pos, spec) if spec else (b.k.double(), torch.zeros(b.k.shape, dtype=torch.float64))
    q_want, q_slack = ref.rope(b.q, b.pos, spec) if spec else (b.q.double(), torch.zeros(b.q.shape, dtype=torch.float64))
    kp, vp, wp = b.k_pool.double(), b.v_pool.clone(), b.w_pool.clone()
    slack = torch.zeros_like(kp)
    for i, m in enumerate(q_len):
        pg, row = (x[kv_len[i] - m:] for x in b.slots(i))
        kp[pg, row], slack[pg, row] = k_want[b.starts[i]:b.starts[i + 1]], k_slack[b.starts[i]:b.starts[i + 1]]
        vp[pg, row] = b.v[b.starts[i]:b.starts[i + 1]]
        wp[pg, :, row] = 0.0
    ref.assert_rounded(t["k_pool"].cpu(), kp, slack)
    assert torch.equal(t["v_pool"].cpu(), vp) and torch.equal(t["w_pool"].cpu(), wp)
    n = b.starts[-1]
    ref.assert_rounded(q_out[:n].cpu(), q_want[:n], q_slack[:n])
    assert bool((q_out[n:] == 7.0).all()), "tokens of no sequence are left as they are"
    if spec:                                                 # in place, and without q and weights
        eng.append(t["batch"], t["q"], t["k"], t["v"], t["pos"], spec, t["k_pool"], t["v_pool"], q_out=t["q"])
        assert torch.equal(t["q"][:n], q_out[:n])
        eng.append(t["batch"], None, t["k"], t["v"], t["pos"], spec, t["k_pool"], t["v_pool"])
        assert torch.equal(t["w_pool"].cpu(), wp)
    _close(eng)


# ---- attention ---------------------------------------------------------------------------------

ATTEND = [
    # q_len, kv_len, page, n_kv, n_q, dtype, options
    ([1], [1], 16, 1, 1, BF, {}),
    ([1], [4160], 64, 8, 32, BF, {}),
    ([1, 1, 1, 1, 1], [64, 1, 129, 1000, 65], 16, 2, 8, BF, dict(tail_tokens=3)),
    ([1, 4, 2, 0, 3], [63, 300, 2, 77, 64], 32, 4, 16, FP, dict(wide=2)),
    ([2, 1], [500, 33], 128, 1, 16, BF, dict(joint=True)),
    ([1, 1], [200, 90], 256, 2, 14, FP, {}),                 # seven heads of a group
    ([5, 3], [40, 3], 16, 3, 9, BF, {}),                     # more rows than one tile of 16 has
    ([40], [40], 64, 2, 8, BF, {}),
    ([128, 7, 0, 300], [128, 400, 9, 811], 64, 4, 16, BF, dict(tail_tokens=2)),
    ([257, 130], [700, 131], 16, 2, 14, FP, {}),
    ([100, 33], [100, 600], 128, 1, 5, BF, dict(joint=True)),
    ([70], [260], 32, 1, 128, BF, {}),                       # one kv head for 128 query heads
    ([20], [150], 64, 1, 33, FP, {}),
    ([300], [1324], 1024, 8, 8, BF, {}),
    ([600], [5000], 64, 2, 8, BF, {}),
]


@pytest.mark.parametrize("case", ATTEND, ids=range(len(ATTEND)))
def test_attention_matches_64_bits(case):
    q_len, kv_len, page, n_kv, n_q, dtype, opt = case
    b = ref.Batch(q_len, kv_len, page, n_kv, n_q, dtype, seed=sum(kv_len), **opt).poison()
    eng = _engine(b)
    t = b.gpu(eng)
    out, lse = torch.full_like(t["q"], 7.0), torch.full((b.n_tokens, n_q), 7.0, device="cuda")
    eng.attention(t["batch"], t["q"], t["k_pool"], t["v_pool"], out=out, lse=lse)
    want, want_lse, tol, tol_lse = ref.attention(b)
    n = b.starts[-1]
    err, err_lse = (out.double().cpu() - want).abs()[:n], (lse.double().cpu() - want_lse).abs()[:n]
    assert bool((err <= tol[:n]).all()), float((err / tol[:n]).max())
    assert bool((err_lse <= tol_lse[:n]).all()), float((err_lse / tol_lse[:n]).max())
    assert bool((out[n:] == 7.0).all()) and bool((lse[n:] == 7.0).all())
    again, none = eng.attention(t["batch"], t["q"], t["k_pool"], t["v_pool"])
    assert none is None and torch.equal(again[:n], out[:n]), "the same call gives the same bits"
    _close(eng)


def test_attention_rows_that_see_nothing():
    """kv_len below the number of new tokens: the first of them see no row; a sequence without any row."""
    b = ref.Batch([5, 200, 3, 2, 60], [3, 150, 0, 2, 0], 16, 2, 8, seed=5)
    eng = _engine(b)
    t = b.gpu(eng)
    out, lse = eng.attention(t["batch"], t["q"], t["k_pool"], t["v_pool"], want_lse=True)
    want, want_lse, tol, tol_lse = ref.attention(b)
    empty = torch.isneginf(want_lse)
    assert bool(empty[:2].all()) and bool(empty[5:55].all()) and bool(empty[205:208].all()) and bool(empty[210:].all())
    assert bool((out.cpu()[empty] == 0).all()) and torch.equal(torch.isneginf(lse.cpu()), empty)
    assert bool(((out.double().cpu() - want).abs() <= tol).all())
    assert bool(((lse.double().cpu() - want_lse).abs() <= tol_lse)[~empty].all())
    w = t["w_pool"].clone()
    eng.accumulate(t["batch"], t["q"], lse, t["k_pool"], w)
    want_w, tol_w = ref.accumulate(b, lse.cpu())
    assert bool(((w.double().cpu() - want_w).abs() <= tol_w).all())
    _close(eng)


def test_attention_large_logits_and_strided_queries():
    """Logits of some hundreds (the running maximum moves far, most probabilities vanish), q a slice of a fused
    projection."""
    for q_len, kv_len in (([1, 2], [700, 300]), ([150, 64], [700, 300])):
        b = ref.Batch(q_len, kv_len, 32, 2, 8, seed=11)
        ramp = torch.linspace(0.1, 6.0, b.k_pool.shape[0])[:, None, None, None]
        b.k_pool = (b.k_pool.float() * ramp * 4).to(BF)
        eng = _engine(b)
        t = b.gpu(eng)
        fused = torch.randn(b.n_tokens, 12, 128, device="cuda").to(BF)
        fused[:, 1:9] = t["q"]
        out, lse = eng.attention(t["batch"], fused[:, 1:9], t["k_pool"], t["v_pool"], want_lse=True)
        want, want_lse, tol, tol_lse = ref.attention(b)
        assert bool(((out.double().cpu() - want).abs() <= tol).all())
        assert bool(((lse.double().cpu() - want_lse).abs() <= tol_lse).all())
        _close(eng)


def test_attention_many_sequences_and_shared_pages():
    """More sequences than a CTA has threads, and a common prefix whose pages all tables name."""
    n = 700
    q_len = [1 + i % 2 for i in range(n)]
    kv_len = [2 + (i * 37) % 150 for i in range(n)]
    b = ref.Batch(q_len, kv_len, 16, 1, 2, seed=1)
    for i in range(n):
        if kv_len[i] > 32:
            b.table[i, :1] = b.table[0, 0]
    eng = _engine(b)
    t = b.gpu(eng)
    out, lse = eng.attention(t["batch"], t["q"], t["k_pool"], t["v_pool"], want_lse=True)
    want, want_lse, tol, tol_lse = ref.attention(b)
    assert bool(((out.double().cpu() - want).abs() <= tol).all())
    assert bool(((lse.double().cpu() - want_lse).abs() <= tol_lse).all())
    _close(eng)


# ---- accumulated weights ---------------------------------------------------------------------------

WEIGH = [
    ([1], [1], 16, 1, 1, BF, {}),
    ([1, 1, 1], [300, 64, 1000], 64, 8, 32, BF, {}),
    ([2, 0, 5], [129, 40, 128], 32, 2, 14, FP, dict(tail_tokens=2)),
    ([130, 257], [130, 700], 16, 4, 16, BF, {}),
    ([300], [1000], 128, 1, 5, FP, dict(joint=True)),
    ([20], [150], 64, 1, 128, BF, {}),
    ([1000], [1000], 1024, 2, 8, BF, {}),
]


@pytest.mark.parametrize("case", WEIGH, ids=range(len(WEIGH)))
def test_accumulated_weights_match_64_bits(case):
    q_len, kv_len, page, n_kv, n_q, dtype, opt = case
    b = ref.Batch(q_len, kv_len, page, n_kv, n_q, dtype, seed=sum(kv_len) + 1, **opt).poison()
    eng = _engine(b)
    t = b.gpu(eng)
    _, lse = eng.attention(t["batch"], t["q"], t["k_pool"], t["v_pool"], want_lse=True)
    w = t["w_pool"].clone()
    assert eng.accumulate(t["batch"], t["q"], lse, t["k_pool"], w) is w
    want, tol = ref.accumulate(b, lse.cpu())
    err = (w.double().cpu() - want).abs()
    assert bool((err <= tol).all()), float((err / tol.clamp_min(1e-30)).max())
    # a token's probabilities sum to one
    gained = float((w.double() - t["w_pool"].double()).sum())
    assert abs(gained - sum(q_len) * n_q) <= 1e-3 * sum(q_len) * n_q
    w2 = t["w_pool"].clone()
    eng.accumulate(t["batch"], t["q"], lse, t["k_pool"], w2)
    assert torch.equal(w, w2), "the same call gives the same bits"
    _close(eng)


# ---- eviction ------------------------------------------------------------------------------------

EVICT = [
    # kv_len, page, n_kv, budget, sink, recent, per_head, options
    ([100], 16, 1, 40, 4, 8, True, {}),
    ([100, 39, 40, 41, 0, 1], 16, 2, 40, 0, 0, True, {}),
    ([1000, 300, 64], 64, 8, 64, 4, 60, False, {}),           # nothing between sinks and recent rows
    ([1000, 300, 64], 32, 4, 65, 4, 60, True, dict(joint=True)),
    ([5000, 3000, 2049], 128, 2, 2048, 0, 512, False, {}),
    ([777], 1024, 3, 500, 100, 0, True, {}),
    ([20000, 9000], 16, 2, 4096, 4, 32, True, {}),
    ([30], 16, 1, 1, 0, 0, False, {}),
]


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("case", EVICT, ids=range(len(EVICT)))
def test_eviction_keeps_and_moves(case, in_place):
    kv_len, page, n_kv, budget, sink, recent, per_head, opt = case
    n = len(kv_len)
    dst_blocks = -(-budget // page)
    b = ref.Batch([0] * n, kv_len, page, n_kv, n_kv, seed=budget, spare=2 + n * dst_blocks, **opt)
    b.w_pool[:, :, ::3] = (b.w_pool[:, :, ::3] * 4).round() / 4                 # ties
    kept = ref.evict_choice(b, budget, sink, recent, per_head)
    dst = torch.tensor(b.free[:n * dst_blocks], dtype=torch.int32).view(n, dst_blocks)
    table = b.table if in_place else dst
    kp, vp, wp = b.k_pool.clone(), b.v_pool.clone(), b.w_pool.clone()
    for i in range(n):
        pg, row = b.slots(i)
        for g in range(n_kv):
            rows = torch.tensor(kept[i][g if per_head else 0], dtype=torch.long)
            to = torch.arange(len(rows))
            dp, dr = table[i, to // page].long(), to % page
            kp[dp, dr, g], vp[dp, dr, g] = b.k_pool[pg[rows], row[rows], g], b.v_pool[pg[rows], row[rows], g]
            wp[dp, g, dr] = b.w_pool[pg[rows], g, row[rows]]
    eng = _engine(b)
    t = b.gpu(eng)
    new_len = t["kv_len"] if in_place else None
    got, length = eng.evict(t["batch"], budget, sink, recent, t["k_pool"], t["v_pool"], t["w_pool"], per_head=per_head,
                            dst_table=None if in_place else dst.cuda(), new_len=new_len)
    assert length.tolist() == [min(k, budget) for k in kv_len]
    want = torch.tensor([[r + [-1] * (budget - len(r)) for r in k] for k in kept], dtype=torch.int32)
    assert torch.equal(got.cpu(), want)
    assert torch.equal(t["k_pool"].cpu(), kp) and torch.equal(t["v_pool"].cpu(), vp)
    assert torch.equal(t["w_pool"].cpu(), wp)
    _close(eng)


def test_eviction_orders_all_weights():
    """Zeros of either sign tie, infinities and NaN are the largest, equal ones go to the lower row."""
    b = ref.Batch([0], [64], 16, 1, 1, seed=3)
    w = torch.zeros(64)
    w[10], w[20], w[30], w[40], w[50] = -0.0, math.inf, math.nan, 1e-40, 3e38
    pg, row = b.slots(0)
    b.w_pool[pg, 0, row] = w
    eng = _engine(b)
    t = b.gpu(eng)
    for per_head in (True, False):
        for budget, want in ((4, [20, 30, 40, 50]), (2, [20, 30]), (1, [30]), (16, list(range(12)) + [20, 30, 40, 50])):
            dst = torch.tensor([b.free[:1]], dtype=torch.int32).cuda()
            kept, _ = eng.evict(t["batch"], budget, 0, 0, t["k_pool"], t["v_pool"], t["w_pool"], per_head=per_head,
                                dst_table=dst)
            assert kept.flatten().tolist() == want
    _close(eng)


# ---- the operators together --------------------------------------------------------------------------

def test_serving_a_compressed_prompt():
    """Two requests: prompt appended, attended, weighed, cut to a budget, then decoded step by step with an eviction
    every few tokens -- every step against the same steps in 64 bits."""
    from paper_2508_17892_b200 import PagedCache
    n_kv, n_q, page, budget = 2, 8, 16, 48
    spec = _spec(scaling="banded", factor=8.0)
    g = torch.Generator().manual_seed(4)
    eng = PagedCache(n_kv_heads=n_kv, n_q_heads=n_q, page_size=page, max_seqs=2)
    n_pages = 16
    pools = [torch.zeros(n_pages, page, n_kv, 128, dtype=BF, device="cuda") for _ in range(2)]
    w_pool = torch.zeros(n_pages, n_kv, page, device="cuda")
    table = torch.randperm(n_pages, generator=g).to(torch.int32).view(2, 8).cuda()
    lens, pos0 = [0, 0], [0, 0]
    for step in range(14):
        q_len = [70, 33] if step == 0 else [1, 1]
        lens = [a + m for a, m in zip(lens, q_len)]
        n = sum(q_len)
        q, k, v = (torch.randn(n, h, 128, generator=g).to(BF) for h in (n_q, n_kv, n_kv))
        pos = torch.cat([torch.arange(p, p + m, dtype=torch.int32) for p, m in zip(pos0, q_len)])
        pos0 = [p + m for p, m in zip(pos0, q_len)]
        q_start = torch.tensor([0, q_len[0], n], dtype=torch.int32).cuda()
        kv_len = torch.tensor(lens, dtype=torch.int32).cuda()
        batch = eng.batch(q_start, kv_len, table, n, max(q_len))
        before = [p.cpu() for p in pools] + [w_pool.cpu()]
        qr = eng.append(batch, q.cuda(), k.cuda(), v.cuda(), pos.cuda(), spec, *pools, w_pool)
        out, lse = eng.attention(batch, qr, *pools, want_lse=True)
        b = ref.Batch(q_len, lens, page, n_kv, n_q)            # the reference sees the cache as it now is
        b.table, b.k_pool, b.v_pool, b.q = table.cpu(), pools[0].cpu(), pools[1].cpu(), qr.cpu()
        for i, m in enumerate(q_len):
            pg, row = (x[lens[i] - m:] for x in b.slots(i))
            want, slack = ref.rope(k[b.starts[i]:b.starts[i + 1]], pos[b.starts[i]:b.starts[i + 1]], spec)
            ref.assert_rounded(b.k_pool[pg, row], want, slack)
            assert torch.equal(b.v_pool[pg, row], v[b.starts[i]:b.starts[i + 1]])
            old = [x[:lens[i] - m] for x in b.slots(i)]
            assert torch.equal(b.k_pool[old[0], old[1]], before[0][old[0], old[1]])
        b.w_pool = w_pool.cpu()
        want, want_lse, tol, tol_lse = ref.attention(b)
        assert bool(((out.double().cpu() - want).abs() <= tol).all())
        assert bool(((lse.double().cpu() - want_lse).abs() <= tol_lse).all())
        eng.accumulate(batch, qr, lse, pools[0], w_pool)
        want_w, tol_w = ref.accumulate(b, lse.cpu())
        assert bool(((w_pool.double().cpu() - want_w).abs() <= tol_w).all())
        if step % 4 == 0:
            b.w_pool = w_pool.cpu()
            kept, new_len = eng.evict(batch, budget, 2, 8, *pools, w_pool, per_head=True, new_len=kv_len)
            choice = ref.evict_choice(b, budget, 2, 8, True)
            lens = new_len.tolist()
            assert lens == [len(c[0]) for c in choice]
            for i in range(2):
                for h in range(n_kv):
                    assert kept[i, h, :lens[i]].tolist() == choice[i][h]
    _close(eng)


# ---- refusals, faults in the batch -------------------------------------------------------------------

def _code(fn, *a, **kw):
    from paper_2508_17892_b200 import IlreError
    with pytest.raises(IlreError) as e:
        fn(*a, **kw)
    return e.value.code


def test_refused_arguments():
    from paper_2508_17892_b200 import PagedCache
    assert _code(PagedCache, head_dim=64) == -2
    assert _code(PagedCache, n_kv_heads=3, n_q_heads=8) == -2
    assert _code(PagedCache, n_kv_heads=1, n_q_heads=129) == -2
    assert _code(PagedCache, page_size=8) == -2
    assert _code(PagedCache, page_size=48) == -2
    assert _code(PagedCache, page_size=2048) == -2
    assert _code(PagedCache, max_seqs=0) == -1
    assert _code(PagedCache, max_seqs=70000) == -3
    b = ref.Batch([1, 1], [40, 40], 16, 2, 8)
    eng = _engine(b)
    t = b.gpu(eng)
    ev = lambda **kw: _code(eng.evict, t["batch"], kw.pop("budget", 8), kw.pop("sink", 0), kw.pop("recent", 0),  # noqa: E731
                            t["k_pool"], t["v_pool"], t["w_pool"], **kw)
    assert ev(sink=4, recent=5) == -4
    assert ev(sink=-1) == -1
    assert ev(budget=40, dst_table=torch.zeros(2, 2, dtype=torch.int32, device="cuda")) == -1
    three = eng.batch(torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda"),
                      torch.zeros(3, 1, dtype=torch.int32, device="cuda"), 2, 1)
    assert _code(eng.attention, three, t["q"], t["k_pool"], t["v_pool"]) == -3
    odd = torch.zeros(2 * 8 * 128 + 1, dtype=BF, device="cuda")[1:].view(2, 8, 128)
    assert _code(eng.attention, t["batch"], odd, t["k_pool"], t["v_pool"]) == -5
    assert _code(eng.append, t["batch"], t["q"], t["k"], t["v"], t["pos"], _spec(rotary_dim=20), t["k_pool"], t["v_pool"]) == -2
    # through the C call: arrays at odd addresses are refused, nothing is launched
    from paper_2508_17892_b200.paged import IlrePagedBatch, IlrePagedPool
    good = (2, 2, 1, 3, t["q_start"].data_ptr(), t["kv_len"].data_ptr(), t["table"].data_ptr())
    pool = IlrePagedPool(t["k_pool"].data_ptr(), t["v_pool"].data_ptr(), t["w_pool"].data_ptr(), 0, 0, b.n_pages)
    out, lse = torch.empty_like(t["q"]), torch.empty(2, 8, device="cuda")
    for i in (4, 5, 6, None):
        a = list(good)
        if i is not None:
            a[i] += 2
        assert eng._lib.ilre_paged_attention(eng._h, ctypes.byref(IlrePagedBatch(*a)), t["q"].data_ptr(), 1024,
                                             ctypes.byref(pool), out.data_ptr(), lse.data_ptr() + (2 if i is None else 0),
                                             None) == -5
    for bad in (dict(q=t["q"][:1]), dict(q=t["q"].float()), dict(k_pool=t["k_pool"][:, :8]), dict(q=t["q"].cpu())):
        a = dict(batch=t["batch"], q=t["q"], k_pool=t["k_pool"], v_pool=t["v_pool"])
        a.update(bad)
        with pytest.raises(AssertionError):
            eng.attention(**a)
    _close(eng)


def test_batches_of_no_work():
    from paper_2508_17892_b200 import PagedCache
    eng = PagedCache(n_kv_heads=2, n_q_heads=8, page_size=16)
    i32 = lambda *n: torch.zeros(*n, dtype=torch.int32, device="cuda")  # noqa: E731
    k_pool = torch.zeros(1, 16, 2, 128, dtype=BF, device="cuda")
    w = torch.zeros(1, 2, 16, device="cuda")
    for n_seqs, n_tokens in ((0, 0), (0, 3), (2, 0), (2, 3)):
        batch = eng.batch(i32(n_seqs + 1), i32(n_seqs), i32(n_seqs, 4), n_tokens, 3)
        q, k = torch.ones(n_tokens, 8, 128, dtype=BF, device="cuda"), torch.ones(n_tokens, 2, 128, dtype=BF, device="cuda")
        out, lse = torch.full_like(q, 7.0), torch.full((n_tokens, 8), 7.0, device="cuda")
        eng.append(batch, q, k, k, i32(n_tokens), _spec(), k_pool, k_pool, w, q_out=q)
        eng.attention(batch, q, k_pool, k_pool, out=out, lse=lse)
        eng.accumulate(batch, q, lse, k_pool, w)
        kept, n = eng.evict(batch, 4, 0, 0, k_pool, k_pool, w)
        assert bool((out == 7.0).all()) and bool((lse == 7.0).all()) and bool((kept == -1).all()) and bool((n == 0).all())
        assert not bool(k_pool.any()) and not bool(w.any())
    _close(eng)


def test_lengths_out_of_range_are_reported_and_left_out():
    """Sequence 1's lengths are wrong in one way after another: the others come out as ever, its rows stay."""
    for field, value in (("kv_len", -1), ("kv_len", 10 ** 6), ("q_len", 3)):
        b = ref.Batch([2, 2, 2], [40, 50, 60], 16, 2, 8, seed=2)
        eng = _engine(b)
        t = b.gpu(eng)
        want = eng.attention(t["batch"], t["q"], t["k_pool"], t["v_pool"])[0]
        if field == "kv_len":
            t["kv_len"][1] = value
            batch, bad = t["batch"], slice(2, 4)
        else:                                                # more new tokens than max_q_len says
            t["q_start"][2] = 5
            t["q_start"][3] = 6
            batch, bad = t["batch"], slice(2, 6)             # sequence 2 now has one token
        out = torch.full_like(want, 7.0)
        eng.attention(batch, t["q"], t["k_pool"], t["v_pool"], out=out)
        assert eng.status() == -10
        assert eng.status() == 0
        assert torch.equal(out[:2], want[:2]) and bool((out[2:4] == 7.0).all())
        if field == "kv_len":
            assert torch.equal(out[4:], want[4:])
        lse = torch.zeros(6, 8, device="cuda")
        w = torch.zeros_like(t["w_pool"])
        eng.accumulate(batch, t["q"], lse, t["k_pool"], w)
        assert eng.status() == -10
        kp, vp = t["k_pool"].clone(), t["v_pool"].clone()
        q_out = torch.full_like(t["q"], 7.0)
        eng.append(batch, t["q"], t["k"], t["v"], t["pos"], _spec(), kp, vp, w, q_out=q_out)
        assert eng.status() == -10
        assert bool((q_out[2:4] == 7.0).all())
        if field == "kv_len":
            kept, n = eng.evict(batch, 8, 0, 0, kp, vp, w)
            assert eng.status() == -10 and n[0] == 8 and n[2] == 8 and bool((kept[1] == -1).all())
        _close(eng)


def test_pages_out_of_range_are_reported():
    b = ref.Batch([1, 1], [40, 40], 16, 2, 8, seed=2)
    eng = _engine(b)
    t = b.gpu(eng)
    want = eng.attention(t["batch"], t["q"], t["k_pool"], t["v_pool"])[0]
    eng.check_status()
    for bad in (-1, b.n_pages, 2 ** 31 - 1, -2 ** 31):
        t["table"][1] = b.table[1].cuda()
        t["table"][1, 1] = bad
        out, lse = eng.attention(t["batch"], t["q"], t["k_pool"], t["v_pool"], want_lse=True)
        assert eng.status() == -10
        assert torch.equal(out[0], want[0])
        # rows of that page count as zeros: logit 0, value 0
        zero = ref.Batch([1, 1], [40, 40], 16, 2, 8, seed=2)
        zero.k_pool[zero.table[1, 1]] = 0
        zero.v_pool[zero.table[1, 1]] = 0
        ref_out, _, tol, _ = ref.attention(zero)
        assert bool(((out.double().cpu() - ref_out).abs() <= tol).all())
        w = t["w_pool"].clone()
        eng.accumulate(t["batch"], t["q"], lse, t["k_pool"], w)
        assert eng.status() == -10
        kp, vp = t["k_pool"].clone(), t["v_pool"].clone()
        eng.evict(t["batch"], 8, 0, 0, kp, vp, w)
        assert eng.status() == -10
        t["table"][1] = b.table[1].cuda()
        t["table"][1, 2] = bad                               # the page that the new row goes to
        kp = t["k_pool"].clone()
        eng.append(t["batch"], None, t["k"], t["v"], None, None, kp, vp)
        assert eng.status() == -10
        same = torch.ones(b.n_pages, 16, dtype=torch.bool)
        same[b.table[0, 2].long(), 7] = False                # the other sequence's new row
        assert torch.equal(kp.cpu()[same], b.k_pool[same])
    _close(eng)


# ---- streams, graphs -----------------------------------------------------------------------------------

def test_other_stream_and_captured_graph():
    """A call on a side stream, and one captured and replayed with other lengths, tables and queries."""
    b = ref.Batch([1, 3, 40], [200, 150, 90], 16, 2, 8, seed=8, wide=4, spare=30)      # a page for every entry
    eng = _engine(b)
    t = b.gpu(eng)
    want = eng.attention(t["batch"], t["q"], t["k_pool"], t["v_pool"], want_lse=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = eng.attention(t["batch"], t["q"], t["k_pool"], t["v_pool"], want_lse=True, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    q_out, out, lse = torch.empty_like(t["q"]), torch.empty_like(t["q"]), torch.empty(44, 8, device="cuda")
    new_len, kept = torch.empty_like(t["kv_len"]), torch.empty(3, 1, 50, dtype=torch.int32, device="cuda")

    def step():
        eng.append(t["batch"], t["q"], t["k"], t["v"], t["pos"], _spec(), t["k_pool"], t["v_pool"], t["w_pool"], q_out=q_out)
        eng.attention(t["batch"], q_out, t["k_pool"], t["v_pool"], out=out, lse=lse)
        eng.accumulate(t["batch"], q_out, lse, t["k_pool"], t["w_pool"])
        eng.evict(t["batch"], 50, 2, 8, t["k_pool"], t["v_pool"], t["w_pool"], new_len=new_len, kept=kept)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    state = {n: t[n].clone() for n in ("k_pool", "v_pool", "w_pool")}
    for kv in ([200, 150, 90], [61, 3, 40], [208, 154, 90]):
        for n, x in state.items():
            t[n].copy_(x)
        t["kv_len"].copy_(torch.tensor(kv, dtype=torch.int32))
        t["table"].copy_(torch.arange(t["table"].numel(), dtype=torch.int32).view_as(t["table"]))
        graph.replay()
        replayed = [x.clone() for x in (out, lse, t["k_pool"], t["w_pool"], kept, new_len)]
        for n, x in state.items():
            t[n].copy_(x)
        step()
        for x, y in zip(replayed, (out, lse, t["k_pool"], t["w_pool"], kept, new_len)):
            assert torch.equal(x, y)
    _close(eng)


# ---- sizes that cross the kernels' own bounds ------------------------------------------------------

@pytest.mark.parametrize("group", [1, 2, 3, 6, 11, 15, 16, 17, 31, 48, 64, 65, 100, 128])
def test_every_size_of_a_group(group):
    """Query heads per kv head: those that share a tile of 16, 64 or 128 rows, fill it or leave rows of it over."""
    for n_new in (1, 2, 9):
        b = ref.Batch([n_new, 1], [n_new + 150, 131], 16, 1 if group > 16 else 2, group * (1 if group > 16 else 2),
                      seed=group * 10 + n_new).poison()
        eng = _engine(b)
        t = b.gpu(eng)
        out, lse = eng.attention(t["batch"], t["q"], t["k_pool"], t["v_pool"], want_lse=True)
        want, want_lse, tol, tol_lse = ref.attention(b)
        assert bool(((out.double().cpu() - want).abs() <= tol).all())
        assert bool(((lse.double().cpu() - want_lse).abs() <= tol_lse).all())
        w = t["w_pool"].clone()
        eng.accumulate(t["batch"], t["q"], lse, t["k_pool"], w)
        want_w, tol_w = ref.accumulate(b, lse.cpu())
        assert bool(((w.double().cpu() - want_w).abs() <= tol_w).all())
        _close(eng)


@pytest.mark.parametrize("n_new", [1, 4, 5, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129])
def test_lengths_around_the_tiles(n_new):
    """New tokens and rows on both sides of the tiles' 16, 64, 128 and 256."""
    kv = [n_new, max(n_new, 63), n_new + 64, n_new + 65, max(n_new, 128), n_new + 127, n_new + 256]
    b = ref.Batch([n_new] * len(kv), kv, 32, 1, 4, seed=n_new, dtype=FP if n_new % 2 else BF).poison()
    eng = _engine(b)
    t = b.gpu(eng)
    out, lse = eng.attention(t["batch"], t["q"], t["k_pool"], t["v_pool"], want_lse=True)
    want, want_lse, tol, tol_lse = ref.attention(b)
    assert bool(((out.double().cpu() - want).abs() <= tol).all())
    assert bool(((lse.double().cpu() - want_lse).abs() <= tol_lse).all())
    w = t["w_pool"].clone()
    eng.accumulate(t["batch"], t["q"], lse, t["k_pool"], w)
    want_w, tol_w = ref.accumulate(b, lse.cpu())
    assert bool(((w.double().cpu() - want_w).abs() <= tol_w).all())
    _close(eng)


def test_pools_beyond_32_bit_offsets():
    """Pools of more than 2^31 elements: the sequences' pages are the first and the last ones."""
    from paper_2508_17892_b200 import PagedCache
    n_kv, n_q, page = 8, 16, 128
    n_pages = (1 << 31) // (page * n_kv * 128) + 40
    g = torch.Generator(device="cuda").manual_seed(1)
    k_pool, v_pool = (torch.zeros(n_pages, page, n_kv, 128, dtype=BF, device="cuda") for _ in range(2))
    assert k_pool.numel() > 1 << 31
    w_pool = torch.zeros(n_pages, n_kv, page, device="cuda")
    b = ref.Batch([3, 40], [600, 300], page, n_kv, n_q, seed=4, spare=5, garbage=False)
    far = torch.tensor([0, 1] + list(range(n_pages - b.n_pages + 2, n_pages)))     # page i of the small pool lies here
    k_pool[far], v_pool[far], w_pool[far] = b.k_pool.cuda(), b.v_pool.cuda(), b.w_pool.cuda()
    eng = PagedCache(n_kv_heads=n_kv, n_q_heads=n_q, page_size=page, max_seqs=2)
    small = b.gpu(eng)
    table = far[b.table.long()].to(torch.int32).cuda()
    batch = eng.batch(small["q_start"], small["kv_len"], table, b.n_tokens, b.max_q)
    spec = _spec()
    q = eng.append(batch, small["q"], small["k"], small["v"], small["pos"], spec, k_pool, v_pool, w_pool)
    q2 = eng.append(small["batch"], small["q"], small["k"], small["v"], small["pos"], spec, small["k_pool"], small["v_pool"],
                    small["w_pool"])
    out, lse = eng.attention(batch, q, k_pool, v_pool, want_lse=True)
    out2, lse2 = eng.attention(small["batch"], q2, small["k_pool"], small["v_pool"], want_lse=True)
    eng.accumulate(batch, q, lse, k_pool, w_pool)
    eng.accumulate(small["batch"], q2, lse2, small["k_pool"], small["w_pool"])
    kept, _ = eng.evict(batch, 200, 2, 30, k_pool, v_pool, w_pool)
    kept2, _ = eng.evict(small["batch"], 200, 2, 30, small["k_pool"], small["v_pool"], small["w_pool"])
    for x, y in ((q, q2), (out, out2), (lse, lse2), (kept, kept2), (k_pool[far], small["k_pool"]),
                 (v_pool[far], small["v_pool"]), (w_pool[far], small["w_pool"])):
        assert torch.equal(x, y)
    want, _, tol, _ = ref.attention(_as_now(b, small, q2, out2))
    assert bool(((out.double().cpu() - want).abs() <= tol).all())
    _close(eng)


def _as_now(b, small, q, out):
    """The batch with its rows as `append` left them (before the eviction moved them, which this undoes by appending
    to a fresh copy)."""
    from paper_2508_17892_b200 import PagedCache
    fresh = ref.Batch(b.q_len, b.kv_len_list, b.page, b.n_kv, b.n_q, seed=4, spare=5, garbage=False)
    eng = PagedCache(n_kv_heads=b.n_kv, n_q_heads=b.n_q, page_size=b.page, max_seqs=2)
    t = fresh.gpu(eng)
    fresh.q = eng.append(t["batch"], t["q"], t["k"], t["v"], t["pos"], _spec(), t["k_pool"], t["v_pool"]).cpu()
    fresh.k_pool, fresh.v_pool = t["k_pool"].cpu(), t["v_pool"].cpu()
    eng.close()
    return fresh


def test_two_caches_on_two_streams():
    """Two handles at work at the same time, and their captured steps replayed side by side."""
    made = []
    for seed, (q_len, kv_len) in enumerate((([1, 1, 30], [3000, 700, 900]), ([200, 1], [900, 2500]))):
        b = ref.Batch(q_len, kv_len, 32, 4, 16, seed=20 + seed)
        eng = _engine(b)
        t = b.gpu(eng)
        out, lse = torch.empty_like(t["q"]), torch.empty(b.n_tokens, 16, device="cuda")
        w = torch.zeros_like(t["w_pool"])

        def step(eng=eng, t=t, out=out, lse=lse, w=w):
            eng.attention(t["batch"], t["q"], t["k_pool"], t["v_pool"], out=out, lse=lse)
            eng.accumulate(t["batch"], t["q"], lse, t["k_pool"], w)

        step()
        torch.cuda.synchronize()
        want = [x.clone() for x in (out, lse, w)]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        made.append((eng, step, (out, lse, w), want, graph, torch.cuda.Stream()))
    for replay in (False, True):
        for eng, step, got, want, graph, stream in made:
            for x in got:
                x.zero_()
        torch.cuda.synchronize()
        for _ in range(10):
            for eng, step, got, want, graph, stream in made:
                with torch.cuda.stream(stream):
                    got[2].zero_()
                    graph.replay() if replay else step()
        torch.cuda.synchronize()
        for eng, step, got, want, graph, stream in made:
            assert all(torch.equal(x, y) for x, y in zip(got, want))
    for eng, *_ in made:
        _close(eng)


# ---- calls that only the documentation makes -------------------------------------------------------------

def test_status_of_a_graph_on_another_stream():
    """The last call by hand is on the current stream, the replay with a bad length on a side stream behind long
    work: the status still tells."""
    b = ref.Batch([1, 1], [40, 40], 16, 2, 8, seed=4)
    eng = _engine(b)
    t = b.gpu(eng)
    out = torch.empty_like(t["q"])
    eng.attention(t["batch"], t["q"], t["k_pool"], t["v_pool"], out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        eng.attention(t["batch"], t["q"], t["k_pool"], t["v_pool"], out=out)
    t["kv_len"][1] = -1
    eng.append(t["batch"], None, t["k"][:2], t["v"][:2], None, None, t["k_pool"], t["v_pool"])
    assert eng.status() == -10
    torch.cuda.synchronize()
    side, big = torch.cuda.Stream(), torch.zeros(1 << 28, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(40):                                  # some 10 ms
            big.add_(1.0)
        graph.replay()
    assert eng.status() == -10
    _close(eng)


def test_refused_overlaps_and_budgets():
    from paper_2508_17892_b200.paged import PagedBatch
    b = ref.Batch([2, 2], [40, 40], 16, 2, 8)
    eng = _engine(b)
    t = b.gpu(eng)
    q = torch.zeros(8, 8, 128, dtype=BF, device="cuda")
    for at in (0, 1, 3):                                     # the output over the queries, or over some of them
        assert _code(eng.attention, t["batch"], q[:4], t["k_pool"], t["v_pool"], out=q[at:at + 4]) == -1
    eng.attention(t["batch"], q[:4], t["k_pool"], t["v_pool"], out=q[4:])
    wide = torch.zeros(4, 16, 128, dtype=BF, device="cuda")
    assert _code(eng.append, t["batch"], wide[:, :8], t["k"], t["v"], t["pos"], _spec(), t["k_pool"], t["v_pool"],
                 q_out=wide.view(8, 8, 128)[:4]) == -1
    from paper_2508_17892_b200.paged import IlrePagedPool
    pool = IlrePagedPool(t["k_pool"].data_ptr(), t["v_pool"].data_ptr(), t["w_pool"].data_ptr(), 0, 0, b.n_pages)
    kept = torch.zeros(4, dtype=torch.int32, device="cuda")
    assert eng._lib.ilre_paged_evict(eng._h, t["batch"].ref, 2 ** 31 - 1, 0, 0, 0, ctypes.byref(pool), None, 0,
                                     kept.data_ptr(), kept.data_ptr(), None) == -3
    host = PagedBatch(t["q_start"].cpu(), t["kv_len"].cpu(), t["table"].cpu(), 4, 2)      # arrays on another device
    with pytest.raises(AssertionError):
        eng.attention(host, t["q"], t["k_pool"], t["v_pool"])
    with pytest.raises(AssertionError):
        eng.append(host, None, t["k"], t["v"], None, None, t["k_pool"], t["v_pool"])
    with pytest.raises(AssertionError):
        eng.evict(host, 8, 0, 0, t["k_pool"], t["v_pool"], t["w_pool"])
    _close(eng)
