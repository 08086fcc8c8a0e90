"""Edges of the paged-cache operators: probabilities far below the largest, sequences and pages that are left out, lists
longer than the selection's shared memory."""
import pytest
import torch

import paged_reference as ref

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float16


def _engine(b):
    from paper_2508_17892_b200 import PagedCache
    return PagedCache(n_kv_heads=b.n_kv, n_q_heads=b.n_q, page_size=b.page, dtype=b.dtype, max_seqs=len(b.q_len))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("n_new", [1, 40])
def test_many_small_probabilities_beside_large_ones(n_new, dtype):
    """Four rows' logits are 26 powers of two above those of 2^17 others, whose values are 1 while theirs are 0: the output
    is what the small probabilities sum up to, 2^-11.  As many sequences as keep a CTA on each, so that the large ones are
    its maximum from the first tile on (one in each run of 16 keys)."""
    from paper_2508_17892_b200 import PagedCache
    page, kv, n_seqs = 1024, 1 << 17, 2 * torch.cuda.get_device_properties(0).multi_processor_count
    eng = PagedCache(n_kv_heads=1, n_q_heads=1, page_size=page, dtype=dtype, max_seqs=n_seqs)
    k_pool = torch.zeros(2, page, 1, 128, dtype=dtype, device="cuda")
    v_pool = torch.ones_like(k_pool)
    for row in (3, 19, 35, 51):
        k_pool[0, row, 0, 0], v_pool[0, row] = 12.75, 0.0
    table = torch.ones(n_seqs, kv // page, dtype=torch.int32, device="cuda")   # all rows but the first page's are one page's
    table[:, 0] = 0
    q_start = torch.arange(n_seqs + 1, dtype=torch.int32, device="cuda") * n_new
    batch = eng.batch(q_start, torch.full((n_seqs,), kv, dtype=torch.int32, device="cuda"), table, n_seqs * n_new, n_new)
    q = torch.zeros(n_seqs * n_new, 1, 128, dtype=dtype, device="cuda")
    q[:, :, 0] = 16.0
    out, lse = eng.attention(batch, q, k_pool, v_pool, want_lse=True)
    eng.check_status()
    top = 16.0 * 12.75 / 128 ** 0.5
    small = torch.exp(torch.tensor(-top, dtype=torch.float64))
    rows = torch.arange(kv - n_new - 3, kv - 3, dtype=torch.float64).repeat(n_seqs)      # small ones that each token sees
    total = 4 + rows * small
    want = (rows * small / total)[:, None]
    # fp16: a probability is rounded at 2^7 times its ratio to the largest one (2^15 where a group's rows are few), so each
    # is off by at most 2^-25-7 of the largest, for 2^17 values of 1; bf16: by half a step of itself.  A thread adds to its
    # sums once per tile of 64 or 128 keys, at most 2^11 times; each addition to a sum between 1 and 2 may lose 2^-24 (the small
    # terms beside a large one do), so a sum is off by at most 2^-13 of itself, numerator and denominator both, and lse
    # by as much and 2^-16 for the logit 18.03 and the logarithm.  The output is rounded by half a step.
    u = ref.half_step(dtype)
    tol = want * (2 * u + 2.0 ** -12) + (kv * 2.0 ** -32 / 4 if dtype == FP else 0.0)
    err = (out[:, 0].double().cpu() - want).abs()
    assert bool((err <= tol).all()), (float(err.max()), float(tol.min()))
    assert float((lse[:, 0].double().cpu() - (top + torch.log(total))).abs().max()) <= 2.0 ** -13 + 2.0 ** -16
    eng.close()


def test_eviction_gives_a_length_to_sequences_left_out():
    """A sequence whose length is out of range has 0 rows in new_len, unless that is the batch's own array."""
    from paper_2508_17892_b200 import PagedCache
    b = ref.Batch([0, 0, 0], [40, 50, 60], 16, 2, 8, seed=2, spare=8)
    for bad in (-1, 10 ** 6):
        for in_place in (True, False):
            eng = PagedCache(n_kv_heads=2, n_q_heads=8, page_size=16, max_seqs=3)
            t = b.gpu(eng)
            t["kv_len"][1] = bad
            dst = None if in_place else torch.tensor(b.free[:6], dtype=torch.int32).view(3, 2)[:, :1].contiguous().cuda()
            for own in (False, True):
                new_len = t["kv_len"] if own else torch.full((3,), 7, dtype=torch.int32, device="cuda")
                kept, n = eng.evict(t["batch"], 8, 0, 0, t["k_pool"].clone(), t["v_pool"].clone(), t["w_pool"].clone(),
                                    new_len=new_len, dst_table=dst)
                assert eng.status() == -10
                assert n.tolist() == [8, bad if own else 0, 8] and bool((kept[1] == -1).all())
            eng.close()


@pytest.mark.parametrize("per_head", [True, False])
def test_eviction_weighs_rows_of_missing_pages_as_zeros(per_head):
    """All weights are 0 and so are those of a page out of range: the lower rows stay, whichever page they lie in."""
    from paper_2508_17892_b200 import PagedCache
    b = ref.Batch([0], [64], 16, 1, 1, seed=3)
    b.w_pool.zero_()
    eng = PagedCache(n_kv_heads=1, n_q_heads=1, page_size=16, max_seqs=1)
    t = b.gpu(eng)
    t["table"][0, 1] = b.n_pages
    kept, n = eng.evict(t["batch"], 40, 0, 0, t["k_pool"], t["v_pool"], t["w_pool"], per_head=per_head)
    assert eng.status() == -10
    assert n.tolist() == [40] and kept.flatten().tolist() == list(range(40))
    eng.close()


def test_eviction_of_a_list_that_shared_memory_does_not_hold():
    """400000 rows: each of the eight CTAs of the list keeps 44032 keys, the others are read again in every pass.  Few
    distinct weights, so that thousands tie at the threshold; then all different."""
    from paper_2508_17892_b200 import PagedCache
    page, kv, budget, sink, recent = 1024, 400_000, 150_001, 5, 70
    blocks = -(-kv // page)
    g = torch.Generator().manual_seed(6)
    table = torch.randperm(blocks, generator=g).to(torch.int32)[None]
    for distinct in (50, 1 << 24):
        w = torch.randint(0, distinct, (blocks, 1, page), generator=g).float()
        eng = PagedCache(n_kv_heads=1, n_q_heads=1, page_size=page, max_seqs=1)
        cu = lambda x: x.cuda()  # noqa: E731
        t = torch.arange(kv)
        key = w[table[0, t // page].long(), 0, t % page]
        mid = torch.sort(key[sink:kv - recent], descending=True, stable=True).indices[:budget - sink - recent] + sink
        want = torch.cat([torch.arange(sink), mid.sort().values, torch.arange(kv - recent, kv)])
        pool = torch.randn(blocks, page, 1, 128, generator=g).to(BF)
        batch = eng.batch(None, torch.tensor([kv], dtype=torch.int32).cuda(), cu(table), 0, 0)
        for per_head in (True, False):
            k, v, wg = cu(pool), cu(pool).neg(), cu(w)
            kept, n = eng.evict(batch, budget, sink, recent, k, v, wg, per_head=per_head)
            eng.check_status()
            assert n.tolist() == [budget] and torch.equal(kept.flatten().long().cpu(), want)
            i = torch.arange(budget)
            to, row, src, src_row = table[0, i // page].long(), i % page, table[0, want // page].long(), want % page
            assert torch.equal(k.cpu()[to, row], pool[src, src_row]) and torch.equal(v.cpu()[to, row], -pool[src, src_row])
            assert torch.equal(wg.cpu()[to, 0, row], w[src, 0, src_row])
        assert eng.check_guards() == 0
        eng.close()


def test_append_refuses_rows_that_are_read_and_written():
    """q_out over some of q's, k's or v's rows is refused before anything is launched; in place in a fused projection, and
    into the gap between its slices, it is as ever."""
    from paper_2508_17892_b200 import IlreError, RopeSpec
    b = ref.Batch([3, 2], [40, 30], 16, 2, 8, seed=7)
    eng = _engine(b)
    t = b.gpu(eng)
    spec = RopeSpec()
    want = eng.append(t["batch"], t["q"], t["k"], t["v"], t["pos"], spec, t["k_pool"], t["v_pool"])
    fused = torch.zeros(5, 24, 128, dtype=BF, device="cuda")
    q, k, v, gap = fused[:, :8], fused[:, 8:10], fused[:, 10:12], fused[:, 14:22]

    def fill():
        fused.zero_()
        q.copy_(t["q"]), k.copy_(t["k"]), v.copy_(t["v"])

    flat = torch.zeros(9, 8, 128, dtype=BF, device="cuda")
    flat[:5] = t["q"]
    for args in ((fused[:, 1:9], k, v, q), (q, k, v, fused[:, 1:9]), (q, k, v, fused[:, 4:12]), (fused[:, 14:22], k, v, fused[:, 3:11]),
                 (flat[:5], t["k"], t["v"], flat[1:6]), (flat[1:6], t["k"], t["v"], flat[:5]),
                 (t["q"], flat.view(36, 2, 128)[:5], t["v"], flat[:5]), (t["q"], t["k"], flat.view(36, 2, 128)[3:8], flat[:5])):
        with pytest.raises(IlreError) as e:
            eng.append(t["batch"], *args[:3], t["pos"], spec, t["k_pool"], t["v_pool"], q_out=args[3])
        assert e.value.code == -1
    for out in (q, gap):
        fill()
        pools = [torch.zeros_like(t["k_pool"]) for _ in range(2)]
        eng.append(t["batch"], q, k, v, t["pos"], spec, *pools, q_out=out)
        assert torch.equal(out, want) and torch.equal(k, t["k"]) and torch.equal(v, t["v"])
        for i in range(2):
            pg, row = (x[b.kv_len_list[i] - b.q_len[i]:].cuda() for x in b.slots(i))
            assert torch.equal(pools[0][pg, row], t["k_pool"][pg, row]) and torch.equal(pools[1][pg, row], t["v_pool"][pg, row])
    eng.check_status()
    eng.close()


@pytest.mark.parametrize("transposed", [False, True])
def test_rope_is_differentiable(transposed):
    """A tensor that requires its gradient gets it: the transposed map of what comes back, also where that is one number
    for all, strided or off its alignment, a second time, on a side stream and inside a captured graph."""
    from paper_2508_17892_b200 import RopeSpec, rope
    g = torch.Generator().manual_seed(5)
    spec = RopeSpec(rotary_dim=64, interleaved=True, scaling="yarn", factor=8.0, orig_len=4096, low=1.0, high=32.0)
    x, y = (torch.randn(9, 3, 128, generator=g).to(BF).cuda() for _ in range(2))
    pos = torch.randint(0, 100000, (9,), generator=g, dtype=torch.int32).cuda()
    turned = rope(x, pos, spec, transposed)
    assert not turned.requires_grad
    leaf = x.clone().requires_grad_()
    out = rope(leaf, pos, spec, transposed)
    assert torch.equal(out, turned) and out.requires_grad
    back = lambda v: rope(v.clone(memory_format=torch.contiguous_format), pos, spec, not transposed)  # noqa: E731
    want, slack = ref.rope(y.cpu(), pos.cpu(), spec, not transposed)
    for v in (y, torch.ones((), dtype=BF, device="cuda").expand(9, 3, 128), y.flip(0).transpose(1, 2).contiguous().transpose(1, 2),
              torch.cat([y.flatten()[:1], y.flatten()])[1:].view(9, 3, 128)):
        grad, = torch.autograd.grad(out, leaf, v, retain_graph=True)
        assert torch.equal(grad, back(v))
    ref.assert_rounded(torch.autograd.grad(out, leaf, y, retain_graph=True)[0].cpu(), want, slack)
    v = y.clone().requires_grad_()
    grad, = torch.autograd.grad(out, leaf, v, create_graph=True)
    assert torch.equal(torch.autograd.grad(grad, v, x)[0], turned)                      # linear: its gradient's gradient
    (out.float() * y.float()).sum().backward()
    assert torch.equal(leaf.grad, back(y))
    with torch.no_grad():
        assert not rope(leaf, pos, spec, transposed).requires_grad
        assert rope(leaf, pos, spec, transposed, out=torch.empty_like(x)).equal(turned)
    for into in (torch.empty_like(x), leaf):
        with pytest.raises(AssertionError):
            rope(leaf, pos, spec, transposed, out=into)
    with pytest.raises(AssertionError):
        rope(x, pos, spec, transposed, out=torch.empty_like(x).requires_grad_())
    side = torch.cuda.Stream()
    other = x.clone().requires_grad_()
    side.wait_stream(torch.cuda.current_stream())
    grad, = torch.autograd.grad(rope(other, pos, spec, transposed, stream=side), other, y)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(grad, back(y))
    static = x.clone().requires_grad_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = rope(static, pos, spec, transposed)
        d, = torch.autograd.grad(o, static, y)
    with torch.no_grad():
        static.copy_(x.flip(0))
    y.copy_(y.flip(1))
    graph.replay()
    assert torch.equal(o, rope(x.flip(0), pos, spec, transposed)) and torch.equal(d, back(y))


def test_rope_gradient_of_a_projection():
    """Through a projection, as a model has it: the weight's gradient against 64 bits and against differences."""
    from paper_2508_17892_b200 import RopeSpec, rope
    g = torch.Generator().manual_seed(8)
    spec = RopeSpec(theta=10000.0)
    a = torch.randn(6, 32, generator=g, dtype=torch.float64)
    w = torch.randn(32, 2 * 128, generator=g, dtype=torch.float64) / 8
    y = torch.randn(6, 2, 128, generator=g).to(FP)
    pos = torch.arange(6, dtype=torch.int32) * 77
    leaf = w.float().cuda().requires_grad_()
    rows = (a.float().cuda() @ leaf).to(FP).view(6, 2, 128)
    (rope(rows, pos.cuda(), spec).float() * y.cuda().float()).sum().backward()
    back, slack = ref.rope(y, pos, spec, True)               # of the rows; linear, so it does not hang on them
    want = a.T @ back.reshape(6, 256)
    # each of the rows' gradients is rounded once to fp16, the product of 6 terms in 32 bits
    u = ref.half_step(FP)
    tol = a.abs().T @ (back.abs() * u + slack * (1 + u) + 2.0 ** -25).reshape(6, 256) + 2.0 ** -20 * (a.abs().T @ back.abs().reshape(6, 256))
    assert bool(((leaf.grad.double().cpu() - want).abs() <= tol).all())
    f = lambda v: float((ref.rope((a @ v).view(6, 2, 128), pos, spec)[0] * y.double()).sum())  # noqa: E731
    for i, j in ((0, 0), (17, 64), (31, 255)):
        d = torch.zeros_like(w)
        d[i, j] = 1e-3
        # linear: the difference is the derivative, but for the roundings of 64 bits
        assert abs((f(w + d) - f(w - d)) / 2e-3 - float(want[i, j])) <= 1e-8


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("n_new", [1, 2, 40, 300])
def test_logits_of_many_millions(n_new, dtype):
    """Keys of 128 channels of +-30000: a query that is one of them has a logit of 10^10 there, and on every other key one
    that is smaller by 10^8 at least.  Its probability is exactly 1 and the output that key's value, bit for bit."""
    n_kv, n_q, kv, page = 2, 6, 900, 64
    g = torch.Generator().manual_seed(n_new)
    b = ref.Batch([n_new, 1], [kv, 70], page, n_kv, n_q, dtype, seed=n_new)
    b.k_pool = ((torch.randint(0, 2, b.k_pool.shape, generator=g) * 2 - 1) * 30000.0).to(dtype)
    want = torch.zeros_like(b.q)
    for i, (m, rows) in enumerate(((n_new, kv), (1, 70))):
        pg, row = b.slots(i)
        for j in range(m):
            for h in range(n_q):
                t = int(torch.randint(0, rows - m + j + 1, (), generator=g))
                b.q[b.starts[i] + j, h] = b.k_pool[pg[t], row[t], h * n_kv // n_q]
                want[b.starts[i] + j, h] = b.v_pool[pg[t], row[t], h * n_kv // n_q]
    eng = _engine(b)
    t = b.gpu(eng)
    out, lse = eng.attention(t["batch"], t["q"], t["k_pool"], t["v_pool"], want_lse=True)
    eng.check_status()
    assert torch.equal(out.cpu(), want)
    top = 128 ** 0.5 * float(b.k_pool.flatten()[0].abs()) ** 2
    assert float((lse.double().cpu() / top - 1).abs().max()) <= 2.0 ** -20
    eng.close()


def test_as_many_kv_heads_as_are_taken():
    """1024 kv heads: appended, attended (few rows and chunks), weighed, cut in place and to other pages."""
    b = ref.Batch([3, 20, 1], [40, 20, 17], 16, 1024, 1024, seed=12, spare=4).poison()
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
    for per_head in (True, False):
        kept = ref.evict_choice(b, 16, 1, 5, per_head)
        k, v, wp = t["k_pool"].clone(), t["v_pool"].clone(), t["w_pool"].clone()
        got, n = eng.evict(t["batch"], 16, 1, 5, k, v, wp, per_head=per_head)
        dst = torch.tensor(b.free[:3], dtype=torch.int32)[:, None]
        k2, v2, wp2 = t["k_pool"].clone(), t["v_pool"].clone(), t["w_pool"].clone()
        got2, _ = eng.evict(t["batch"], 16, 1, 5, k2, v2, wp2, per_head=per_head, dst_table=dst.cuda())
        assert n.tolist() == [16, 16, 16] and torch.equal(got, got2) and got.cpu().tolist() == kept
        for i in range(3):
            a, c = b.table[i, 0], dst[i, 0]
            pg, row = b.slots(i)
            src = got[i].long().cpu().expand(1024, 16)
            heads = torch.arange(1024)[:, None]
            want_k = b.k_pool[pg[src], row[src], heads].transpose(0, 1)
            assert torch.equal(k[a].cpu(), want_k) and torch.equal(k2[c].cpu(), want_k)
            assert torch.equal(v[a], v2[c]) and torch.equal(wp[a], wp2[c])
            assert torch.equal(wp[a].cpu(), b.w_pool[pg[src], heads, row[src]])
    new = eng.append(t["batch"], t["q"], t["k"], t["v"], None, None, t["k_pool"], t["v_pool"], t["w_pool"])
    assert torch.equal(new, t["q"])
    for i in range(3):
        pg, row = (x[b.kv_len_list[i] - b.q_len[i]:].cuda() for x in b.slots(i))
        assert torch.equal(t["k_pool"][pg, row], t["k"][b.starts[i]:b.starts[i + 1]])
        assert torch.equal(t["v_pool"][pg, row], t["v"][b.starts[i]:b.starts[i + 1]]) and not bool(t["w_pool"][pg, :, row].any())
    eng.check_status()
    assert eng.check_guards() == 0
    eng.close()


def test_as_many_sequences_as_are_taken():
    """65535 sequences of one to three rows on a page each, the newest row of this call: every operator once."""
    from paper_2508_17892_b200 import PagedCache, RopeSpec
    n = 65535
    g = torch.Generator(device="cuda").manual_seed(3)
    eng = PagedCache(n_kv_heads=1, n_q_heads=2, page_size=16, max_seqs=n)
    k_pool, v_pool = (torch.randn(n, 16, 1, 128, generator=g, device="cuda").to(BF) for _ in range(2))
    w_pool = torch.rand(n, 1, 16, generator=g, device="cuda")
    table = torch.randperm(n, generator=g, device="cuda").to(torch.int32)[:, None].contiguous()
    kv = (torch.arange(n, device="cuda") % 3 + 1).to(torch.int32)
    batch = eng.batch(torch.arange(n + 1, dtype=torch.int32, device="cuda"), kv, table, n, 1)
    q, k, v = (torch.randn(n, h, 128, generator=g, device="cuda").to(BF) for h in (2, 1, 1))
    page, last = table[:, 0].long(), kv.long() - 1
    qr = eng.append(batch, q, k, v, last.to(torch.int32), RopeSpec(), k_pool, v_pool, w_pool)
    assert torch.equal(v_pool[page, last], v) and not bool(w_pool[page, 0, last].any())
    out, lse = eng.attention(batch, qr, k_pool, v_pool, want_lse=True)
    s = torch.einsum("nhd,nkd->nhk", qr.double(), k_pool[page][:, :3, 0].double()) / 128 ** 0.5
    s = s.masked_fill(torch.arange(3, device="cuda") > last[:, None, None], float("-inf"))
    z = torch.logsumexp(s, dim=-1)
    p = torch.exp(s - z[..., None])
    vals = v_pool[page][:, :3, 0].double()
    # logits off by 2^-17 at most (128 products of sizes below 2^5 in 32 bits, their sum below 2^9), the probabilities and
    # the output rounded to bf16
    u = ref.half_step(BF)
    want = torch.einsum("nhk,nkd->nhd", p, vals)
    tol = u * want.abs() + (u + 2.0 ** -15) * (1 + u) * torch.einsum("nhk,nkd->nhd", p, vals.abs()) + 1e-30
    assert bool(((out.double() - want).abs() <= tol).all())
    assert float((lse.double() - z).abs().max()) <= 2.0 ** -14
    before = w_pool.clone()
    eng.accumulate(batch, qr, lse, k_pool, w_pool)
    gain = (w_pool - before)[page][:, 0, :3].double()
    assert float((gain - p.sum(dim=1)).abs().max()) <= 2 * (2.0 ** -14 + 2.0 ** -20) + 2.0 ** -22
    kept, new_len = eng.evict(batch, 2, 0, 1, k_pool, v_pool, w_pool)
    assert torch.equal(new_len, kv.clamp(max=2))
    w3 = before[page][:, 0, :3].double() + gain
    heavier = (w3[:, 1] > w3[:, 0]).long()
    three = kv == 3
    assert torch.equal(kept[three, 0, 1], torch.full((int(three.sum()),), 2, dtype=torch.int32, device="cuda"))
    clear = three & ((w3[:, 1] - w3[:, 0]).abs() > 1e-3)
    assert int(clear.sum()) > 15000 and torch.equal(kept[clear, 0, 0].long(), heavier[clear])
    assert bool((kept[kv == 1, 0] == torch.tensor([0, -1], dtype=torch.int32, device="cuda")).all())
    eng.check_status()
    assert eng.check_guards() == 0
    eng.close()
