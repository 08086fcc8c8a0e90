"""Calls that the paged cache's entry points refuse, as far as they can be told without a device: nothing is launched and
no pointer followed before the arguments have passed."""
import ctypes
import os
import subprocess
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    from paper_2508_17892_b200 import build, recall
    build.build()
    return recall.load_library()


def _shares(a, b, n, row_a, row_b):
    """Do n rows at a = (address, stride) and at b share a byte?  By counting, strides and rows in elements of 2 bytes."""
    cells = lambda p, s, r: {p + 2 * (i * s + j) for i in range(n) for j in range(r)}  # noqa: E731
    return bool(cells(*a, row_a) & cells(*b, row_b))


@pytest.mark.skipif(torch.cuda.is_available(), reason="what is not refused would be launched on these addresses")
def test_rope_refuses_rows_that_are_read_and_written(lib):
    """Rows of 16 elements at every distance on both sides, slices of one tensor among them; -6 (no device) is what a call
    gets that has passed."""
    from paper_2508_17892_b200.paged import IlreRopeSpec
    spec = IlreRopeSpec(10000.0, 16, 0, 0, 1.0, 0.0, 0.0, 0.0, 0.0)
    x = 1 << 20
    passed = set()
    for n, xs, os_ in ((1, 16, 16), (1, 16, 48), (2, 16, 16), (3, 48, 48), (4, 56, 56), (3, 16, 48), (4, 48, 16)):
        for step in range(-40, 41):
            out = x + 16 * step
            code = lib.ilre_rope(ctypes.byref(spec), x, xs, out, os_, 4096, n, 1, 16, 0, 0, None)
            shared = _shares((x, xs), (out, os_), n, 16, 16)
            if out == x:
                assert (code == -1) == (n > 1 and xs != os_)
            elif xs == os_ or n == 1:
                assert (code == -1) == shared, (n, xs, step)
            else:                                            # two strides: refused where the spans meet
                assert code == -1 or not shared
                assert code != -1 or -((n - 1) * os_ + 16) * 2 < out - x < ((n - 1) * xs + 16) * 2
            if code != -1:
                passed.add(code)
    assert passed == {-6}


def _optimised(code):
    """Runs `code` in an interpreter that leaves assert statements out."""
    r = subprocess.run([sys.executable, "-O", "-c", "import sys\nsys.path.insert(0, %r)\n" % ROOT + code], capture_output=True,
                       text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-1000:] + r.stderr[-3000:]


def test_checks_of_tensors_hold_without_assert_statements(lib):
    """Under ``python -O`` tensors of another device, type or shape still do not reach the library."""
    _optimised(r'''
import torch
from paper_2508_17892_b200 import paged

class Library:                                               # stands in for the shared object: counts the calls
    calls = 0
    def __getattr__(self, name):
        def call(*a):
            Library.calls += 1
            return 0
        return call

def refused(fn, *a, **kw):
    try:
        fn(*a, **kw)
    except AssertionError:
        return
    raise SystemExit("not refused: %s" % (fn,))

paged.load_library = Library
paged._raw_stream = lambda index: 0
x, pos = torch.zeros(4, 8, 128, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
refused(paged.rope, x, pos, paged.RopeSpec())                # host tensors
c = paged.PagedCache.__new__(paged.PagedCache)
c._lib, c._h, c.dtype, c._n_q, c._dim, c._index, c.device = Library(), None, torch.bfloat16, 8, 128, 0, torch.device("cuda", 0)
c._page_shape, c._weight_shape, c._page_stride = (16, 2, 128), (2, 16), (256, 128, 1)
i32 = lambda *n: torch.zeros(*n, dtype=torch.int32)
refused(c.batch, i32(3), i32(2), i32(2, 4), 4, 2)
b = paged.PagedBatch(i32(3), i32(2), i32(2, 4), 4, 2)
k = torch.zeros(4, 2, 128, dtype=torch.bfloat16)
pool, w = torch.zeros(3, 16, 2, 128, dtype=torch.bfloat16), torch.zeros(3, 2, 16)
for index in (0, -1):                                        # the handle's device; then as if the host's tensors were there
    c._index = index
    # right shapes pass where the device is the tensors' own
    if index < 0:
        c.attention(b, x, pool, pool)
        c.append(b, x, k, k, pos, None, pool, pool)
        if Library.calls != 2:
            raise SystemExit("a call that is right did not reach the library")
        Library.calls = 0
    wrong = [x.float(), x[:3], x[:, :4], x.transpose(0, 1)] if index < 0 else [x]
    for q in wrong:
        refused(c.attention, b, q, pool, pool)
        refused(c.append, b, q, k, k, pos, None, pool, pool)
        refused(c.accumulate, b, q, torch.zeros(4, 8), pool, w)
    for bad in ([pool.half(), pool[:, :8], pool[:, :, :1]] if index < 0 else [pool]):
        refused(c.attention, b, x, bad, pool)
        refused(c.append, b, x, k, k, pos, None, bad, bad)
        refused(c.evict, b, 8, 0, 0, bad, pool, w)
    if index < 0:
        refused(c.attention, b, x, pool, pool, out=x[:2])
        refused(c.attention, b, x, pool, pool, lse=torch.zeros(4, 7))
        refused(c.append, b, x, k[:3], k, pos, None, pool, pool)
        refused(c.append, b, x, k, k, None, paged.RopeSpec(), pool, pool)
        refused(c.append, b, x, k, k, pos.long(), paged.RopeSpec(), pool, pool)
        refused(c.append, b, None, k, k, pos, None, pool, pool, q_out=x)
        refused(c.accumulate, b, x, None, pool, w)
        refused(c.accumulate, b, x, torch.zeros(4, 8), pool, w.double())
        refused(c.evict, b, 0, 0, 0, pool, pool, w)
        refused(c.evict, b, 8, 0, 0, pool, pool, w, dst_table=i32(2, 4).long())
        refused(c.evict, b, 8, 0, 0, pool, pool, w, kept=i32(2, 1, 7))
if Library.calls:
    raise SystemExit("a refused call reached the library")
''')


def test_the_bindings_have_no_assert_statements():
    import ast
    import paper_2508_17892_b200 as package
    for name in ("paged.py", "recall.py", "sharded.py"):
        tree = ast.parse(open(os.path.join(os.path.dirname(package.__file__), name)).read())
        assert not [n.lineno for n in ast.walk(tree) if isinstance(n, ast.Assert)], name


def test_batches_made_by_hand_are_checked():
    """``PagedBatch`` is public: what it is given decides how much the kernels read of it."""
    from paper_2508_17892_b200 import PagedBatch
    i32 = lambda *n: torch.zeros(*n, dtype=torch.int32)  # noqa: E731
    wide = i32(2, 8)
    b = PagedBatch(i32(3), i32(2), i32(2, 4), 4, 2)
    assert (b._c.n_seqs, b._c.n_tokens, b._c.max_q_len, b._c.max_blocks) == (2, 4, 2, 4)
    PagedBatch(None, i32(0), i32(0, 4), 0, 0)
    for bad in ((i32(2), i32(2), i32(2, 4)), (i32(4), i32(2), i32(2, 4)), (i32(3).long(), i32(2), i32(2, 4)),
                (i32(3), i32(2).long(), i32(2, 4)), (i32(3), i32(2), i32(2, 4).float()), (i32(3), i32(2), i32(1, 4)),
                (i32(3), i32(2), i32(8)), (i32(3), i32(2), wide[:, :4]), (i32(3), i32(4)[::2], i32(2, 4)),
                (i32(3), i32(1, 2), i32(2, 4)), (i32(3).to("meta"), i32(2), i32(2, 4)), (i32(3), i32(2), i32(2, 4).to("meta"))):
        with pytest.raises(AssertionError):
            PagedBatch(*bad, 4, 2)


def test_streams_of_another_device_are_refused(monkeypatch):
    """The kernels run on the device of the tensors; another device's stream would not be the one that they run on."""
    from types import SimpleNamespace
    from paper_2508_17892_b200 import paged
    x, pos = torch.zeros(2, 1, 128, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    used = []
    monkeypatch.setattr(paged.torch.cuda, "stream", lambda s: used.append(s) or pytest.fail("the stream was made current"))
    other = SimpleNamespace(device=SimpleNamespace(index=1))
    with pytest.raises(AssertionError):
        paged.rope(x, pos, paged.RopeSpec(), stream=other)
    cache = paged.PagedCache.__new__(paged.PagedCache)
    cache._index = 0
    batch = paged.PagedBatch(torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(2, 1, dtype=torch.int32), 2, 1)
    for call in (lambda: cache.append(batch, x, x, x, None, None, x, x, stream=other),
                 lambda: cache.attention(batch, x, x, x, stream=other), lambda: cache.accumulate(batch, x, x, x, x, stream=other),
                 lambda: cache.evict(batch, 1, 0, 0, x, x, x, stream=other)):
        with pytest.raises(AssertionError):
            call()
    assert not used


def _host_cache(monkeypatch=None):
    """A cache without a handle, as if the host's tensors were its device's, and the calls that reached its library."""
    from paper_2508_17892_b200 import paged
    calls = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: calls.append((name, a)) or 0

    c = paged.PagedCache.__new__(paged.PagedCache)
    c._lib, c._h, c.dtype, c._n_q, c._dim, c._index, c.device = Library(), None, torch.bfloat16, 8, 128, -1, torch.device("cpu")
    c._page_shape, c._weight_shape, c._page_stride = (16, 2, 128), (2, 16), (256, 128, 1)
    if monkeypatch is not None:
        monkeypatch.setattr(paged, "_raw_stream", lambda index: 0)
    return c, calls


def test_pools_of_one_page_shown_many_times_are_refused(monkeypatch):
    """A pool that is one page expanded has a stride of 0 from page to page, which the C call reads as back to back: pages
    that are not there.  Pages that overlap are left to the C call, which refuses their stride."""
    from paper_2508_17892_b200 import PagedBatch
    c, calls = _host_cache(monkeypatch)
    i32 = lambda *n: torch.zeros(*n, dtype=torch.int32)  # noqa: E731
    b = PagedBatch(i32(3), i32(2), i32(2, 4), 4, 2)
    q, k = torch.zeros(4, 8, 128, dtype=torch.bfloat16), torch.zeros(4, 2, 128, dtype=torch.bfloat16)
    page, pool, w = torch.zeros(1, 16, 2, 128, dtype=torch.bfloat16), torch.zeros(3, 16, 2, 128, dtype=torch.bfloat16), torch.zeros(3, 2, 16)
    shown = page.expand(3, 16, 2, 128)
    for kp, vp in ((shown, pool), (pool, shown), (shown, shown)):
        for call in (lambda: c.attention(b, q, kp, vp), lambda: c.append(b, q, k, k, None, None, kp, vp),
                     lambda: c.evict(b, 8, 0, 0, kp, vp, w)):
            with pytest.raises(AssertionError):
                call()
    with pytest.raises(AssertionError):
        c.accumulate(b, q, torch.zeros(4, 8), shown, w)
    assert not calls
    c.attention(b, q, page, page)                            # one page, shown once
    c.attention(b, q, page.expand(1, 16, 2, 128), page)
    c.attention(b, q, pool, torch.zeros(3, 2, 16, 2, 128, dtype=torch.bfloat16)[:, 0])
    strides = [a[4]._obj.v_page_stride for _, a in calls]
    assert strides == [0, 0, 2 * 16 * 2 * 128]


def test_numbers_of_more_than_32_bits_are_refused(monkeypatch):
    """The C structures hold 32 bits; ctypes would cut a larger number down to its low ones."""
    from paper_2508_17892_b200 import PagedBatch, PagedCache, RopeSpec
    c, calls = _host_cache(monkeypatch)
    i32 = lambda *n: torch.zeros(*n, dtype=torch.int32)  # noqa: E731
    big = 1 << 32
    for kw in (dict(n_tokens=big + 4), dict(max_q_len=big + 1), dict(n_tokens=1 << 31), dict(max_q_len=-big)):
        with pytest.raises(AssertionError):
            PagedBatch(i32(3), i32(2), i32(2, 4), **{**dict(n_tokens=4, max_q_len=2), **kw})
    with pytest.raises(AssertionError):
        RopeSpec(rotary_dim=big + 64)
    for name in ("n_kv_heads", "n_q_heads", "page_size", "max_seqs", "head_dim", "device"):
        with pytest.raises(AssertionError):
            PagedCache(**{name: big + 64})
    b = PagedBatch(None, i32(0), i32(0, 4), 0, 0)
    pool, w = torch.zeros(3, 16, 2, 128, dtype=torch.bfloat16), torch.zeros(3, 2, 16)
    for budget, sink, recent in ((big + 8, 0, 0), (8, big, 0), (8, 0, big), (8, 1 - big, 0), (8, 0, 1 - big)):
        with pytest.raises(AssertionError):
            c.evict(b, budget, sink, recent, pool, pool, w)
    assert not calls
    c.evict(b, (1 << 31) - 1, 0, 0, pool, pool, w)           # the C call's to refuse
    assert len(calls) == 1
