"""The paged cache's C entry points without a device: null handles, and the rotary call's refusals (nothing is
launched, no pointer followed, before the arguments have passed)."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    from paper_2508_17892_b200 import build, recall
    build.build()
    return recall.load_library()


def test_null_handles(lib):
    for name in ("status", "last_launch_count", "check_guards", "destroy"):
        assert getattr(lib, "ilre_paged_" + name)(None) == -1
    assert lib.ilre_paged_create(None, None) == -1
    assert lib.ilre_paged_append(None, None, None, None, None, 0, None, 0, None, 0, None, 0, None, None) == -1
    assert lib.ilre_paged_attention(None, None, None, 0, None, None, None, None) == -1
    assert lib.ilre_paged_accumulate(None, None, None, 0, None, None, None) == -1
    assert lib.ilre_paged_evict(None, None, 1, 0, 0, 0, None, None, 0, None, None, None) == -1


def test_create_refuses_before_it_looks_for_a_device(lib):
    from paper_2508_17892_b200.paged import IlrePagedConfig
    good = dict(n_kv_heads=8, n_q_heads=32, head_dim=128, page_size=64, dtype=0, max_seqs=4, device=0)
    out = ctypes.c_void_p()

    def create(**kw):
        cfg = IlrePagedConfig(**{**good, **kw})
        return lib.ilre_paged_create(ctypes.byref(cfg), ctypes.byref(out))

    for kw, code in ((dict(n_kv_heads=0), -1), (dict(dtype=2), -1), (dict(dtype=-1), -1), (dict(page_size=0), -1),
                     (dict(max_seqs=0), -1), (dict(device=-1), -1), (dict(head_dim=64), -2), (dict(n_q_heads=12), -2),
                     (dict(n_kv_heads=1, n_q_heads=129), -2), (dict(page_size=8), -2), (dict(page_size=24), -2),
                     (dict(page_size=2048), -2), (dict(max_seqs=65536), -3), (dict(n_kv_heads=2048, n_q_heads=2048), -3)):
        assert create(**kw) == code, kw
    assert out.value is None


def test_rope_refusals(lib):
    from paper_2508_17892_b200.paged import IlreRopeSpec
    good = dict(theta=10000.0, rotary_dim=64, layout=0, scaling=0, factor=1.0, orig_len=0.0, low=0.0, high=0.0,
                attn_factor=0.0)
    x, odd = 4096, 4098                                    # never read: refused first

    def call(n_tokens=4, n_heads=2, head_dim=128, dtype=0, xp=x, xs=256, op=x, os_=256, pos=x, **kw):
        spec = IlreRopeSpec(**{**good, **kw})
        return lib.ilre_rope(ctypes.byref(spec), xp, xs, op, os_, pos, n_tokens, n_heads, head_dim, dtype, 0, None)

    for kw, code in ((dict(theta=1.0), -1), (dict(theta=float("nan")), -1), (dict(theta=float("inf")), -1),
                     (dict(rotary_dim=0), -1), (dict(rotary_dim=24), -2), (dict(rotary_dim=144), -2),
                     (dict(rotary_dim=272, head_dim=512, xs=1024, os_=1024), -2), (dict(layout=2), -1), (dict(scaling=4), -1),
                     (dict(scaling=1, factor=0.5), -1), (dict(scaling=2, factor=2.0), -1),
                     (dict(scaling=2, factor=2.0, orig_len=8192.0, low=4.0, high=1.0), -1),
                     (dict(scaling=3, factor=2.0, orig_len=8192.0, low=0.0, high=32.0), -1),
                     (dict(scaling=3, factor=2.0, orig_len=8192.0, low=1.0, high=float("inf")), -1),
                     (dict(attn_factor=-1.0), -1), (dict(attn_factor=float("nan")), -1), (dict(n_tokens=-1), -1),
                     (dict(n_heads=0), -1), (dict(head_dim=120), -2), (dict(head_dim=2048), -2), (dict(dtype=2), -1),
                     (dict(n_heads=70000), -3), (dict(n_tokens=2 ** 31), -3), (dict(pos=None), -1), (dict(xp=None), -1),
                     (dict(op=None), -1), (dict(xs=255), -1), (dict(xs=260), -5), (dict(xp=odd), -5), (dict(op=odd), -5),
                     (dict(os_=128), -1), (dict(pos=odd), -5)):
        assert call(**kw) == code, kw
    assert lib.ilre_rope(None, x, 256, x, 256, x, 4, 2, 128, 0, 0, None) == -1
    assert call(n_tokens=0, xp=None, op=None, pos=None) == 0


def test_the_bindings_constants_are_the_headers():
    from paper_2508_17892_b200 import paged
    text = open(os.path.join(ROOT, "include", "ilre_recall.h")).read()
    value = {k: int(v) for k, v in re.findall(r"#define (ILRE_\w+) (\d+)\n", text)}
    assert {str(k).rsplit(".")[-1]: v for k, v in paged._DTYPES.items()} == {"bfloat16": value["ILRE_BF16"],
                                                                          "float16": value["ILRE_F16"]}
    assert paged._SCALINGS == {"none": value["ILRE_ROPE_PLAIN"], "linear": value["ILRE_ROPE_LINEAR"],
                               "banded": value["ILRE_ROPE_BANDED"], "yarn": value["ILRE_ROPE_YARN"]}


def test_rope_in_place_needs_one_stride(lib):
    from paper_2508_17892_b200.paged import IlreRopeSpec
    spec = IlreRopeSpec(10000.0, 64, 0, 0, 1.0, 0.0, 0.0, 0.0, 0.0)
    call = lambda xs, os_: lib.ilre_rope(ctypes.byref(spec), 4096, xs, 4096, os_, 4096, 4, 2, 128, 0, 0, None)  # noqa: E731
    assert call(256, 512) == -1 and call(512, 256) == -1


def test_rope_specs_are_copied_and_pickled():
    import copy
    import pickle
    from paper_2508_17892_b200 import RopeSpec
    a = RopeSpec(theta=10000.0, rotary_dim=64, interleaved=True, scaling="yarn", factor=4.0, low=1.0, high=32.0)
    for b in (copy.copy(a), copy.deepcopy(a), pickle.loads(pickle.dumps(a))):
        assert b == a and bytes(b._c) == bytes(a._c) and b.ref is not a.ref
