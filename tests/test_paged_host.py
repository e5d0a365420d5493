"""Argument checks of the paged-cache calls (all made before any HIP call) and
the rotary frequency tables."""
import ctypes

import numpy as np
import pytest

from paper_2606_00422_amd import upr
from tests.paged_util import frequencies

A = 1 << 12         # an aligned address that nothing dereferences


@pytest.mark.parametrize("rot", [2, 4, 10, 32, 64, 128])
@pytest.mark.parametrize("scaling", ["none", "linear", "ntk", "by_parts"])
def test_rope_frequencies(rot, scaling):
    if scaling == "ntk" and rot == 2:
        with pytest.raises(upr.UprError) as e:
            upr.rope(rot, scaling=scaling, factor=2.0)
        assert e.value.status == upr.UPR_ERR_LIMIT
        return
    r = upr.rope(rot, 50000.0, "interleaved", scaling, 8.0, 4096)
    f, mag = frequencies(rot, 50000.0, scaling, 8.0, 4096)
    assert r.rot_dim == rot and r.layout == upr.UPR_ROPE_INTERLEAVED
    np.testing.assert_allclose(list(r.freq)[:rot // 2], f, rtol=1e-13)
    assert r.magnitude == pytest.approx(mag, rel=1e-14)
    assert not any(list(r.freq)[rot // 2:])


@pytest.mark.parametrize("args", [
    (0, 0, 1e4, 0, 1.0, 0.0), (3, 0, 1e4, 0, 1.0, 0.0), (130, 0, 1e4, 0, 1.0, 0.0), (-2, 0, 1e4, 0, 1.0, 0.0),
    (64, 2, 1e4, 0, 1.0, 0.0), (64, 0, 1.0, 0, 1.0, 0.0), (64, 0, float("nan"), 0, 1.0, 0.0),
    (64, 0, 1e4, 4, 1.0, 0.0), (64, 0, 1e4, 1, 0.5, 0.0), (64, 0, 1e4, 1, float("inf"), 0.0),
    (64, 0, 1e4, 3, 2.0, 0.0), (64, 0, 1e4, 3, 2.0, float("inf")), (4, 0, 1e300, 2, 1e300, 0.0),
])
def test_rope_init_refusals(args):
    out = upr.upr_rope()
    out.rot_dim = 7
    assert upr.load().upr_rope_init(*args, ctypes.byref(out)) == upr.UPR_ERR_LIMIT
    assert out.rot_dim == 7 and upr.upr_last_error()
    assert upr.load().upr_rope_init(*args, None) == upr.UPR_ERR_NULL


def _rope(rot=64):
    return upr.rope(rot)


@pytest.mark.parametrize("change,status", [
    ({}, upr.UPR_ERR_NULL),                                   # no rope
    (dict(rope=_rope, dtype=5), upr.UPR_ERR_DTYPE),
    (dict(rope=_rope, dtype=upr.UPR_BF16_MXFP8), upr.UPR_ERR_DTYPE),
    (dict(rope=_rope, dim=48), upr.UPR_ERR_CONFIG),
    (dict(rope=_rope, dim=32), upr.UPR_ERR_LIMIT),            # rot_dim past the head
    (dict(rope=_rope, heads=0), upr.UPR_ERR_LIMIT),
    (dict(rope=_rope, heads=4096), upr.UPR_ERR_LIMIT),
    (dict(rope=_rope, rows=-1), upr.UPR_ERR_LIMIT),
    (dict(rope=_rope, rows=1 << 31), upr.UPR_ERR_LIMIT),
    (dict(rope=_rope, x=0), upr.UPR_ERR_NULL),
    (dict(rope=_rope, out=0), upr.UPR_ERR_NULL),
    (dict(rope=_rope, pos=0), upr.UPR_ERR_NULL),
    (dict(rope=_rope, x=A + 8), upr.UPR_ERR_LIMIT),
    (dict(rope=_rope, ld=255), upr.UPR_ERR_LIMIT),            # shorter than a row
    (dict(rope=_rope, ld=260), upr.UPR_ERR_LIMIT),            # not 16 bytes
    (dict(rope=_rope, out=A, old=264), upr.UPR_ERR_LIMIT),    # in place, other stride
    (dict(rope=_rope, rows=0, x=0, out=0, pos=0), upr.UPR_OK),
])
def test_rope_apply_refusals(change, status):
    a = dict(rope=lambda: None, dtype=upr.UPR_BF16, heads=4, dim=64, x=A, ld=256, pos=A, rows=3, out=A + 65536, old=256)
    a.update(change)
    r = a["rope"]()
    st = upr.load().upr_rope_apply(None if r is None else ctypes.byref(r), a["dtype"], a["heads"], a["dim"], a["x"],
                                   a["ld"], a["pos"], a["rows"], a["out"], a["old"], None)
    assert st == status


def test_rope_apply_checks_a_struct_filled_by_hand():
    lib = upr.load()
    for field, value in [("rot_dim", 7), ("rot_dim", 0), ("layout", 9), ("magnitude", float("inf")), ("magnitude", 1e300)]:
        r = _rope()
        setattr(r, field, value)
        assert lib.upr_rope_apply(ctypes.byref(r), 1, 4, 64, A, 256, A, 3, A, 256, None) == upr.UPR_ERR_LIMIT
    for bad in (float("nan"), 1e9):
        r = _rope()
        r.freq[31] = bad
        assert lib.upr_rope_apply(ctypes.byref(r), 1, 4, 64, A, 256, A, 3, A, 256, None) == upr.UPR_ERR_LIMIT


class Call:
    """One paged call's arguments, aligned made-up addresses by default."""

    def __init__(self, counts=(2, 0, 3), rows=(5, 9, 40), **kw):
        self.off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        self.rows = None if rows is None else np.asarray(rows, np.int32)
        self.shape = upr.upr_attn_shape(upr.UPR_BF16, 8, 2, 64)
        self.cache = upr.upr_paged_cache(A, 10, 16, 3, A)
        self.opt = upr.upr_attn_options(0.125, 0.0, 0, None, None, None, 0)
        self.seg = upr.segments(self.off)
        self.p = dict(q=A, q_ld=512, k=A, k_ld=128, v=A, v_ld=128, out=A, out_ld=512, rope=None, ws=A, ws_bytes=1 << 40)
        for key, v in kw.items():
            obj, _, field = key.partition("__")
            if obj == "p":
                self.p[field] = v
            elif field:
                setattr(getattr(self, obj), field, v)
            else:
                setattr(self, obj, v)

    def _ref(self, x):
        return None if x is None else ctypes.byref(x)

    def append(self):
        p = self.p
        return upr.load().upr_paged_append(self._ref(self.shape), self._ref(self.cache), self._ref(self.seg),
                                           None if self.rows is None else self.rows.ctypes.data, self._ref(p["rope"]),
                                           p["k"], p["k_ld"], p["v"], p["v_ld"], p["q"], p["q_ld"], p["out"],
                                           p["out_ld"], None)

    def attend(self):
        p = self.p
        return upr.load().upr_paged_attention(self._ref(self.shape), self._ref(self.cache), self._ref(self.seg),
                                              None if self.rows is None else self.rows.ctypes.data, self._ref(self.opt),
                                              p["q"], p["q_ld"], p["out"], p["out_ld"], p["ws"], p["ws_bytes"], None)

    def bytes(self):
        return upr.load().upr_paged_attention_workspace_bytes(
            self._ref(self.shape), self._ref(self.cache), self._ref(self.seg),
            None if self.rows is None else self.rows.ctypes.data, self._ref(self.opt))


COMMON = [
    (dict(shape=None), upr.UPR_ERR_NULL), (dict(cache=None), upr.UPR_ERR_NULL), (dict(seg=None), upr.UPR_ERR_NULL),
    (dict(rows=None), upr.UPR_ERR_NULL), (dict(seg__offsets_host=None), upr.UPR_ERR_NULL),
    (dict(shape__dtype=2), upr.UPR_ERR_DTYPE), (dict(shape__dtype=-1), upr.UPR_ERR_DTYPE),
    (dict(shape__head_dim=96), upr.UPR_ERR_CONFIG), (dict(shape__n_kv_heads=0), upr.UPR_ERR_CONFIG),
    (dict(shape__n_kv_heads=3), upr.UPR_ERR_CONFIG), (dict(shape__n_heads=1), upr.UPR_ERR_CONFIG),
    (dict(shape__n_heads=2048), upr.UPR_ERR_CONFIG),
    (dict(cache__page_rows=8), upr.UPR_ERR_LIMIT), (dict(cache__page_rows=48), upr.UPR_ERR_LIMIT),
    (dict(cache__page_rows=2048), upr.UPR_ERR_LIMIT), (dict(cache__page_rows=0), upr.UPR_ERR_LIMIT),
    (dict(cache__n_pages=-1), upr.UPR_ERR_LIMIT), (dict(cache__n_pages=1 << 31), upr.UPR_ERR_LIMIT),
    (dict(cache__table_stride=-1), upr.UPR_ERR_LIMIT), (dict(cache__table_stride=2), upr.UPR_ERR_CAPACITY),
    (dict(seg__num_users=-1), upr.UPR_ERR_OFFSETS), (dict(rows=(5, -1, 40)), upr.UPR_ERR_OFFSETS),
    (dict(rows=(1, 9, 40)), upr.UPR_ERR_OFFSETS), (dict(counts=(2, -1, 3)), upr.UPR_ERR_OFFSETS),
    (dict(rows=(5, 9, (1 << 30) + 1)), upr.UPR_ERR_LIMIT),
    (dict(counts=((1 << 22) + 1, 0, 3), rows=(1 << 23, 9, 40), cache__table_stride=1 << 20), upr.UPR_ERR_LIMIT),
    (dict(counts=(1 << 20, 0, 3), rows=(1 << 20, 9, 40), cache__table_stride=1 << 20, shape__n_heads=256), upr.UPR_ERR_LIMIT),
    (dict(cache__data=None), upr.UPR_ERR_NULL), (dict(cache__tables=None), upr.UPR_ERR_NULL),
    (dict(cache__data=A + 4), upr.UPR_ERR_LIMIT),
    (dict(p__q=A + 2), upr.UPR_ERR_LIMIT), (dict(p__q_ld=511), upr.UPR_ERR_LIMIT), (dict(p__q_ld=516), upr.UPR_ERR_LIMIT),
    (dict(p__out_ld=504), upr.UPR_ERR_LIMIT), (dict(p__out=A + 8), upr.UPR_ERR_LIMIT), (dict(p__out=None), upr.UPR_ERR_NULL),
    (dict(p__q=None), upr.UPR_ERR_NULL),
]


@pytest.mark.parametrize("kw,status", COMMON + [
    (dict(p__k=None), upr.UPR_ERR_NULL), (dict(p__v=None), upr.UPR_ERR_NULL), (dict(p__k_ld=64), upr.UPR_ERR_LIMIT),
    (dict(p__v_ld=130), upr.UPR_ERR_LIMIT), (dict(p__out_ld=1024), upr.UPR_ERR_LIMIT),     # in place, other stride
    (dict(p__rope=upr.rope(128)), upr.UPR_ERR_LIMIT),
])
def test_append_refusals(kw, status):
    assert Call(**kw).append() == status
    assert upr.upr_last_error()


@pytest.mark.parametrize("kw,status", COMMON + [
    (dict(opt=None), upr.UPR_ERR_NULL), (dict(opt__scale=0.0), upr.UPR_ERR_LIMIT), (dict(opt__scale=-1.0), upr.UPR_ERR_LIMIT),
    (dict(opt__scale=float("nan")), upr.UPR_ERR_LIMIT), (dict(opt__scale=float("inf")), upr.UPR_ERR_LIMIT),
    (dict(opt__softcap=-1.0), upr.UPR_ERR_LIMIT), (dict(opt__softcap=float("inf")), upr.UPR_ERR_LIMIT),
    (dict(opt__softcap=1e-44), upr.UPR_ERR_LIMIT), (dict(opt__window=-1), upr.UPR_ERR_LIMIT),
    (dict(opt__k_self=A), upr.UPR_ERR_NULL), (dict(opt__v_self=A), upr.UPR_ERR_NULL),
    (dict(opt__k_self=A, opt__v_self=A, opt__self_ld=64), upr.UPR_ERR_LIMIT),
    (dict(opt__k_self=A + 8, opt__v_self=A, opt__self_ld=128), upr.UPR_ERR_LIMIT),
    (dict(opt__k_self=A, opt__v_self=A + 8, opt__self_ld=128), upr.UPR_ERR_LIMIT),
])
def test_attention_refusals(kw, status):
    assert Call(**kw).attend() == status
    assert upr.upr_last_error()


def test_calls_without_rows_touch_nothing():
    none = dict(counts=(0, 0), rows=(5, 900), cache__data=None, cache__tables=None, p__q=None, p__k=None, p__v=None,
                p__out=None, p__ws=None, p__ws_bytes=0)
    assert Call(**none).append() == upr.UPR_OK and Call(**none).attend() == upr.UPR_OK
    assert Call(**none).bytes() == 0
    no_users = Call()
    no_users.seg.num_users, no_users.rows = 0, None
    assert no_users.attend() == upr.UPR_OK and no_users.append() == upr.UPR_OK


def test_attention_workspace_is_checked():
    # one row over a long history: split over the device, joined from the workspace
    long = dict(counts=(1,), rows=(40000,), cache__table_stride=4000, cache__n_pages=4000)
    need = Call(**long).bytes()
    if need > 0:
        assert Call(p__ws_bytes=need - 1, **long).attend() == upr.UPR_ERR_WORKSPACE
        assert Call(p__ws=A + 16, **long).attend() == upr.UPR_ERR_WORKSPACE
        assert Call(p__ws=None, **long).attend() == upr.UPR_ERR_NULL
    assert Call(rows=(1, 1, 1)).bytes() == 0            # invalid: fewer rows than queries


def test_paged_cache_bytes():
    cfg = upr.make_config(128, 2, 3, 256, "bf16")
    assert upr.upr_paged_cache_bytes(cfg, 10, 64) == 3 * 10 * 2 * 2 * 64 * 64 * 2
    assert upr.upr_paged_cache_bytes(cfg, -1, 64) == 0 and upr.upr_paged_cache_bytes(cfg, 10, 63) == 0
    assert upr.upr_paged_cache_bytes(upr.make_config(96, 3, 1, 256, "bf16"), 10, 64) == 0


def test_model_calls_refuse_before_any_hip_call():
    lib = upr.load()
    c = Call()
    assert lib.upr_extend_user(None, ctypes.byref(c.cache), None, ctypes.byref(c.seg), c.rows.ctypes.data, None, None, 0,
                               None) == upr.UPR_ERR_NULL
    assert lib.upr_rank_candidates_paged(None, ctypes.byref(c.cache), c.rows.ctypes.data, None, ctypes.byref(c.seg), None,
                                         None, None, 0, None) == upr.UPR_ERR_NULL
    assert lib.upr_extend_workspace_bytes(None, ctypes.byref(c.cache), ctypes.byref(c.seg), c.rows.ctypes.data) == 0
    assert lib.upr_rank_paged_workspace_bytes(None, ctypes.byref(c.cache), ctypes.byref(c.seg), c.rows.ctypes.data) == 0
