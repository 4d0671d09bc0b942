"""Refusals of the rotary and paged calls that need no GPU: every bad size,
stride, pointer and rotation is turned away before anything is enqueued."""
import ctypes

import pytest

from paper_2606_10671_amd import fademem as fm

F32, BF16 = fm.FADEMEM_F32, fm.FADEMEM_BF16
A = 1 << 20  # an aligned address that is never read


@pytest.mark.parametrize("args", [(128, 0, 22, 21, 22, 1e4), (128, 2, 22, 21, 21, 1e4), (120, 0, 8, 8, 8, 1e4),
                                  (0, 0, 1, 0, 0, 1e4), (272, 0, 8, 8, 8, 1e4), (64, 0, 0, 0, 0, 1e4),
                                  (64, 0, -1, 8, 8, 1e4), (64, 0, 8, 8, 8, 1.0), (64, 0, 8, 8, 8, float("nan")),
                                  (64, 0, 8, 8, 8, float("inf")), (64, -1, 8, 8, 8, 1e4),
                                  (64, 0, 2**31 - 1, 2**31 - 1, 2**31 - 1, 1e4)])
def test_bad_rotations_are_refused(args):
    with pytest.raises(fm.FademError) as e:
        fm.fademem_rope_init(*args)
    assert e.value.code == fm.FADEMEM_EINVAL


def test_rope_init_gives_each_axis_its_frequencies():
    r = fm.fademem_rope_init(128, 0, 22, 21, 21, 10000.0)
    want = [10000.0 ** (-k / n) for n in (22, 21, 21) for k in range(n)]
    assert all(abs(r.freq[i] - w) <= 4e-16 * w for i, w in enumerate(want))
    assert list(r.pairs) == [22, 21, 21] and r.head_dim == 128


GOOD = dict(dtype=BF16, pos_ptr=A, rows=8, heads=2, x_ptr=A, x_stride=128, y_ptr=2 * A, y_stride=128, inverse=0)


@pytest.mark.parametrize("change", [dict(dtype=2), dict(pos_ptr=0), dict(pos_ptr=A + 2), dict(rows=-1),
                                    dict(rows=(1 << 23) + 1), dict(heads=0), dict(heads=5000), dict(x_ptr=0),
                                    dict(x_ptr=A + 8), dict(y_ptr=2 * A + 2), dict(y_ptr=0), dict(x_stride=127),
                                    dict(x_stride=132), dict(y_stride=120), dict(y_stride=-128), dict(inverse=2),
                                    dict(y_ptr=A + 128),                     # one row over another
                                    dict(y_ptr=A, y_stride=256),             # the same start, other rows
                                    dict(x_stride=256, y_stride=256, y_ptr=A + 240),
                                    dict(x_stride=(1 << 32) + 8)])
def test_bad_rope_calls_are_refused(change):
    rope = fm.fademem_rope_init(64, 0, 8, 8, 8, 1e4)
    with pytest.raises(fm.FademError) as e:
        fm.fademem_rope_apply(rope, **{**GOOD, **change})
    assert e.value.code == fm.FADEMEM_EINVAL


def test_rope_with_changed_fields_is_checked_again():
    for field, value in (("head_dim", 72), ("layout", 3)):
        rope = fm.fademem_rope_init(64, 0, 8, 8, 8, 1e4)
        setattr(rope, field, value)
        with pytest.raises(fm.FademError):
            fm.fademem_rope_apply(rope, **GOOD)
    rope = fm.fademem_rope_init(64, 0, 8, 8, 8, 1e4)
    rope.freq[23] = float("inf")
    with pytest.raises(fm.FademError):
        fm.fademem_rope_apply(rope, **GOOD)
    rope.freq[23] = 0.5
    fm.fademem_rope_apply(rope, **{**GOOD, "rows": 0, "x_ptr": 0, "y_ptr": 0, "pos_ptr": 0})  # no rows: nothing to do
    assert fm.lib().fademem_rope_apply(None, BF16, A, 8, 2, A, 128, 2 * A, 128, 0, None) == fm.FADEMEM_EINVAL


CONFIG = dict(seqs=4, layers=2, heads=8, kv_heads=2, head_dim=128, dtype=BF16, page_tokens=64, sinks=1, pages=100,
              max_tokens=5000, max_rows=300, block_tokens=1, window=1000, grid_h=1, grid_w=1)


def test_paged_bytes():
    n = fm.fademem_paged_bytes(fm.fademem_paged_config(**CONFIG))
    pages = 2 * 100 * 2 * 2 * 64 * 128 * 2
    scratch = 2 * 256 * 256 * (128 + 2) * 4  # two slots a workgroup: O, row max, row sum of 256 rows
    assert pages + scratch <= n <= pages + scratch + 64 * 1024


@pytest.mark.parametrize("field,value", [("seqs", 0), ("seqs", 1025), ("layers", 0), ("layers", 4097), ("heads", 7),
                                         ("heads", 0), ("kv_heads", 0), ("kv_heads", 3), ("head_dim", 96),
                                         ("dtype", 2), ("page_tokens", 0), ("page_tokens", 65537), ("pages", 0),
                                         ("pages", (1 << 24) + 1), ("max_tokens", 0), ("max_tokens", (1 << 30) + 1),
                                         ("max_rows", 0), ("max_rows", (1 << 23) + 1), ("block_tokens", 0),
                                         ("block_tokens", (1 << 30) + 1), ("window", -1),
                                         ("window", (1 << 30) + 1), ("sinks", -1), ("grid_h", 0), ("grid_w", 0),
                                         ("grid_h", (1 << 30) + 1)])
def test_bad_paged_configs_are_refused(field, value):
    with pytest.raises(fm.FademError) as e:
        fm.fademem_paged_bytes(fm.fademem_paged_config(**{**CONFIG, field: value}))
    assert e.value.code == fm.FADEMEM_EINVAL


def test_sinks_without_a_window_are_allowed():
    """Everything is visible then; the sinks are among it."""
    assert fm.fademem_paged_bytes(fm.fademem_paged_config(**{**CONFIG, "window": 0})) > 0


def test_sizes_that_overflow_are_refused():
    big = {**CONFIG, "pages": 1 << 24, "page_tokens": 65536, "layers": 4096, "kv_heads": 4096, "heads": 4096}
    with pytest.raises(fm.FademError):
        fm.fademem_paged_bytes(fm.fademem_paged_config(**big))
    rows = {**CONFIG, "max_rows": 1 << 23, "heads": 4096, "kv_heads": 1}
    with pytest.raises(fm.FademError):
        fm.fademem_paged_bytes(fm.fademem_paged_config(**rows))


def test_create_validates_before_touching_the_device():
    cfg = fm.fademem_paged_config(**CONFIG)
    need = fm.fademem_paged_bytes(cfg)
    L, h = fm.lib(), ctypes.c_void_p(0)
    assert L.fademem_paged_create(cfg, None, need, None, ctypes.byref(h)) == fm.FADEMEM_EINVAL
    assert L.fademem_paged_create(cfg, 4096 + 16, need, None, ctypes.byref(h)) == fm.FADEMEM_EINVAL
    assert L.fademem_paged_create(cfg, 4096, need - 1, None, ctypes.byref(h)) == fm.FADEMEM_ENOMEM
    assert L.fademem_paged_create(cfg, 4096, need, None, None) == fm.FADEMEM_EINVAL
    assert L.fademem_paged_create(None, 4096, need, None, ctypes.byref(h)) == fm.FADEMEM_EINVAL
    assert h.value is None and L.fademem_paged_bytes(cfg, None) == fm.FADEMEM_EINVAL


def test_null_stores_are_refused():
    L = fm.lib()
    p, n = ctypes.c_void_p(0), ctypes.c_int64(0)
    assert L.fademem_paged_plan(None, A, A, 1, 1, None) == fm.FADEMEM_EINVAL
    assert L.fademem_paged_array(None, 0, 0, ctypes.byref(p), ctypes.byref(n)) == fm.FADEMEM_EINVAL
    assert L.fademem_paged_insert(None, 0, A, 256, A, 256, None, None) == fm.FADEMEM_EINVAL
    assert L.fademem_paged_attend(None, 0, A, 1024, ctypes.c_float(0), A, 1024, None, None) == fm.FADEMEM_EINVAL
    assert L.fademem_paged_destroy(None) == fm.FADEMEM_OK
    assert L.fademem_paged_last_hip_error(None) == 0


def test_the_binding_refuses_unknown_names():
    from paper_2606_10671_amd.rotary import Rotary
    with pytest.raises(ValueError):
        Rotary(64, (8, 8, 8), layout="thirds")
    with pytest.raises(ValueError):
        Rotary(64, (8, 8))
    with pytest.raises(ValueError):
        Rotary(64, (8, 8, 8), freq=[1.0])
