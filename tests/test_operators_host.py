"""Row and prefix calls without a device: what they refuse, and the oracle's forms against closed ones."""
import ctypes as C

import numpy as np
import pytest

from oracle import lazyev_oracle as orc
from paper_2506_15969_b200 import binding


@pytest.fixture
def handle():
    lib, h = binding.lib(), C.c_void_p()
    assert lib.lazyev_create(C.byref(h), 2, 8, 2, 128, 512, 128, 1e-3) == binding.OK
    yield h
    assert lib.lazyev_destroy(h) == binding.OK


def freqs(*values):
    return (C.c_double * max(1, len(values)))(*values)


@pytest.mark.parametrize("pairs,values,amplitude", [
    (7, [1.0] * 64, 1.0), (-8, [1.0] * 64, 1.0), (72, [1.0] * 72, 1.0), (8, [float("nan")] * 8, 1.0), (8, [float("inf")] * 8, 1.0),
    (8, [1.0] * 8, float("nan")), (8, [1.0] * 8, float("inf")),
])
def test_set_rope_refuses(handle, pairs, values, amplitude):
    assert binding.lib().lazyev_set_rope(handle, freqs(*values), pairs, 0, amplitude) == binding.EINVAL
    assert binding.lib().lazyev_last_error(handle)


def test_set_rope_and_norm_arguments(handle):
    lib = binding.lib()
    assert lib.lazyev_set_rope(handle, None, 8, 0, 1.0) == binding.EINVAL
    assert lib.lazyev_set_rope(handle, None, 0, 0, 1.0) == binding.OK
    assert lib.lazyev_set_rope(handle, freqs(*[0.5] * 64), 64, 1, -2.0) == binding.OK
    assert lib.lazyev_set_rope(None, None, 0, 0, 1.0) == binding.EINVAL
    assert lib.lazyev_set_head_norm(handle, 8, None, 1e-6) == binding.EINVAL           # misaligned
    for eps in (0.0, -1.0, float("nan"), float("inf")):
        assert lib.lazyev_set_head_norm(handle, 256, None, eps) == binding.EINVAL
    assert lib.lazyev_set_head_norm(handle, 256, 512, 1e-6) == binding.OK
    assert lib.lazyev_set_head_norm(handle, None, None, 0.0) == binding.OK             # off
    assert lib.lazyev_set_head_norm(None, None, None, 1e-6) == binding.EINVAL


def test_calls_that_need_a_bound_handle(handle):
    lib, bytes_ = binding.lib(), C.c_size_t()
    assert lib.lazyev_norm_rope(handle, 256, 256, 1, None, 0, 256, 256) == binding.ESTATE
    assert lib.lazyev_append(handle, 256, 256, 1, None) == binding.ESTATE
    assert lib.lazyev_decode_step_rows(handle, 256, 256, 256, None, 256) == binding.ESTATE
    assert lib.lazyev_attend(handle, 256, 256) == binding.ESTATE
    other = C.c_void_p()
    assert lib.lazyev_create(C.byref(other), 2, 8, 2, 128, 512, 128, 1e-3) == binding.OK
    assert lib.lazyev_query_prefix_workspace(handle, other, C.byref(bytes_)) == binding.ESTATE
    assert lib.lazyev_attach_prefix(handle, other, 256) == binding.ESTATE
    assert lib.lazyev_attach_prefix(handle, handle, 256) == binding.EINVAL
    assert lib.lazyev_detach_prefix(handle) == binding.OK                              # nothing attached
    assert lib.lazyev_destroy(other) == binding.OK
    for call, args in (("norm_rope", (256, 256, 1, None, 0, 256, 256)), ("append", (256, 256, 1, None)), ("attend", (256, 256)),
                       ("detach_prefix", ()), ("decode_step_rows", (256, 256, 256, None, 256)), ("attach_prefix", (other, 256))):
        assert getattr(lib, "lazyev_" + call)(None, *args) == binding.EINVAL


def test_state_layout_follows_the_sizes(handle):
    lib = binding.lib()
    off = [C.c_size_t() for _ in range(4)]
    assert lib.lazyev_query_state_layout(handle, *(C.byref(o) for o in off)) == binding.OK
    info, kv, st, sc = binding.Info(), C.c_size_t(), C.c_size_t(), C.c_size_t()
    lib.lazyev_get_info(handle, C.byref(info))
    lib.lazyev_query_sizes(handle, C.byref(kv), C.byref(st), C.byref(sc))
    slots = info.units * info.capacity
    table, ts_mri, pos, pbar = (o.value for o in off)
    assert table == 0 and ts_mri >= 4 * info.units * info.pages_per_unit and pos >= ts_mri + 8 * slots and pbar >= pos + 4 * slots
    assert pbar + 4 * slots <= st.value and all(o % 256 == 0 for o in (ts_mri, pos, pbar))
    assert (info.prefix_tokens, info.prefix_blocks, info.next_position) == (0, 0, 0)


# ---- the oracle -------------------------------------------------------------------------------------------------------

def test_oracle_norm_rope_closed_forms():
    r = np.random.RandomState(0)
    x, w = r.randn(5, 3, 128), r.rand(128) + 0.5
    f = [10.0 ** (-j / 16) for j in range(64)]
    for inter in (False, True):
        y = orc.norm_rope(x, None, 0, np.zeros(5), f, inter)
        assert np.allclose(y, x)                                                       # position 0
        y = orc.norm_rope(x, None, 0, np.arange(5) * 1000, f, inter, 1.5)
        assert np.allclose((y ** 2).sum(-1), 2.25 * (x ** 2).sum(-1))                  # a rotation, times the amplitude
        # scores depend on distances only
        q, k = orc.norm_rope(x, None, 0, np.arange(5) + 70, f, inter), orc.norm_rope(x, None, 0, np.arange(5) + 30, f, inter)
        q2, k2 = orc.norm_rope(x, None, 0, np.arange(5) + 47, f, inter), orc.norm_rope(x, None, 0, np.arange(5) + 7, f, inter)
        assert np.allclose(np.einsum("ihd,jhd->hij", q, k), np.einsum("ihd,jhd->hij", q2, k2))
        # a quarter turn
        e = np.zeros((1, 128))
        e[0, 0] = 1.0
        z = orc.norm_rope(e, None, 0, [1.0], [np.pi / 2] + [0.0] * 63, inter)
        assert np.isclose(z[0, 1 if inter else 64], 1.0) and np.isclose(abs(z).sum(), 1.0)
        part = orc.norm_rope(x, None, 0, np.arange(5), f[:8], inter)
        assert np.array_equal(part[..., 16:], x[..., 16:]) and not np.allclose(part[1:, :, :16], x[1:, :, :16])
    y = orc.norm_rope(x, w, 0.0, np.zeros(5), [])
    assert np.allclose(((y / w) ** 2).mean(-1), 1.0)


def test_oracle_prefixed_unit_is_a_unit_that_never_evicts_its_prefix():
    r = np.random.RandomState(1)
    kp, vp, K, V = r.randn(9, 128), r.randn(9, 128), r.randn(4, 128), r.randn(4, 128)
    a = orc.PrefixedUnit(kp, vp, 9, 2, 128, 100, 10, 0.05)
    b = orc.OracleUnit(2, 128, 100, 10, 0.05)
    a.load(K, V)
    b.prefill(np.vstack([kp, K]), np.vstack([vp, V]))
    for _ in range(6):
        q, kn, vn = r.randn(2, 128) * 2, r.randn(128), r.randn(128)
        oa, pa = a.attend(q, kn, vn)
        ob, pb = b.attend(q, kn, vn)
        assert np.allclose(oa, ob) and np.allclose(pa, pb[9:])
        a.track(pa), b.track(pb)
        assert np.array_equal(a.pos, b.pos[9:]) and np.array_equal(a.TS, b.TS[9:]) and np.array_equal(a.MRI, b.MRI[9:])
