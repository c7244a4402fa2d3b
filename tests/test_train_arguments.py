"""What the entry points of a training step in few bits refuse, before any launch (no GPU)."""
import ctypes
import math

import pytest
import torch

from paper_2302_02390_amd import binding as qb

OK, ODD, EIGHT, FOUR = (ctypes.c_void_p(4096 + i) for i in (0, 1, 8, 4))
BIG = 1 << 31
E, A = qb.QSDP_EINVAL, qb.QSDP_EALIGN


def _variants(name, good, changes):
    """Every change of one argument of a call that would be launched is refused with its status."""
    fn = getattr(qb.lib(), name)
    for at, value, status in changes:
        args = list(good)
        args[at] = value
        assert fn(*args) == status, (name, at, value)


def test_layer_norm():
    good = [OK, 1, 4, 100, 100, OK, OK, 0, 1e-5, OK, 1, 104, OK, None]
    _variants("qsdp_layer_norm", good, [
        (0, None, E), (0, ODD, A), (1, 3, E), (1, 2, E), (1, -1, E), (2, BIG, E), (3, 0, E), (3, (1 << 24) + 1, E), (4, 99, E),
        (5, ODD, A), (6, ODD, A), (7, 2, E), (7, 5, E), (8, -1e-5, E), (8, math.nan, E), (8, math.inf, E), (9, None, E), (9, ODD, A),
        (10, 0, E), (10, 2, E), (11, 99, E), (12, ODD, A)])
    assert qb.lib().qsdp_layer_norm(None, 1, 0, 100, 0, None, None, 0, 1e-5, None, 1, 0, None, None) == qb.QSDP_OK


def test_layer_norm_backward():
    room = qb.layer_norm_backward_bytes(4, 100)
    assert room == 2 * 100 * 4  # four rows of one workgroup
    good = [OK, 1, 4, 100, 100, OK, 0, OK, OK, 1, 100, OK, 100, OK, OK, 0, OK, room, None]
    _variants("qsdp_layer_norm_backward", good, [
        (0, None, E), (0, ODD, A), (1, 7, E), (1, 2, E), (2, BIG, E), (3, 0, E),
        (4, 99, E), (5, ODD, A), (6, 2, E), (7, None, E), (7, ODD, A), (8, None, E), (8, ODD, A), (9, 0, E), (10, 99, E),
        (11, ODD, A), (12, 99, E), (13, ODD, A), (14, ODD, A), (16, None, E), (16, EIGHT, A), (17, room - 1, E)])
    none = list(good)
    none[11] = none[13] = none[14] = None
    assert qb.lib().qsdp_layer_norm_backward(*none) == E
    assert qb.layer_norm_backward_bytes(4, 0) == 0 and qb.layer_norm_backward_bytes(BIG, 4) == 0
    assert qb.layer_norm_backward_bytes(1, (1 << 24) + 1) == 0 and qb.layer_norm_backward_bytes(0, 100) == 0


def test_quantize_blocks():
    good = [OK, 1, 300, 100, 100, 0, OK, OK, OK, OK, None]
    _variants("qsdp_quantize_blocks", good, [
        (0, None, E), (0, ODD, A), (1, 3, E), (2, (1 << 26) + 1, E), (3, 0, E), (3, (1 << 26) + 1, E), (4, 99, E), (6, None, E),
        (7, None, E), (8, None, E), (9, None, E), (6, EIGHT, A), (7, ODD, A), (8, EIGHT, A), (9, ODD, A)])
    assert qb.lib().qsdp_quantize_blocks(OK, 1, 3, 100, 100, 0, None, None, None, None, None) == E


def test_products():
    good = [OK, OK, 4, OK, OK, 1, 100, 1000, OK, 1, OK, 100, 0, OK, 1 << 30, None]
    _variants("qsdp_matmul_blocks", good, [
        (0, None, E), (1, None, E), (2, BIG, E), (3, None, E), (4, None, E), (6, 0, E), (6, (1 << 26) + 1, E), (7, 0, E),
        (7, (1 << 20) + 1, E), (9, 3, E), (10, None, E), (11, 99, E), (0, EIGHT, A), (1, ODD, A), (3, EIGHT, A), (4, ODD, A),
        (8, ODD, A), (10, ODD, A), (13, EIGHT, A)])
    room = qb.linear_blocks_bytes(4, 100, 1000)
    good = [OK, 1, 4, 1000, 1000, OK, OK, 100, OK, 1, OK, 100, OK, room, None]
    _variants("qsdp_linear_blocks", good, [
        (0, None, E), (0, ODD, A), (1, 3, E), (2, BIG, E), (3, 0, E), (4, 999, E), (5, None, E), (5, EIGHT, A), (6, None, E),
        (6, ODD, A), (7, 0, E), (8, ODD, A), (9, 3, E), (10, None, E), (10, ODD, A), (11, 99, E), (12, None, E), (12, EIGHT, A),
        (13, room - 1, E)])
    assert qb.linear_blocks_bytes(4, 0, 10) == 0 and qb.linear_blocks_bytes(BIG, 10, 10) == 0


def _entry(n=1000, at=1 << 20, bits=8, **changed):
    """A tensor whose buffers lie behind each other from `at` on."""
    t = qb.AdamWTensor(x=at, g=at + 32768, m=at + 65536, v=at + 98304, scale=at + 131072 if bits == 8 else None, n=n, lr_scale=1.0,
                       g_dtype=0, state_bits=bits)
    for k, v in changed.items():
        setattr(t, k, v)
    return t


def _build(*entries):
    table = (qb.AdamWTensor * len(entries))(*entries)
    return int(qb.lib().qsdp_adamw_build(table, len(entries))), [t.first for t in table]


def test_adamw_table():
    far = 1 << 22
    assert _build(_entry(), _entry(4097, far, 32), _entry(0, 0), _entry(5, far << 1)) == (1 + 3 + 1, [0, 1, 4, 4])
    assert _build(_entry(2048, x16=far, x16_dtype=1), _entry(2049, far << 1)) == (3, [0, 1])
    for bad in (dict(x=None), dict(g=None), dict(m=None), dict(v=None), dict(scale=None), dict(x=4097), dict(g=4098), dict(m=4100),
                dict(v=4100), dict(scale=4100), dict(x16=4097, x16_dtype=1), dict(x16=8192, x16_dtype=0), dict(x16=8192, x16_dtype=3),
                dict(g_dtype=3), dict(g_dtype=-1), dict(state_bits=16), dict(reserved=1), dict(lr_scale=math.inf),
                dict(weight_decay=math.nan), dict(n=(1 << 40) + 1)):
        assert _build(_entry(**bad))[0] == 0, bad
        assert _build(_entry(0, 0), _entry(100, far), _entry(**bad))[0] == 0, bad
    assert _build(_entry(100, 1 << 20, 32, scale=4096))[0] == 0
    assert _build(_entry(0, 0))[0] == 0 and qb.lib().qsdp_adamw_build(None, 1) == 0


def test_adamw_tables_share_no_memory():
    one = _entry(1000)
    at = one.x
    assert _build(one, _entry(1000))[0] == 0                                   # the same tensor twice
    for name in ("x", "m", "v", "scale", "x16"):
        for where, size in ((at, 4000), (one.g, 4000), (one.m, 1000), (one.v, 1000), (one.scale, 32)):
            inside = where + size - 8
            other = _entry(1000, 1 << 22, x16_dtype=1, **{name: inside})
            assert _build(one, other)[0] == 0 and _build(other, one)[0] == 0, (name, where)
    assert _build(one, _entry(1000, 1 << 22, g=one.g))[0] == 2                  # a gradient may serve two
    assert _build(_entry(1000, g=at))[0] == 0                                   # but not be what is written
    assert _build(_entry(1000, at, m=at + 4000, v=at + 5000, scale=at + 6000))[0] == 1  # side by side


def test_adamw_tensors():
    good = [OK, 3, 5, 1e-3, 0.9, 0.95, 1e-8, 0.1, 0.05, 0, OK, OK, OK, None]
    _variants("qsdp_adamw_tensors", good, [
        (0, None, E), (0, FOUR, A), (1, 0, E), (2, 0, E), (3, math.nan, E), (3, math.inf, E), (4, 1.0, E), (4, -0.1, E),
        (4, math.nan, E), (5, 1.0, E), (6, 0.0, E), (6, 1e-39, E), (6, -1.0, E), (6, math.inf, E), (7, 0.0, E), (7, math.nan, E), (8, -1.0, E),
        (8, math.inf, E), (10, FOUR, A), (11, ODD, A), (12, ODD, A)])


def test_the_binding_refuses_tensors_on_the_cpu():
    x = torch.zeros((4, 128))
    codes = torch.zeros((4, 128), dtype=torch.uint8)
    scale = torch.zeros((1, 4))
    for call in (lambda: qb.qsdp_layer_norm(x, None, None, 1e-5, x), lambda: qb.qsdp_layer_norm_backward(x, None, x, x, x),
                 lambda: qb.qsdp_quantize_blocks(x, False, codes, scale),
                 lambda: qb.qsdp_matmul_blocks(codes, scale, codes, scale, 128, None, x),
                 lambda: qb.qsdp_linear_blocks(x, codes, scale, None, x),
                 lambda: qb.AdamWTensors([x], [x], [x], [x])):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError):
        qb.AdamWTensors([], [], [], [])
    with pytest.raises(qb.QsdpError):
        qb.alloc_moments(x, 16)
