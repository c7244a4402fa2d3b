"""What the C entry points of the operators on logits and on packed weights refuse, before any launch (no GPU)."""
import ctypes
import math

from paper_2302_02390_amd import binding as qb

OK, ODD = ctypes.c_void_p(4096), ctypes.c_void_p(4097)
BIG = 1 << 31
E, A = qb.QSDP_EINVAL, qb.QSDP_EALIGN


def _variants(name, good, changes):
    """Every change of one argument of a call that would be launched is refused with its status."""
    fn = getattr(qb.lib(), name)
    for at, value, status in changes:
        args = list(good)
        args[at] = value
        assert fn(*args) == status, (name, at, value)


def test_token_logprobs():
    good = [OK, 1, 4, 100, 100, OK, 1.0, 5, OK, OK, OK, OK, OK, None, 0, None]
    _variants("qsdp_token_logprobs", good, [
        (0, None, E), (0, ODD, A), (1, 3, E), (1, -1, E), (2, BIG, E), (3, 0, E), (3, BIG, E), (4, 99, E), (5, None, E),
        (5, ctypes.c_void_p(4100), A), (6, 0.0, E), (6, -1.0, E), (6, math.inf, E), (6, math.nan, E), (6, 1e-45, E),
        (7, -1, E), (7, 101, E), (7, 129, E), (8, ODD, A), (9, ODD, A), (10, ODD, A), (11, None, E), (12, None, E),
        (11, ODD, A), (12, ODD, A), (13, ctypes.c_void_p(4104), A)])
    nothing = [OK, 1, 4, 100, 100, OK, 1.0, 0, None, None, None, None, None, None, 0, None]
    assert qb.lib().qsdp_token_logprobs(*nothing) == E
    none = [None, 1, 0, 100, 100, None, 1.0, 5, None, None, None, None, None, None, 0, None]
    assert qb.lib().qsdp_token_logprobs(*none) == qb.QSDP_OK


def test_token_logprobs_backward():
    good = [OK, 0, 4, 100, 104, OK, 1.0, OK, OK, OK, OK, OK, 100, None]
    _variants("qsdp_token_logprobs_backward", good, [
        (0, None, E), (0, ctypes.c_void_p(4098), A), (1, 3, E), (2, BIG, E), (3, 0, E), (4, 99, E), (5, None, E), (6, 0.0, E),
        (7, None, E), (8, None, E), (11, None, E), (12, 99, E), (7, ODD, A), (9, ODD, A), (10, ODD, A), (11, ODD, A)])
    assert qb.lib().qsdp_token_logprobs_backward(OK, 0, 4, 100, 100, OK, 1.0, OK, OK, None, None, OK, 100, None) == E


def test_distill_loss():
    good = [OK, 2, 4, 100, 100, OK, OK, 10, OK, 1.0, 0.5, OK, OK, OK, OK, 100, None]
    _variants("qsdp_distill_loss", good, [
        (0, None, E), (0, ODD, A), (1, 9, E), (2, BIG, E), (3, 0, E), (4, 99, E), (5, None, E), (6, None, E), (7, -1, E),
        (7, 0, E), (7, 129, E), (8, None, E), (9, 0.0, E), (9, math.nan, E), (10, -0.1, E), (10, 1.1, E), (10, math.nan, E),
        (12, None, E), (15, 99, E), (5, ODD, A), (6, ODD, A), (8, ctypes.c_void_p(4100), A), (11, ODD, A), (12, ODD, A),
        (13, ODD, A), (14, ODD, A)])
    assert qb.lib().qsdp_distill_loss(None, 2, 0, 9, 9, None, None, 200, None, 1.0, 0.5, None, None, None, None, 0, None) == E


def test_distill_loss_backward():
    good = [OK, 2, 4, 100, 100, OK, OK, 10, OK, 1.0, 0.5, OK, OK, OK, 100, None]
    _variants("qsdp_distill_loss_backward", good, [
        (0, None, E), (1, 9, E), (3, 0, E), (4, 99, E), (5, None, E), (7, 0, E), (8, None, E), (9, -1.0, E), (10, 2.0, E),
        (11, None, E), (12, None, E), (13, None, E), (14, 99, E), (11, ODD, A), (12, ODD, A), (13, ODD, A)])


def test_products():
    good = [OK, 1, 4, 1000, 1000, 1024, OK, OK, OK, None]
    _variants("qsdp_quantize_tokens", good, [
        (0, None, E), (0, ODD, A), (1, 3, E), (2, BIG, E), (3, 0, E), (3, (1 << 20) + 1, E), (4, 999, E), (5, 0, E), (5, 31, E),
        (5, 8224, E), (5, 96, E), (6, None, E), (6, ctypes.c_void_p(4104), A), (7, None, E), (8, None, E), (7, ODD, A)])
    good = [OK, OK, OK, 4, OK, OK, 100, 1000, 1024, OK, 1, OK, 100, None]
    _variants("qsdp_matmul_codes", good, [
        (0, None, E), (1, None, E), (2, None, E), (3, BIG, E), (4, None, E), (5, None, E), (6, 0, E), (7, 0, E), (8, 160, E),
        (10, 3, E), (11, None, E), (12, 99, E), (0, ctypes.c_void_p(4104), A), (4, ctypes.c_void_p(4104), A),
        (5, ctypes.c_void_p(4100), A), (9, ODD, A), (11, ODD, A)])
    room = qb.tokens_bytes(4, 1000, 1024)
    good = [OK, 1, 4, 1000, 1000, OK, OK, 100, 1024, OK, 1, OK, 100, OK, room, None]
    _variants("qsdp_linear_codes", good, [
        (0, None, E), (1, 3, E), (2, BIG, E), (3, 0, E), (4, 999, E), (5, None, E), (6, None, E), (7, 0, E), (8, 96, E),
        (10, 7, E), (11, None, E), (12, 99, E), (13, None, E), (14, room - 1, E), (0, ODD, A), (5, ctypes.c_void_p(4104), A),
        (9, ODD, A), (11, ODD, A), (13, ctypes.c_void_p(4104), A)])


def test_sizes():
    assert qb.tokens_bytes(3, 1000, 1024) == 3 * (1024 + 4 + 4)
    assert qb.tokens_bytes(3, 2048, 1024) == 3 * (2048 + 4 + 8)
    assert qb.tokens_bytes(3, 1, 32) == 3 * (128 + 8)
    assert qb.tokens_bytes(3, 1000, 100) == 0 and qb.tokens_bytes(3, 0, 32) == 0 and qb.tokens_bytes(3, 1000, 96) == 0
    assert qb.token_logprobs_bytes(0, 100, 0) == 0 and qb.token_logprobs_bytes(1, 0, 0) == 0
