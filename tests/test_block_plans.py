"""What the plans of an image model's block refuse before anything reaches a GPU."""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2308_09187_amd import qgx  # noqa: E402


def refused(f):
    with pytest.raises(qgx.QgxError) as e:
        f()
    assert e.value.status == qgx.ERR_ARG and str(e.value)


def test_rotary_plans():
    r = qgx.Rotary.by_base((3, 2), 100.0, neighbours=True)
    assert r.pairs == [3, 2] and list(r.frequencies) == [1.0, 100.0 ** (-1 / 3), 100.0 ** (-2 / 3), 1.0, 0.1] and r.neighbours
    qgx.Rotary((256,), [0.5] * 256)
    for pairs, f in (((), []), ((0,), []), ((2, -1), [1.0]), ((1, 1, 1, 1, 1), [1.0] * 5), ((257,), [1.0] * 257), ((3,), [1.0] * 2), ((1,), [math.nan]), ((1,), [math.inf])):
        refused(lambda: qgx.Rotary(pairs, f))


def test_checkpoints_of_other_memory():
    codes, powers = torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.uint8)
    refused(lambda: qgx.Checkpoint(codes, powers, 40))     # not on a GPU


def test_no_context():
    lib = qgx.load()
    shape = qgx._GroupShape(0, 0, 0.0, 1, 1, 1, 1, 1)
    from ctypes import addressof
    assert lib.qgx_checkpoint(None, 0, 1, 1, 1, None, 0, 0, 0, 0, None, None) == qgx.ERR_ARG
    assert lib.qgx_restore(None, None, 0, None, 0, None) == qgx.ERR_ARG
    assert lib.qgx_weight_gradient_scratch(None, 0, 1, 1, 1, 1, 1, None) == qgx.ERR_ARG
    assert lib.qgx_weight_gradient(None, None, 0, 1, 1, 1, None, 0, 0, None, 0, None, 0, None, 0, None) == qgx.ERR_ARG
    assert lib.qgx_group_norm_scratch(None, addressof(shape), 0, None) == qgx.ERR_ARG
    assert lib.qgx_group_norm(None, addressof(shape), None, None, None, 0.0, None, None, None, None, 0, 0, None, 0, None) == qgx.ERR_ARG
    assert lib.qgx_group_norm_backward(None, addressof(shape), None, None, None, None, None, None, None, None, None, None, 0, None, 0, None) == qgx.ERR_ARG
    assert lib.qgx_rotate(None, None, None, 0, 0, 0, None, None, 0, None) == qgx.ERR_ARG
