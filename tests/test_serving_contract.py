"""Host-side promises of the serving calls' Python side that need no GPU."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2503_01483_b200 import build, kurtail


def ints(*a):
    return torch.zeros(*a, dtype=torch.int32)


def a_cache(page=16):
    return kurtail.KvCache(*[torch.zeros(3, 2, page, 64, dtype=torch.uint8)] * 2, *[torch.zeros(3, 2, page, 2)] * 2, 8)


def test_a_table_of_a_wider_ones_columns_bounds_the_lengths_by_its_own():
    # the library is told the pitch of its rows and would follow page ids behind them, past the last row's end
    wide = ints(2, 10)
    for table, page, want in ((wide[:, 4:], 16, 96), (wide[:, :5], 16, 80), (wide[:, 4:], 64, 100), (wide, 16, 100),
                              (wide[:1, 4:], 16, 100)):
        b = kurtail.KvBatch(ints(table.shape[0] + 1), ints(table.shape[0]), table, 1, 100)
        b._own_columns(a_cache(page))
        assert b._c.max_length == b.max_length == want
        assert b._c.max_length <= table.shape[1] * page or b._c.table_ld == table.shape[1]
        b._fits(a_cache(page), -1)


def test_such_a_table_is_for_one_page_size():
    b = kurtail.KvBatch(ints(3), ints(2), ints(2, 10)[:, 4:], 1, 100)
    for cache in (a_cache(16), a_cache(64)):
        with pytest.raises(ValueError):
            b._fits(cache, -1)
    b._own_columns(a_cache(16))
    b._fits(a_cache(16), -1)
    with pytest.raises(ValueError):
        b._fits(a_cache(32), -1)
    with pytest.raises(ValueError):
        b._fits(a_cache(16), 0)
    whole = kurtail.KvBatch(ints(3), ints(2), ints(2, 10), 1, 100)
    whole._own_columns(a_cache(16))
    whole._fits(a_cache(64), -1)


def test_bounds_that_do_not_fit_32_bits_are_refused():
    # (a ctypes field takes such a number modulo 2^32)
    make = lambda rows=1, length=10, table=ints(2, 5): kurtail.KvBatch(ints(3), ints(2), table, rows, length)  # noqa: E731
    assert make(2**30, 2**30)._c.max_length == 2**30
    for bad in (dict(rows=2**32 + 1), dict(length=2**32 + 10), dict(rows=2**31), dict(length=-(2**31) - 5)):
        with pytest.raises(ValueError):
            make(**bad)


def test_strides_of_single_columns_and_rows_say_nothing():
    build.build()
    kurtail.lib()
    from paper_2503_01483_b200 import _serving
    call = lambda x: _serving.rmsnorm_quant(0, -1, x, None, None, None, 1e-6, None, 1.0, None, None, x)  # noqa: E731
    x = torch.zeros(8, 8)
    for t in (x[:1].t(), x[:, 2:3], torch.zeros(8, 1).t()):                  # (no context: status 1, behind all checks of tensors)
        assert call(t) == 1
    for t in (x[:2].t(), x[:, ::2], x[:, :1].t()):
        with pytest.raises(ValueError):
            call(t)


WITHOUT = """
import sys, torch
{before}
from paper_2503_01483_b200 import kurtail
assert kurtail.lib().kt_status_string(0) and kurtail.default_config().eps > 0     # the library's other calls work
ctx = object.__new__(kurtail.Context)
ctx._h, ctx._at, ctx._index, ctx.stream = None, 0, -1, None
x = torch.zeros(1, 64)
try:
    ctx.rmsnorm_quant(x, bits=None, values=x)
except ImportError as e:
    assert {text!r} in str(e), e
else:
    raise SystemExit("no error")
"""


@pytest.mark.parametrize("before,text", [
    ("sys.modules['paper_2503_01483_b200._serving'] = None", "_serving.so"),
    ("import paper_2503_01483_b200._serving as m; del m.built_for", "another version of this library"),
    ("import paper_2503_01483_b200.build as b; b.built_for = lambda: 'Python 2.7, torch 0.1'", "this is Python 2.7, torch 0.1")])
def test_the_library_works_without_the_serving_module(before, text):
    build.build()
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", WITHOUT.format(before=before, text=text)], cwd=root, capture_output=True,
                       text=True, timeout=300)
    assert r.returncode == 0, r.stderr


def test_a_serving_module_of_another_torch_is_built_anew(monkeypatch):
    build.build()
    assert not build.needs_build()
    monkeypatch.setattr(build, "built_for", lambda: "Python 2.7, torch 0.1")
    assert build.needs_build()


def test_the_serving_module_needs_the_library_first():
    # its entry points are null until lib() binds them
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    code = """
import torch
from paper_2503_01483_b200 import _serving
x = torch.zeros(1, 64)
try:
    _serving.rmsnorm_quant(0, -1, x, None, None, None, 1e-6, None, 1.0, None, None, x)
except ValueError as e:
    assert "not loaded" in str(e), e
else:
    raise SystemExit("no error")
"""
    build.build()
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
