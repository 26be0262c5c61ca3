"""GPU parity of the append where rows are many: from 2048 bf16 rows on a workgroup takes four tokens.  Both pairings and V
layouts, with and without a norm, last groups of one to four tokens, rows without a slot in them, in place."""

import pytest

from test_gpu_norm_rope import F, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [2047, 2048, 2049, 2050, 2051])
@pytest.mark.parametrize("vt", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("eps", [0.0, 1e-6])
def test_rows(rows, vt, interleaved, eps):
    """Rows without a slot: whole groups, single rows, the last ones."""
    hole = (0, 5, 1024, 1025, 1026, 1027, 2044, rows - 1)
    run(rows, hq=3, hkv=1, dim=64, vt=vt, interleaved=interleaved, eps=eps, hole=hole, pos0=777, seed=rows)


@pytest.mark.parametrize("hq,hkv,dim", [(1, 1, 16), (6, 3, 32), (10, 2, 128), (40, 8, 128), (2, 1, 256), (4, 4, 256)])
@pytest.mark.parametrize("vt", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
def test_forms(hq, hkv, dim, vt, interleaved):
    """Heads that leave a workgroup's items whole or not, packed rows and rows of their own, a layer among others."""
    run(2049, hq=hq, hkv=hkv, dim=dim, vt=vt, interleaved=interleaved, hole=(3, 2048), seed=dim, layers=2, layer=1)
    run(2050, hq=hq, hkv=hkv, dim=dim, vt=vt, interleaved=interleaved, packed=False, weights=False, seed=dim + 1)


@pytest.mark.parametrize("vt", [False, True])
@pytest.mark.parametrize("rows", [2048, 2051])
def test_in_place(rows, vt):
    run(rows, hq=5, hkv=1, dim=128, vt=vt, packed=False, in_place=True, hole=(7, rows - 2), seed=rows)
    run(rows, hq=4, hkv=2, dim=64, vt=vt, packed=False, in_place=True, interleaved=True, eps=0.0, seed=rows)


def test_magnitudes():
    """Squares past fp32's largest number and below its smallest, in groups of four."""
    run(2049, hq=4, hkv=2, dim=64, size=1e25, seed=4)
    run(2049, hq=4, hkv=2, dim=64, size=1e-25, eps=1e-30, seed=4)


def test_fp32_rows_stay_one_a_workgroup():
    run(2051, hq=2, hkv=1, dim=64, dtype=F, vt=True, interleaved=True, hole=(2050,), seed=1)
    run(2051, hq=2, hkv=1, dim=128, dtype=F, pos0=100000, seed=2)
