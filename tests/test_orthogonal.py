"""CPU-side checks of the orthogonalisation's entry points: workspace sizes and refusals, before anything is launched (the
addresses are made up: argument checks touch no memory)."""
import ctypes

import numpy as np
import pytest

from paper_2305_12201_amd import binding as B

TABLE = [(0, 10, 20, 20), (200, 30, 7, 7)]


def _args(matrices=TABLE, n=1000, steps=5, coefficients=None, eps=1e-7, type=B.FLOAT32, ws=0x10000, ws_bytes=1 << 40):
    m = np.asarray(matrices, dtype=np.int64).reshape(-1, 4)
    c = None if coefficients is None else np.ascontiguousarray(np.asarray(coefficients, dtype=np.float64))
    ptr = lambda a: None if a is None else a.ctypes.data_as(ctypes.c_void_p)  # noqa: E731
    return m, c, ptr, n, steps, eps, type, ws, ws_bytes


def _orthogonalize(x=0x1000, out=0x2000, n_mat=None, no_table=False, **kw):
    m, c, ptr, n, steps, eps, type, ws, ws_bytes = _args(**kw)
    return B.lib().gravac_orthogonalize(x, out, type, n, None if no_table else ptr(m), m.shape[0] if n_mat is None else n_mat, steps,
                                        ptr(c), eps, ws, ws_bytes, None)


def _update(grad=0x1000, momentum=0x2000, params=0x3000, flags=0, **kw):
    m, c, ptr, n, steps, eps, type, ws, ws_bytes = _args(**kw)
    f = ctypes.c_float
    return B.lib().gravac_orthogonal_update(grad, momentum, params, type, n, ptr(m), m.shape[0], f(0.9), f(1.0), f(-0.1), None,
                                            steps, ptr(c), eps, ws, ws_bytes, flags, None)


BAD_TABLES = [
    [(-1, 10, 20, 20)], [(0, 0, 20, 20)], [(0, 10, 0, 20)], [(0, 10, 20, 19)], [(801, 10, 20, 20)], [(0, 10, 20, 110)],
    [(0, (1 << 20) + 1, 1, 1)], [(0, 1, (1 << 20) + 1, (1 << 20) + 1)],
    [(0, 10, 20, 20), (199, 5, 5, 5)], [(100, 5, 5, 5), (0, 10, 20, 20)], [(0, 10, 20, 20), (0, 10, 20, 20)],
    [(0, 10, 8, 20), (7, 10, 8, 20)], [(0, 10, 12, 20), (12, 10, 9, 20)], [(0, 10, 8, 20), (8, 10, 8, 21)]]


@pytest.mark.parametrize("table", BAD_TABLES)
def test_refuses_tables(table):
    assert _orthogonalize(matrices=table) == B.ERR_INVALID_ARG
    assert _update(matrices=table) == B.ERR_INVALID_ARG


def test_refuses_large_squares():
    table = [(0, 32_769, 32_769, 32_769)]
    assert _orthogonalize(matrices=table, n=1 << 40) == B.ERR_INVALID_ARG
    with pytest.raises(B.GravacError):
        B.gravac_orthogonalize_workspace_bytes(table)


@pytest.mark.parametrize("bad", [{"n": 0}, {"n": 409}, {"n": (1 << 40) + 1}, {"steps": 0}, {"steps": B.MAX_STEPS + 1}, {"eps": -1.0},
                                 {"eps": float("nan")}, {"eps": float("inf")}, {"type": 3}, {"type": -1}])
def test_refuses(bad):
    assert _orthogonalize(**bad) == B.ERR_INVALID_ARG
    assert _update(**bad) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("bad", [{"x": 0}, {"out": 0}, {"x": 0x1002}, {"out": 0x2001, "type": B.BFLOAT16}, {"n_mat": 0},
                                 {"n_mat": B.MAX_MATRICES + 1}, {"n_mat": -1}, {"no_table": True}])
def test_orthogonalize_refuses(bad):
    assert _orthogonalize(**bad) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("bad", [{"grad": 0}, {"momentum": 0}, {"params": 0}, {"grad": 0x1002}, {"momentum": 0x2002}, {"params": 0x3002},
                                 {"params": 0x3001, "type": B.FLOAT16}, {"flags": 1}, {"flags": 16}])
def test_update_refuses(bad):
    assert _update(**bad) == B.ERR_INVALID_ARG


def test_refuses_vectors_that_overlap():
    # 1000 elements: 4000 bytes, or 2000 of bfloat16
    assert _orthogonalize(x=0x1000, out=0x1000 + 3996) == B.ERR_INVALID_ARG
    assert _orthogonalize(x=0x1000 + 1998, out=0x1000, type=B.BFLOAT16) == B.ERR_INVALID_ARG
    for bad in ({"grad": 0x2000}, {"momentum": 0x3000}, {"params": 0x1000}, {"grad": 0x2000 - 3996}, {"params": 0x2000 - 1998, "type": B.FLOAT16},
                {"params": 0x1000 + 3996, "type": B.BFLOAT16}):
        assert _update(**bad) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("triple", [(float("nan"), 0, 0), (1, float("inf"), 0), (4.0, 0, 0), (1.0, 3.0, 0), (0, 0, 3.95), (1.0, -16.0, 0),
                                    (0, 0, 1e9)])
def test_refuses_coefficients_that_leave_the_range(triple):
    assert _orthogonalize(steps=1, coefficients=[triple]) == B.ERR_INVALID_ARG
    assert _update(steps=2, coefficients=[(1.0, 0, 0), triple]) == B.ERR_INVALID_ARG


def test_refuses_coefficients_that_leave_the_range_in_a_later_step():
    # 1.9 s is 1.9 at most after one step and 3.61 after two, which is allowed; a third one is not
    ws = {"ws": 0}    # (allowed ones go on to the workspace's check)
    assert _orthogonalize(steps=2, coefficients=[(1.9, 0, 0)] * 2, **ws) == B.ERR_WORKSPACE
    assert _orthogonalize(steps=3, coefficients=[(1.9, 0, 0)] * 3, **ws) == B.ERR_INVALID_ARG
    assert _orthogonalize(steps=32, coefficients=[(3.4445, -4.7750, 2.0315)] * 32, **ws) == B.ERR_WORKSPACE
    assert _orthogonalize(steps=32, coefficients=[(1.5, -0.5, 0.0)] * 32, **ws) == B.ERR_WORKSPACE
    assert _orthogonalize(steps=32, coefficients=[(15 / 8, -10 / 8, 3 / 8)] * 32, **ws) == B.ERR_WORKSPACE


def test_refuses_workspaces():
    need = B.gravac_orthogonalize_workspace_bytes(TABLE)
    for f in (_orthogonalize, _update):
        assert f(ws=0) == B.ERR_WORKSPACE
        assert f(ws=0x10080) == B.ERR_WORKSPACE
        assert f(ws_bytes=need - 1) == B.ERR_WORKSPACE


def test_columns_of_one_matrix_lie_apart():
    # three matrices side by side in the columns of a larger one, in any order
    table = [(8, 10, 4, 20), (0, 10, 8, 20), (12, 10, 8, 20)]
    assert _orthogonalize(matrices=table, ws=0) == B.ERR_WORKSPACE
    assert _orthogonalize(matrices=[(300, 5, 5, 5), (0, 10, 20, 20)], ws=0) == B.ERR_WORKSPACE


def test_workspace_bytes():
    size = B.gravac_orthogonalize_workspace_bytes
    import torch
    one, both = size([(0, 1024, 4096)]), size([(0, 1024, 4096), (1 << 22, 1024, 4096)])
    assert one < both <= 2 * one
    assert 12 * 1024 * 4096 + 8 * 1024 * 1024 <= one <= 1.01 * (12 * 1024 * 4096 + 8 * 1024 * 1024)
    assert size([(0, 1024, 4096)], torch.bfloat16) < one
    assert size([(0, 1, 1)]) == size([(5, 1, 1)]) <= 512 * 1024
    for bad in ([], [(0, 0, 1)], [(0, 1, 1)] * (B.MAX_MATRICES + 1)):
        with pytest.raises(B.GravacError) as e:
            size(bad)
        assert e.value.code == B.ERR_INVALID_ARG
    with pytest.raises(ValueError):
        size([(0, 1)])


def test_refuses_workspaces_in_the_vectors():
    need = B.gravac_orthogonalize_workspace_bytes(TABLE)
    assert need > 0x1000
    for bad in ({"x": 0x10000}, {"out": 0x10000}, {"x": 0x10000 - 3996}, {"out": 0x10000 + (need - 4) // 4 * 4}, {"x": 0x10800, "out": 0x10800}):
        assert _orthogonalize(**bad) == B.ERR_INVALID_ARG
    for bad in ({"grad": 0x10000}, {"momentum": 0x10000 - 3996}, {"params": 0x10000 + (need - 4) // 4 * 4}, {"params": 0x10000 - 1998, "type": B.BFLOAT16}):
        assert _update(**bad) == B.ERR_INVALID_ARG


def test_tables_are_refused_exactly_where_elements_are_shared():
    """Small tables in any order, of any strides, against sets of elements."""
    rng = np.random.default_rng(5)
    apart = 0
    for _ in range(4000):
        n, table, seen, ok = 70, [], set(), True
        for _ in range(int(rng.integers(2, 4))):
            rows, cols = int(rng.integers(1, 6)), int(rng.integers(1, 5))
            table.append((int(rng.integers(0, 30)), rows, cols, cols + int(rng.integers(0, 12))))
        for off, rows, cols, stride in table:
            mine = {off + i * stride + j for i in range(rows) for j in range(cols)}
            ok = ok and max(mine) < n and not (mine & seen)
            seen |= mine
        # (an allowed table goes on to the workspace's check)
        assert _orthogonalize(matrices=table, n=n, ws=0) == (B.ERR_WORKSPACE if ok else B.ERR_INVALID_ARG), table
        apart += ok
    assert 200 < apart < 3800


def test_tables_of_different_strides_lie_apart():
    # one row between two others; two row lengths of the same buffer; long ones
    for table in ([(0, 10, 8, 20), (8, 1, 12, 12)], [(0, 10, 8, 20), (28, 4, 8, 40)], [(0, 1 << 20, 1, 1 << 19), (1, 1 << 18, 7, 1 << 20)]):
        assert _orthogonalize(matrices=table, n=1 << 40, ws=0) == B.ERR_WORKSPACE
    assert _orthogonalize(matrices=[(0, 10, 8, 20), (8, 2, 12, 15)], ws=0) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("c", [0.0, 1e-17, -1e-17, 1e-12, -1e-9, 1e-300, 5e-324])
def test_refuses_coefficients_by_their_largest_value_inside_the_range(c):
    """11 s - 11 s^3 is 4.23 at s = 3^-1/2 and 0 at s = 1; 10 s - 10 s^3 is 3.85.  A fifth power that adds next to nothing changes
    neither."""
    assert _orthogonalize(steps=1, coefficients=[(11.0, -11.0, c)], ws=0) == B.ERR_INVALID_ARG
    assert _orthogonalize(steps=1, coefficients=[(-11.0, 11.0, c)], ws=0) == B.ERR_INVALID_ARG
    assert _orthogonalize(steps=1, coefficients=[(10.0, -10.0, c)], ws=0) == B.ERR_WORKSPACE


def test_coefficients_against_values_on_a_grid():
    """Every triple's largest values on a fine grid of [0, 1] decide, where they are not within 1e-3 of the limits."""
    rng = np.random.default_rng(6)
    s = np.linspace(0.0, 1.0, 20_001)
    taken = 0
    for _ in range(1500):
        a, b, c = rng.normal(size=3) * 10.0 ** rng.uniform(-1, 1.3, 3)
        most, poly = np.abs(a * s + b * s ** 3 + c * s ** 5).max(), np.abs(b * s ** 2 + c * s ** 4).max()
        if abs(most - 3.9) < 4e-3 or abs(poly - 15.0) < 15e-3:
            continue
        ok = most < 3.9 and poly < 15.0
        taken += ok
        assert _orthogonalize(steps=1, coefficients=[(a, b, c)], ws=0) == (B.ERR_WORKSPACE if ok else B.ERR_INVALID_ARG), (a, b, c)
    assert 100 < taken < 1400


def test_an_orthogonalizer_keeps_its_tables():
    table, each = np.array(TABLE, dtype=np.int64), np.array([(1.0, 0.0, 0.0), (1.5, -0.5, 0.0)])
    o = B.Orthogonalizer(1000, table, steps=2, coefficients=each, device="cpu")
    before = o.matrices.tolist(), o.coefficients.tolist(), o.workspace.numel()
    table[:, 1] *= 2
    each[:] = 7.0
    assert (o.matrices.tolist(), o.coefficients.tolist()) == before[:2]
    assert B.gravac_orthogonalize_workspace_bytes(o.matrices) == before[2]
