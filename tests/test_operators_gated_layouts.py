"""Gated units on layouts that the documentation allows: a shared weight or x of odd rows, single rows of any row stride, padded rows, parameters."""
import ctypes as C

import pytest

from test_operators_gated import _case, _run, _verify


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows", [1, 4, 100, 300])
@pytest.mark.parametrize("width", [33, 1001])
def test_a_shared_weight_and_a_shared_x_of_odd_rows(width, rows, dtype):
    c = _case(3, rows, width, 41, dtype, shared=True, seed=rows)
    _verify(c, "silu")
    _verify({**c, "x": c["x"][1:2].expand(3, -1, -1), "dh": c["dh"][2:].expand(3, -1, -1)}, "gelu")
    _verify({**_case(3, rows, width, 41, dtype, seed=rows + 1), "x": c["x"][:1].expand(3, -1, -1)}, "sigmoid")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("width", [64, 77])
def test_a_single_row_may_carry_any_row_stride(width, dtype):
    import torch
    c = _case(3, 1, width, 24, dtype, seed=width)
    for stride in (0, 3, width + 1, 1 << 40):
        moved = {k: c[k].as_strided(c[k].shape, (c[k].stride(0), stride, 1)) for k in ("x", "dh")}
        got, want = _verify({**c, **moved}, "silu"), _verify(c, "silu")
        assert all(torch.equal(got[k], want[k]) for k in want)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [3, 100, 400])
def test_rows_padded_to_eight_elements_need_no_workspace(rows):
    """bfloat16 rows of an odd width in memory whose rows are multiples of 16 bytes; what lies between them is never used."""
    import torch
    import paper_1711_09846_b200 as pbt
    c = _case(2, rows, 77, 40, "bfloat16", seed=rows)

    def padded(t):
        whole = torch.full((*t.shape[:2], 80), float("nan"), dtype=t.dtype, device="cuda")
        whole[..., :77] = t
        return whole[..., :77]
    wide = {**c, "x": padded(c["x"]), "weight": padded(c["weight"])}
    got, want = _verify(wide, "gelu"), _verify(c, "gelu")
    assert all(torch.equal(got[k], want[k]) for k in want)
    unit, n = pbt.GatedUnit(wide["weight"]), C.c_size_t(1)
    d = unit._call(unit._describe(wide["x"]), wide["x"], None)
    assert pbt.load_library().pbt_gated_query_workspace(C.byref(d), 0, C.byref(n)) == 0 and n.value == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_parameters_and_inference_mode(dtype):
    """Parameters are taken as plain numbers; the results need no gradient."""
    import torch
    import paper_1711_09846_b200 as pbt
    c = _case(2, 40, 72, 40, dtype, seed=8)
    want, _ = _run(c, "silu")
    learned = {**c, "weight": torch.nn.Parameter(c["weight"]), "x": c["x"].clone().requires_grad_()}
    got, _ = _run(learned, "silu")
    with torch.inference_mode():
        other, _ = _run(learned, "silu", layer=pbt.GatedUnit(learned["weight"], "silu"))
        fresh, _ = _run({**c, "x": c["x"].clone(), "weight": c["weight"].clone()}, "silu")
    for k in want:
        assert not got[k].requires_grad
        assert all(torch.equal(want[k], r[k]) for r in (got, other, fresh)), k
