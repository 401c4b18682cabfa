"""The GPU tests of large products take the kernels that they are for: the host code that decides it is asked for their shapes."""
import pytest

import product_shapes as shapes
from product_plans import plans


def call(gradient, size, types, act=0, accumulate=False, more=False, room=0):
    """As test_gpu_linear.Layer places a matrix."""
    W, T, inputs, outputs, at = size
    transposed, gap, cols = at.get("transposed", False), at.get("gap", 0), inputs if at.get("transposed") else outputs
    row_stride = cols + at.get("apart", 0)
    end = gap + (outputs if transposed else inputs) * row_stride
    layer = (gap, inputs, outputs, end + (gap & 1) if at.get("bias", True) else -1, transposed, row_stride)
    return dict(gradient=gradient, W=W, T=T, layer=layer, stride=-(-(end + outputs + 3) // 64) * 64, act=act, types=types, accumulate=accumulate,
                more=more, room=room)


@pytest.mark.parametrize("types", shapes.RANGE_TYPES, ids=str)
def test_rows_far_apart_are_packed(types):
    (_, products), = plans([call(False, shapes.RANGE, types)])
    floats = types.count("f32") - (types[2] == "f32")
    assert len(products) == 1 and products[0]["f16"] == 1 and products[0]["tile"] > 0
    assert products[0]["parts"] == tuple((3 if types[2] == "f32" else 2) if t == "f32" else 1 for t in types[:2]) and floats >= 1


@pytest.mark.parametrize("act", [0, 1])
def test_padding_in_a_gradient_is_packed(act):
    (_, products), = plans([call(True, shapes.RANGE, ("f32",) * 5, act)])
    assert len(products) == 2 and all(p["f16"] == 1 and p["parts"] == (3, 3) and p["tile"] > 0 for p in products)


def test_lowest_numbers_are_rounded_to_bf16():
    (_, of_gradient), (_, of_forward) = plans([call(True, shapes.RANGE, ("bf16", "f32", "bf16", "bf16", "bf16")), call(False, shapes.RANGE, ("bf16", "f32", "bf16"))])
    for p, which in ((of_gradient[1], 0), (of_forward[0], 1)):
        assert p["tile"] > 0 and p["f16"] == 0 and p["packed"][which] == 1 and p["parts"] == (1, 1)


def _without_parts(W, T, inputs, outputs):
    """What noloco.h says that a plan's workspace takes but for sums in parts: dz as float and six bytes for each number that may be packed, the
    sides of an operand in whole vectors of eight."""
    padded, i, o = -(-T // 8) * 8, -(-inputs // 8) * 8, -(-outputs // 8) * 8
    return W * (4 * T * o + 6 * (padded * o + padded * i + i * o) + 20000)


@pytest.mark.parametrize("size", [(8, 256, 96, 192, {}), (4, 100, 300, 64, {}), (1, 20, 320, 310, {}), (2, 1, 64, 300, dict(transposed=True))], ids=str)
def test_no_room_for_parts_that_no_call_makes(size):
    """Sums of 320 products and less are never shared out."""
    for types in (("f32",) * 5, ("bf16",) * 5):
        for room, products in plans([call(gradient, size, types) for gradient in (False, True)]):
            assert all(p["splits"] == 1 for p in products) and room <= _without_parts(*size[:4])


def test_room_for_parts_that_calls_make():
    size = (2, 24, 16384, 4096, {})
    (room, products), = plans([call(False, size, ("bf16",) * 3)])
    assert products[0]["splits"] >= 8 and products[0]["splits"] * 2 * 24 * 4096 * 4 <= room <= _without_parts(*size[:4]) + (64 << 20)
    # parts of one token: 32 of the longer side at most
    size = (2, 1, 16384, 4096, {})
    (room, products), = plans([call(False, size, ("bf16",) * 3)])
    assert products[0]["splits"] >= 8 and room <= _without_parts(*size[:4]) + 32 * 2 * 16384 * 4
