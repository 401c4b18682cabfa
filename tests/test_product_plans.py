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


@pytest.mark.parametrize("size", shapes.NARROW, ids=str)
def test_short_rows_are_packed(size):
    (_, products), = plans([call(False, size, ("f32",) * 3)])
    assert products[0]["f16"] == 1 and products[0]["tile"] > 0 and products[0]["packed"] == (1, 1)


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


def _ways(calls):
    return [p for _, products in plans(calls) for p in products]


def test_large_shapes_take_every_kernel():
    forward = _ways([call(False, *case) for case in shapes.FORWARD])
    gradient = _ways([call(True, size, types) for size in shapes.GRADIENT_SIZES for types in shapes.GRADIENT_TYPES])
    gradient += _ways([call(True, shapes.GRADIENT_SIZES[0], shapes.MIXED)])
    ways = forward + gradient
    assert all(p["tile"] > 0 for p in ways)
    taken = {(p["tile"], p["along"], p["f16"]) for p in ways}
    layouts = [(tile, along) for tile in (128, 256) for along in ((1, 0), (1, 1), (0, 0))] + [(32, (1, 0)), (32, (1, 1))]
    assert taken == {(*layout, f16) for layout in layouts for f16 in (0, 1)}
    # more stages of 64 than are under way at first, in every part of k; shared out and not
    assert all(-(-p["k"] // 64) / p["splits"] > (4 if p["tile"] == 32 else 2) for p in ways)
    assert {(p["tile"], p["splits"] > 1) for p in ways} == {(tile, shared) for tile in (32, 128, 256) for shared in (False, True)}
    assert {p["parts"] for p in ways if p["f16"]} == {(3, 3), (3, 1), (1, 3), (2, 2)}
    assert any(p["tile"] == 256 and p["W"] > 1 for p in ways)
    assert {(p["tile"], p["end"]) for p in ways if p["splits"] == 1} >= {(128, 8), (128, 4), (128, 1), (256, 8), (256, 1), (32, 8)}
    # operands that are packed beside ones that are read as they lie
    assert {p["packed"] for p in ways if not p["f16"]} == {(0, 0), (0, 1), (1, 0), (1, 1)}


def test_added_gradients_take_the_end_that_adds():
    ways = _ways([call(True, size, types, accumulate=True, more=True) for size in shapes.GRADIENT_SIZES for types in shapes.GRADIENT_TYPES])
    assert {(p["tile"], p["f16"]) for p in ways if p["adds"]} >= {(256, 0), (256, 1), (128, 0)}
    assert {p["end"] for p in ways if not p["adds"] and p["splits"] == 1} == {1, 4, 8}
    # parts joined a number to a thread and in vectors
    vectors = {p["W"] * p["m"] * -(-p["n"] // 8) >= 1 << 18 for p in ways if p["splits"] > 1}
    assert vectors == {False, True}


@pytest.mark.parametrize("room", shapes.BATCH_ROOMS)
@pytest.mark.parametrize("types", shapes.BATCH_TYPES, ids=str)
def test_batches_of_workers_share_the_workspace(types, room):
    ways = _ways([call(True, shapes.BATCHES, types, act=4, room=room)])
    assert len(ways) > 2 and max(p["W"] for p in ways) < shapes.BATCHES[0] and all(p["tile"] > 0 and p["f16"] == 1 for p in ways)


@pytest.mark.parametrize("types", [shapes.WHOLE, shapes.FLOAT, shapes.SINGLE], ids=str)
def test_bad_numbers_are_packed_as_floats(types):
    p, = _ways([call(False, shapes.RANGE, types)])
    assert p["tile"] > 0 and p["f16"] == (types != shapes.WHOLE)
