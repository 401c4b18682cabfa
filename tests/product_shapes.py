"""Sizes of matrices whose products have to go a certain way, for the tests on the GPU and for the one that asks the host code which way they
go: (W, T, inputs, outputs, more of test_gpu_linear.Layer)."""

# Rows of very different sizes: operands that are packed to binary16, or to bf16 parts.
RANGE = (2, 1500, 712, 1544, dict(bias=False))
# The same with rows that several of a wave's lanes take: 4, 8 and 16.
NARROW = [(2, 3000, 20, 5000, dict(bias=False)), (2, 2040, 64, 4090, dict(bias=False)), (2, 1000, 100, 3000, dict(bias=False))]
RANGE_TYPES = [("f32", "f32", "f32"), ("bf16", "f32", "f32"), ("f32", "bf16", "f32"), ("f32", "f32", "bf16")]

# Every kernel of large products: tiles of 256, 128 and 32 x 256, operands along k or across it, bf16 or binary16; odd edges of tiles, stages and
# vectors, k shared out or not, ends of eight, four and single numbers.
WHOLE, FLOAT, SINGLE = ("bf16",) * 3, ("f32",) * 3, ("f32", "f32", "bf16")
ALONE = dict(bias=False)
TURNED = dict(bias=False, transposed=True)
FORWARD = [((1, 4090, 200, 4088, at), types) for at in (ALONE, TURNED) for types in (WHOLE, FLOAT, SINGLE, ("bf16", "f32", "f32"))]
FORWARD += [((2, 1500, 712, 1544, at), types) for at in (ALONE, TURNED) for types in (WHOLE, FLOAT, SINGLE, ("f32", "bf16", "f32"))]
FORWARD += [((1, 20, 6001, 6008, ALONE), types) for types in (WHOLE, ("bf16", "f32", "bf16"), ("f32", "bf16", "f32"))]
FORWARD += [((1, 20, 9001, 9003, TURNED), types) for types in (WHOLE, ("f32", "bf16", "f32"))]
FORWARD += [((8, 20, 768, 8200, ALONE), WHOLE)]

GRADIENT_SIZES = [(1, 200, 4090, 4088, ALONE), (1, 4090, 4088, 200, TURNED), (2, 2056, 2050, 2048, ALONE), (1, 3000, 2052, 2060, {}), (1, 3000, 2051, 2061, {}),
                  (3, 600, 1000, 1004, dict(transposed=True))]
GRADIENT_TYPES = [("f32",) * 5, ("bf16",) * 5, ("bf16", "bf16", "f32", "bf16", "f32")]
MIXED = ("f32", "bf16", "f32", "f32", "f32")          # of dz and x the former alone is float

# Operands of batches of workers that share the workspace.
BATCHES = (5, 1500, 712, 1544, {})
BATCH_TYPES = [("f32",) * 5, ("bf16", "f32", "f32", "bf16", "f32")]
BATCH_ROOMS = (1, 40 << 20)
