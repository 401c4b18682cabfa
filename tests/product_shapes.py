"""Sizes of matrices whose products have to go a certain way, for the tests on the GPU and for the one that asks the host code which way they
go: (W, T, inputs, outputs, more of test_gpu_linear.Layer)."""

# Rows of very different sizes: operands that are packed to binary16, or to bf16 parts.
RANGE = (2, 1500, 712, 1544, dict(bias=False))
RANGE_TYPES = [("f32", "f32", "f32"), ("bf16", "f32", "f32"), ("f32", "bf16", "f32"), ("f32", "f32", "bf16")]
