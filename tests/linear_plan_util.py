"""Shapes of linear layers by the kernels that their passes take, for the tests of these kernels: on the host a test holds the library's plan against
them, so that a rule that moves does not leave a kernel without its test."""

# M, K, N of bf16 layers whose three products all take tiles of 256: steps of 64 in odd and even numbers, ends inside a step, a tile and a half of one
LARGE = [(3080, 2872, 3128), (3064, 2936, 2936), (2824, 2824, 2824)]
