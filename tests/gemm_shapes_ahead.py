"""Sizes of the gated feed-forward block that take the 256 x 256 tile with two buffers, and
with the projections saved the one with three: activation, tokens, dim, hidden."""

BOTH = [("silu", 4100, 456, 9001), ("gelu", 8200, 776, 4100), ("relu", 2049, 776, 16001)]
