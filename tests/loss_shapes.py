"""Sizes that take every tile of the vocabulary loss's products, in one piece of the
vocabulary and in several, with k whole and in runs: tokens, dim, classes.  What the GPU
tests of the tiles run, and the host test holds against the rule."""

SIZES = [
    (2, 70, 129), (65, 70, 20001), (4100, 451, 129), (4100, 70, 5001), (3001, 70, 140001), (4100, 2100, 2049), (4100, 131, 66001),
    (130, 4100, 30001), (9001, 2100, 1001), (9001, 451, 8200), (9001, 1283, 129), (9001, 259, 30001), (4100, 259, 66001),
    (4100, 451, 8200), (9001, 451, 30001), (9001, 777, 30001), (9001, 1283, 30001), (6001, 1283, 66001), (2048, 64, 140001),
]
