"""Sizes of the vocabulary's loss that take its 256 x 256 tiles, with what they are there for; (rows, words, elements, share of rows ignored)."""

CASES = {
    "forward, gradient of the logits, dx in splits, dw at once": (1003, 11003, 1000, 0.2),
    "dx and dw at once": (3300, 3290, 3301, 0.0),
    "pieces: dx summed over them and its splits, the last piece's dw in splits": (5000, 30011, 520, 0.1),
    "pieces: dx summed over them alone": (5000, 29501, 2000, 0.0),
}
