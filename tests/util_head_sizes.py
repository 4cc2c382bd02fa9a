"""Sizes (rows, tokens, elements) at which the products on the output head take each of their tile shapes."""

# log probabilities and the 8-bit product, more than 64 rows; odd vocabularies end inside a tile
FORWARD = [(65, 1001, 64), (100, 40001, 64), (150, 17003, 64), (333, 20011, 64), (500, 20011, 128), (1100, 5003, 64), (577, 7001, 192)]
# its gradient: the products with the hidden elements as rows need several tiles of these, too
GRADIENT = [(65, 1001, 64), (100, 40001, 64), (333, 20011, 320), (500, 20011, 128), (550, 7001, 320), (1100, 5003, 64), (40, 3001, 64)]
# the gradient goes through the vocabulary in several pieces: few rows, and many
PIECES = [(3, 450003, 8), (70, 280003, 64), (600, 130003, 64)]
