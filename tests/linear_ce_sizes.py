"""Sizes of the cross-entropy of a linear layer that take every tile of its kernels, and several pieces of packed operands: (rows, width, classes, type, type of dw, whether rows start on 16-byte
boundaries) -> what bsr_linear_ce_tiles is to say: tile of the forward's logits, of the backward's, of the products; pieces of the classes forward, backward (the least)."""
L, SHORT, SMALL, MID, FEW = 2256256, 2128128, 3128128, 3064128, 4032256

TILES = [
    ((2048, 768, 21841, "bf16", "bf16", True), (L, L, L, 1, 1)),
    ((129, 801, 39950, "bf16", "bf16", False), (L, L, L, 1, 1)),
    ((1500, 1000, 9001, "bf16", "fp32", True), (L, L, L, 1, 1)),
    ((7394, 598, 1038, "bf16", "fp32", False), (L, L, SMALL, 1, 1)),
    ((1025, 200, 21841, "fp32", "fp32", True), (L, L, L, 1, 1)),
    ((137, 275, 49953, "fp32", "fp32", False), (L, L, L, 1, 1)),
    ((5013, 130, 4789, "bf16", "bf16", True), (SHORT, SHORT, L, 1, 1)),
    ((8545, 137, 2209, "bf16", "fp32", False), (SHORT, SHORT, L, 1, 1)),
    ((2300, 200, 9001, "fp32", "fp32", True), (SHORT, SHORT, SMALL, 1, 1)),
    ((79, 233, 23464, "bf16", "bf16", True), (SMALL, SMALL, SMALL, 1, 1)),
    ((5903, 201, 299, "bf16", "fp32", False), (SMALL, SMALL, SMALL, 1, 1)),
    ((77, 191, 18822, "fp32", "fp32", True), (SMALL, SMALL, SMALL, 1, 1)),
    ((999, 4784, 1178, "bf16", "bf16", True), (MID, MID, L, 1, 1)),
    ((5731, 958, 49, "bf16", "fp32", True), (MID, MID, SMALL, 1, 1)),
    ((4487, 1358, 45, "fp32", "fp32", False), (MID, MID, SMALL, 1, 1)),
    ((4590, 3757, 3, "bf16", "bf16", True), (0, 0, L, 0, 1)),
    ((2259, 3043, 5, "fp32", "fp32", False), (0, 0, L, 0, 1)),
]
PIECES = [
    ((2, 300, 5000000, "bf16", "bf16", False), (FEW, FEW, L, 10, 10)),
    ((2, 300, 5000000, "bf16", "fp32", True), (FEW, FEW, L, 10, 10)),
    ((32, 69, 5000000, "fp32", "fp32", True), (FEW, FEW, SMALL, 8, 8)),
    ((300, 130, 1500000, "bf16", "bf16", False), (SHORT, SHORT, L, 3, 8)),
    ((1100, 500, 150001, "bf16", "fp32", True), (SHORT, SHORT, L, 1, 4)),
    ((1100, 500, 150001, "fp32", "fp32", False), (SHORT, L, L, 2, 6)),
    ((90, 200, 400000, "fp32", "fp32", True), (SHORT, SHORT, SMALL, 2, 2)),
]
