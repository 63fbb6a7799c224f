"""Sizes of the row operators for the kernels that the sizes of test_rows_gpu.py do not reach, and what reaches what.

reached() is the set of kernels (by the planner's names) that the tests' sizes launch; planned() those that sizes drawn over
the whole range do.
"""
import math
import random

import torch

import test_rows_gpu as rows
from paper_2309_15812_amd import _lib

F32, BF16 = torch.float32, torch.bfloat16
CODE = {F32: _lib.O1D_F32, BF16: _lib.O1D_BF16}

# (M, C): rows of every number of lanes and runs per lane
LAYER_NORM = [(M, C) for C in (33, 40, 47, 49, 56, 296, 303, 317, 320, 393, 400, 427, 504, 1032, 1127, 1128, 1361, 1544, 1720)
              for M in (3, 1500)]
# (M, I, O, dtype, whole runs)
FORWARD = [(24, 100, 70, F32, True), (24, 100, 70, BF16, False), (32, 96, 128, F32, True), (32, 96, 128, BF16, True),
           (14419, 59, 1051, BF16, False), (17721, 112, 624, F32, True), (43208, 128, 224, F32, True)]
INPUT_GRADIENT = [(24, 100, 70, F32, True), (24, 100, 70, BF16, False), (32, 96, 128, F32, True), (32, 96, 128, BF16, True),
                  (21328, 392, 496, BF16, False), (55304, 96, 181, BF16, False), (26309, 579, 72, F32, True),
                  (22297, 184, 304, F32, True), (18008, 312, 168, BF16, True), (16243, 296, 184, BF16, True)]
WEIGHT_GRADIENT = [(47272, 49, 539, F32, True), (1984, 1784, 353, F32, True), (19384, 952, 208, BF16, True),
                   (3104, 1925, 385, BF16, False)]


def names(op, M, I, O, dt, whole, act="none", held=False):
    return set(_lib.rows_kernel_name(op, M, I, O, act, held, CODE[dt], whole).split("+")) - {""}


def reached():
    got = set()

    def add(*args, **kw):
        got.update(names(*args, **kw))

    for dt in (F32, BF16):
        for M, C in rows.LN + LAYER_NORM:
            add("ln_fwd", M, C, 1, dt, True)
            for held in (False, True):
                add("ln_bwd", M, C, 1, dt, True, held=held)
        for M, I, O in rows.MM:
            for k, act in enumerate(rows.ACTS):  # (odd ones in rows off their alignment)
                for held in (False, True):
                    add("linear_fwd", M, I, O, dt, k % 2 == 0, held=held)
                    add("linear_bwd_weight", M, I, O, dt, k % 2 == 0, act=act, held=held)
                add("linear_bwd_input", M, I, O, dt, k % 2 == 0)
    tiles = [(BF16, *c) for c in rows.TILES_BF16 + rows.TILES_BF16_ODD] + [(F32, *c) for c in rows.TILES_F32]
    for dt, M, K, N in tiles:
        for held in (False, True):
            add("linear_fwd", M, K, N, dt, K % 8 == 0, held=held)
        add("linear_bwd_input", M, N, K, dt, K % 8 == 0)
    for dt, O, I, M in [m for m in rows.test_every_weight_gradient_tile.pytestmark if m.name == "parametrize"][0].args[1]:
        for act, held in (("none", False), ("gelu", True), ("silu", False)):
            add("linear_bwd_weight", M, I, O, dt, True, act=act, held=held)
    for c in FORWARD:
        for held in (False, True):
            add("linear_fwd", *c, held=held)
    for c in INPUT_GRADIENT:
        add("linear_bwd_input", *c)
    for c in WEIGHT_GRADIENT:
        add("linear_bwd_weight", *c)
        add("linear_bwd_weight", *c, act="gelu", held=True)
    return got


def planned(count):
    """{kernel: one call that launches it} of `count` calls over the whole range."""
    rng, got = random.Random(2), {}

    def size(lo, hi):
        n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return n | 1 if rng.random() < 0.4 else n - n % 8 if n >= 16 else n

    while count:
        M, I, O = size(1, 200704), size(1, 2048), size(1, 2048)
        if M * I * O > 4e10:
            continue
        count -= 1
        call = (rng.choice(list(_lib.ROWS_OP)), M, I, O, rng.choice((F32, BF16)), rng.random() < 0.6, rng.choice(rows.ACTS),
                rng.random() < 0.5)
        for n in names(*call):
            got.setdefault(n, call)
    return got
