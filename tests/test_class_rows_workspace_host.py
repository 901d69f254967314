"""Workspace of the class layer on rows: what is asked for the largest batch is enough for every smaller one."""
import random

import pytest

from paper_1302_1690_amd import mpcnn

# features, classes: few rows' ways and where they end, kept scores and not, pieces, little work only, one class
SHAPES = [(1000, 30011), (768, 50257), (64, 1100), (16, 30), (5, 6), (2048, 19600), (100, 37), (320, 13000), (1000, 1000), (4096, 3000), (127, 20011), (1, 1), (3, 400000),
          (4096, 128000), (1031, 9700), (20000, 700)]


def _one(rows, features, classes, dtype, training):
    return mpcnn.lib().mpcnn_workspace_bytes_class_call(rows, features, classes, dtype, 1 if training else 0)


@pytest.mark.parametrize("training", [False, True], ids=["loss", "gradients"])
@pytest.mark.parametrize("dtype", [0, 1], ids=["f32", "bf16"])
@pytest.mark.parametrize("features,classes", SHAPES)
def test_enough_for_every_smaller_batch(features, classes, dtype, training):
    most, asked = 0, random.Random(features + classes).sample(range(300, 9000), 12)
    for rows in range(9001):
        most = max(most, _one(rows, features, classes, dtype, training))
        if rows < 300 or rows % 1000 == 0 or rows in asked:
            assert mpcnn.class_workspace_bytes(rows, features, classes, dtype, training) == most, rows


@pytest.mark.parametrize("dtype", [0, 1], ids=["f32", "bf16"])
def test_it_never_shrinks(dtype):
    size = mpcnn.class_workspace_bytes
    last = 0
    for rows in (1, 7, 64, 100, 1000, 5000):
        now = size(rows, 256, 1000, dtype, True)
        assert now >= last
        last = now
    assert size(16, 1000, 30011, dtype, True) <= size(17, 1000, 30011, dtype, True)
    assert size(5106, 768, 50257, dtype, True) <= size(6207, 768, 50257, dtype, True)


def test_up_to_the_most_rows():
    rng = random.Random(3)
    for features, classes in ((5, 6), (24, 40003), (200, 1000)):
        enough = mpcnn.class_workspace_bytes(1 << 20, features, classes, 0, True)
        for _ in range(3000):
            assert _one(int(2 ** rng.uniform(0, 20)), features, classes, 0, True) <= enough
        assert _one(1 << 20, features, classes, 0, True) <= enough


def test_of_one_call():
    for bad in ((-1, 16, 30, 0), (20, 0, 30, 0), (20, 16, 0, 0), (20, 16, 30, 2), ((1 << 20) + 1, 16, 30, 0)):
        assert _one(*bad, True) == mpcnn.class_workspace_bytes(*bad, True) == 0
    assert 0 < _one(0, 16, 30, 0, True) <= _one(20, 16, 30, 0, True)
