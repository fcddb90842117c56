"""Host side of calls around the key / value cache that meet one another (no GPU)."""
import numpy as np

from oracle import cache_oracle as co


def test_the_model_grows_on_a_copy_of_a_shared_page():
    """fork, shorten into a page that both share, grow: a page of its own with the same tokens, and the other sequence's as they were."""
    c, rng = co.Cache(2, 8, 1, 64, 2, 4), np.random.default_rng(0)
    c.grow([0], [150])
    for layer in range(2):
        c.append(layer, *(rng.standard_normal((150, 1, 64)).astype(np.float32) for _ in range(2)), [0, 150], [0])
    c.fork([0], [1])
    co.keep(c, [1], [150], [70])
    shared, before = int(c.table[0, 1]), [c.sequence(layer, 0) for layer in range(2)]
    assert int(c.table[1, 1]) == shared and c.refs[shared] == 2
    c.grow([1], [2])
    assert int(c.table[1, 1]) != shared and c.refs[shared] == c.refs[c.table[1, 1]] == 1 and c.refs[c.table[0, 0]] == 2
    x = rng.standard_normal((2, 1, 64)).astype(np.float32)
    for layer in range(2):
        c.append(layer, x, x, [0, 2], [1])
        for a, b in zip(before[layer], c.sequence(layer, 0)):
            np.testing.assert_array_equal(a, b)
        for a, b in zip(before[layer][:2], c.sequence(layer, 1)[:2]):
            np.testing.assert_array_equal(a[:, :70], b[:, :70])
    c.grow([1], [1])
    assert c.refs.sum() == (c.table >= 0).sum()
