"""Which form a feed-forward product takes, without a GPU: every form is reached by some test's shapes on a B200's 148
multiprocessors, so that a change of the limits cannot leave one untested."""
import test_gpu_operator_forms as large
import test_gpu_operators as small

from paper_2505_23725_b200 import binding

ALL = {"gate", "y", "gate_back", "dx"}


def test_forms_of_the_tested_shapes():
    for shape in large.FFN_SHAPES:
        forms, tiles = binding.ffn_forms(*shape)
        assert forms == ALL and min(tiles) > 74, (shape, forms, tiles)
    few = set()
    for shape in small.FFN_SHAPES:
        few |= ALL - binding.ffn_forms(*shape)[0]
    assert few == ALL


def test_tiles_of_a_known_size():
    # 4100 tokens: 17 tile rows; d = 1032 and F = 1160: 5 tiles of 256, 10 of 128 columns of W1 and W3
    assert binding.ffn_forms(4100, 1032, 1160) == (ALL, [170, 85, 85, 85 + 3 * 25])
    # one token: only the weight gradients are on such tiles
    assert binding.ffn_forms(1, 768, 2048) == (set(), [0, 0, 0, 3 * 24])
