"""Host-side checks of the operators around the optimizer step: struct layouts of the binding, and the
oracle's own formulas (gradients against differences, the dither's distribution, the stall that it
prevents) before anything on a GPU is compared with them."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

from oracle import operators_oracle as O

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_struct_layouts_match_the_header(tmp_path):
    from paper_2505_23725_b200 import binding as B
    src = tmp_path / "t.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "muloco.h"\n'
                   'int main(void){printf("%zu %zu %zu %zu %zu %zu %zu %d\\n", sizeof(muloco_adamw_config),'
                   ' sizeof(muloco_adamw_tensor), sizeof(muloco_qk_norm), sizeof(muloco_ffn),'
                   ' offsetof(muloco_adamw_tensor, wd_mult), offsetof(muloco_qk_norm, gain_q), offsetof(muloco_ffn, x),'
                   ' MULOCO_ADAMW_BLOCK); printf("%zu %zu\\n", offsetof(muloco_config, adam_state_bits),'
                   ' (size_t)MULOCO_ADAMW_STATE8_BYTES(257)); return 0;}\n')
    exe = tmp_path / "t"
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    out = [int(x) for x in subprocess.check_output([str(exe)]).decode().split()]
    assert out == [C.sizeof(B.AdamwConfig), C.sizeof(B.AdamwTensor), C.sizeof(B.QkNorm), C.sizeof(B.Ffn),
                   B.AdamwTensor.wd_mult.offset, B.QkNorm.gain_q.offset, B.Ffn.x.offset, B.ADAMW_BLOCK,
                   B.Config.adam_state_bits.offset, 2 * (256 + 4)]
    # the packed forms are the structs' bytes
    assert len(B._QK_PACK(*range(8), 0.5, *range(12))) == C.sizeof(B.QkNorm)
    assert len(B._FFN_PACK(*range(13))) == C.sizeof(B.Ffn)
    a = B.QkNorm.from_buffer_copy(B._QK_PACK(1, 2, 3, 4, 5, 6, 1, 0, 0.25, 0, *range(10, 21)))
    assert (a.tokens, a.heads_k, a.rotary_dim, a.eps, a.gain_q, a.k, a.k_head_stride) == (1, 4, 6, 0.25, 10, 16, 20)


def test_a_null_context_is_an_argument_error():
    from paper_2505_23725_b200 import binding as B
    lib = B.load_library()
    assert lib.muloco_adamw_create(None, None, None, 0, None) == B.EINVAL
    assert lib.muloco_adamw_step(None, None, 1, 1.0) == B.EINVAL
    assert lib.muloco_adamw_moments(None, None, None) == B.EINVAL
    lib.muloco_adamw_destroy(None)
    assert lib.muloco_qk_norm_rope(None, b"", None, 0, 0, None, 0, 0) == B.EINVAL
    assert lib.muloco_qk_norm_rope_backward(None, b"", None, 0, 0, None, 0, 0, None, None, None, None) == B.EINVAL
    assert lib.muloco_gated_ffn(None, b"", None, None, None, None) == B.EINVAL
    assert lib.muloco_gated_ffn_backward(None, b"", None, 0, *[None] * 9) == B.EINVAL


def _differences(f, x, h=1e-5):
    d = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        y = x.copy()
        y[i] += h
        z = x.copy()
        z[i] -= h
        d[i] = (f(y) - f(z)) / (2 * h)
    return d


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,rot", [(6, 6), (8, 4), (4, 0)])
def test_norm_gradient_against_differences(dim, rot, interleaved):
    rng = np.random.default_rng(dim + rot)
    x, gain = rng.standard_normal((2, 3, dim)), rng.standard_normal(dim)
    ang = rng.standard_normal((2, rot // 2))
    cos, sin = np.cos(ang), np.sin(ang)
    dy = rng.standard_normal(x.shape)
    dx, dgain, _ = O.qk_norm_backward(dy, x, gain, cos, sin, 1e-3, interleaved)
    loss = lambda x_, g_: float((O.qk_norm(x_, g_, cos, sin, 1e-3, interleaved) * dy).sum())   # noqa: E731
    # central differences of step 1e-5: truncation about 1e-10, rounding about 1e-11
    assert np.allclose(dx, _differences(lambda y: loss(y, gain), x), atol=1e-8)
    assert np.allclose(dgain, _differences(lambda y: loss(x, y), gain), atol=1e-8)


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_feed_forward_gradient_against_differences(act):
    rng = np.random.default_rng(3)
    x, w1, w3, w2 = (rng.standard_normal(s) for s in ((3, 4), (4, 5), (4, 5), (5, 4)))
    dy = rng.standard_normal((3, 4))
    _, g, u, h = O.gated_ffn(x, w1, w3, w2, act)
    grads = O.gated_ffn_backward(dy, x, w1, w3, w2, g, u, h, act)[:4]
    args = [x, w1, w3, w2]
    for i, d in zip((0, 1, 2, 3), grads):
        def loss(z, i=i):
            a = list(args)
            a[i] = z
            return float((O.gated_ffn(*a, act)[0] * dy).sum())
        assert np.allclose(d, _differences(loss, args[i]), atol=1e-7)


def test_dither_is_uniform_and_differs_from_step_to_step():
    n = 1 << 16
    u1, u2 = O.dither(n, 12345, 7, 3)
    for u in (u1, u2):
        assert 0 <= u.min() and u.max() < 1
        # mean of n uniforms: standard deviation 1 / sqrt(12 n) = 0.0011; five of them
        assert abs(u.mean() - 0.5) < 0.006
        counts = np.histogram(u, 64, (0, 1))[0]
        # 63 degrees of freedom: mean 63, standard deviation 11
        assert ((counts - n / 64) ** 2 / (n / 64)).sum() < 63 + 6 * 11.3
    # correlations of n pairs have standard deviation 1 / sqrt(n) = 0.004
    assert abs(np.corrcoef(u1, u2)[0, 1]) < 0.02
    assert abs(np.corrcoef(u1, O.dither(n, 12345, 7, 4)[0])[0, 1]) < 0.02
    assert abs(np.corrcoef(u1[:-1], u1[1:])[0, 1]) < 0.02


def test_second_moment_follows_a_falling_gradient():
    """beta2 = 0.99 and gradients that drop to a hundredth: the average has to come down although a step moves
    it by less than half a code (rounding to nearest would keep it where it is)."""
    rng = np.random.default_rng(0)
    n = 2 * O.BLOCK
    c1, s1 = np.zeros(n, np.int8), np.zeros(2, np.float32)
    c2, s2 = np.full(n, 200, np.uint8), np.full(2, 1 / 200, np.float32)      # sqrt(v) = 1
    for t in range(1, 301):
        g = (0.01 * rng.standard_normal(n)).astype(np.float32)
        c1, s1, c2, s2, _, root = O.adamw8(g, c1, s1, c2, s2, t, 0, 11, 0.9, 0.99)
    # exact: v = 0.99^300 + about 1e-4 = 0.0491, root 0.2216; the spread of the codes adds to the mean of the
    # square, by less than a quarter code squared a step, summed with the average's weights
    want = np.sqrt(0.99 ** 300 + (1 - 0.99 ** 300) * 1e-4)
    assert abs(root.mean() / want - 1) < 0.05
