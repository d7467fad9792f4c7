"""The 4-bit format's definition, and refusals of the packed-prompt calls that need no device."""
import numpy as np

from oracle import prompt_oracle as po
from paper_2503_05840_b200 import binding as B


def test_missing_arguments_are_refused():
    L = B.lib()
    assert L.slim_prompt_workspace_bytes(None, 1, 1, 1, 1) == 0
    assert L.slim_prompt_attention(None, None, None, None, 0, 1, None, None, 1, 1, 1, 1, 1, None, None, None) == B.SLIM_ERR_INVALID_ARG
    assert L.slim_append_rows(None, None, None, None, None, 1, None) == B.SLIM_ERR_INVALID_ARG
    assert L.slim_read_rows(None, None, None, None, 1, None, None) == B.SLIM_ERR_INVALID_ARG
    assert L.slim_decode_typed(None, None, None, None, None, None, B.SLIM_F32, None, None) == B.SLIM_ERR_INVALID_ARG
    assert L.slim_decode_typed(None, None, None, None, None, None, B.SLIM_FP4, None, None) == B.SLIM_ERR_INVALID_ARG


def test_scales_are_float16_without_sign_and_lower_bits():
    bits = (np.arange(0xe3, dtype=np.uint16) << 7).view(np.float16).astype(np.float64)
    assert np.array_equal(bits, po.SCALES) and po.SCALES[-1] == 10240


def test_quantised_keys_are_the_nearest_values():
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.standard_normal((20, 70)) * 10.0 ** rng.integers(-6, 5, (20, 1)), rng.integers(-12, 13, (20, 70)) / 2.0, np.zeros((1, 70))])
    codes, scales = po.fp4_quantise(x)
    v = po.fp4_values(codes, scales)
    s = np.repeat(po.SCALES[scales], 32, axis=1)[:, :70]
    inside = np.abs(x) <= 6 * s
    assert (np.abs(v - x) <= s)[inside].all()                       # half the widest gap
    assert ((6 * s >= np.abs(x)) | (s == 10240)).all()
    again = po.fp4_values(*po.fp4_quantise(v))
    # A value of the format stands for itself where the scale is a normal float16: the scale before it is then at least 8/9 s, so the
    # largest key is above 5.3 s and stored as 6 s, which asks for the same scale.
    normal = s >= 2.0 ** -14
    assert normal.mean() > 0.5 and np.array_equal(again[normal], v[normal])


def test_attention_of_one_key_is_its_value():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((3, 4, 8)), rng.standard_normal((1, 2, 8)), rng.standard_normal((1, 2, 8))
    o, _, _ = po.attention(q, k, v, 1e4, False)
    assert np.allclose(o, v[:, [0, 0, 1, 1]])
    o, _, _ = po.attention(q, k, v, 1e4, True)                      # three queries, one key: only the last attends it
    assert not o[:2].any() and np.allclose(o[2], v[0, [0, 0, 1, 1]])
