"""mx_attn_decode refuses a scale whose product with the kernel's own factors (2^33 log2 e) is not finite: it made zero scores NaN."""
from tests.test_serving_cpu import BAD, NULL, attend


def test_scales_beyond_the_range():
    for scale in (2.0 ** 94, 1e30, -2.0 ** 94, 3.4e38, float("inf"), float("nan")):
        assert attend(scale=scale) == BAD
    for scale in (0.0, -1.0, 2.0 ** 93, -1.99 * 2.0 ** 93):
        assert attend(scale=scale, q=None) == NULL            # nothing wrong with the scale
