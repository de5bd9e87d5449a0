"""Which launches the calls of window attention and of the paged cache take, and which of them are refused, at sizes that no test runs (see test_operator_kernels.py)."""
from test_operator_kernels import NONE, launches  # noqa: F401 (the fixture)


def test_the_largest_backward(launches):  # noqa: F811
    # 4.3 million tokens of 32 heads, 138 million rows: a bfloat16 backward has no launch that would be too large
    x = launches("window", [1000000] * 4 + [300000], 32, 8, 128, 0, 1000, 0)
    assert [k for k, _, _ in x] == ["window_fwd_kernel", "window_dq_kernel", "window_dkv_kernel"]
