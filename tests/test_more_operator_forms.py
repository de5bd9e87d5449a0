"""Which launches the four-bit cache's calls make, so that a change of the rules does not leave forms without a test of their values."""
import pytest

from test_more_operator_kernels import launches  # noqa: F401 (a fixture)


@pytest.mark.parametrize("dtype,total,workgroups", [(0, 2048, 512), (0, 4096, 1024), (0, 4097, 1025), (0, 6000, 1500), (0, 7680, 1920), (0, 8193, 2049), (0, 10000, 2500), (0, 16384, 4096),
                                                    (0, 100000, 25000), (1, 4097, 1025), (1, 8192, 2048), (1, 8193, 2049)])
def test_append_of_many_tokens_fills_the_chip(launches, dtype, total, workgroups):  # noqa: F811
    """A token more never makes much fewer wavefronts than the 4096 that fill the chip: four to a workgroup, a token each."""
    assert launches("append", 2, total, total, 9000, 32, 8, 128, dtype, 1) == [("cache4_append_kernel", workgroups, 1)]
