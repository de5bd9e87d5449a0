"""Which launches the calls of window attention and of the paged cache take, and which of them are refused, at sizes that no test runs (see test_operator_kernels.py)."""
import ctypes as C

from paper_2604_13847_amd import binding as sb
from test_operator_kernels import NONE, launches  # noqa: F401 (the fixture)


def test_the_largest_backward(launches):  # noqa: F811
    # 4.3 million tokens of 32 heads, 138 million rows: a bfloat16 backward has no launch that would be too large
    x = launches("window", [1000000] * 4 + [300000], 32, 8, 128, 0, 1000, 0)
    assert [k for k, _, _ in x] == ["window_fwd_kernel", "window_dq_kernel", "window_dkv_kernel"]


def serving(S, total, most, length, Hq=32, Hkv=8, D=128, page=64, pages=None):
    c = sb.sb_cache(1 << 20, page, Hkv, D, sb.SB_BF16, -(-length // page) if pages is None else pages, 4096, 4096, 4096)
    return c, sb.sb_chunk(S, Hq, total, most, length, 0.0, 4096, 4096)


def ws_bytes(c, n, window=NONE):
    out = C.c_int64()
    sb._check(sb.lib().sb_cache_attn_ws_bytes(C.byref(c), C.byref(n), window, 0, C.byref(out)))
    return out.value


def test_a_prompt_beside_single_tokens_asks_for_no_sums_of_its_own():
    """What the joined runs take is counted in the rows of sequences that have runs, not in the prompt's."""
    alone = ws_bytes(*serving(64, 64, 1, 32768))
    assert alone == 64 * 32 * 32 * (4 + 4 * 128)                                       # 32 runs of 64 rows of 32 heads
    # with up to 16 rows (64 of a group of four) of 64 sequences
    assert ws_bytes(*serving(64, 8192 + 63, 8192, 32768)) <= 16 * alone
    assert ws_bytes(*serving(64, 65536 + 63, 65536, 131072)) <= 4 * 16 * alone
    assert ws_bytes(*serving(64, 100, 37, 32768)) <= alone * 100 // 64 + 512           # fewer tokens in all than that


def test_a_length_that_the_table_cannot_hold():
    """max_length is about how long a sequence gets, whatever the caller knows of that; keys behind the page table do not exist."""
    assert ws_bytes(*serving(64, 64, 1, NONE, pages=512)) == ws_bytes(*serving(64, 64, 1, 32768))
    assert ws_bytes(*serving(2, 300, 200, NONE, pages=512)) == ws_bytes(*serving(2, 300, 200, 32768))
    assert ws_bytes(*serving(1, 1, 1, NONE, pages=1)) == ws_bytes(*serving(1, 1, 1, NONE, pages=0)) == 0
