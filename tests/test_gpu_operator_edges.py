"""Window attention and the paged cache where their inputs end or hold what is no number: against the same plain 64-bit forms as test_gpu_operators.py."""
import pytest
import torch

import operator_reference as ref
from paper_2604_13847_amd import binding as sb
from test_gpu_operators import DEV, NONE, Served, batch, nan, normal

pytestmark = pytest.mark.gpu
INF = float("inf")


# ---------------------------------------------------------------- tokens behind the page table
# (have, new, page, columns of the table, window, sinks): prompts' chunks and single tokens, rows in front of the table's end and behind it, windows and sinks that pass it
SHORT = [([0, 300], [200, 150], 16, 5, NONE, 0), ([70, 0], [130, 90], 16, 5, 40, 10), ([0, 130], [200, 100], 32, 3, 50, 500), ([64], [300], 16, 1, NONE, 7),
         ([100, 79, 80, 81, 40], [1, 1, 1, 1, 1], 16, 5, NONE, 0), ([200, 90], [1, 3], 16, 5, 20, 300), ([900, 30], [150, 1], 64, 2, 30, 400),
         ([0, 500], [180, 1], 16, 0, NONE, 3), ([600], [200], 64, 0, 100, 700)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("have,new,page,columns,window,sinks", SHORT)
def test_tokens_behind_the_page_table_are_seen_by_no_row(have, new, page, columns, window, sinks, dtype):
    x = Served(have, new, 8, 2, 128, page, dtype, spare_rows=1)
    x.table = x.table[:, :columns].contiguous()
    x.cache = sb.Cache(x.k_pages, x.v_pages, x.table)
    o, lse = x.check(window, sinks, there=lambda s, u: u < columns * page)
    for s, a in enumerate(have):
        if columns == 0 or (a - window + 1 >= columns * page and sinks == 0):
            rows = slice(x.cu[s], x.cu[s + 1])
            assert float(o[rows].abs().max()) == 0 and bool((lse[:, rows] == -INF).all())
