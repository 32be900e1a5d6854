"""Outputs of the attention whose rows or heads overlap are refused: several workgroups would write the same elements."""
import itertools

from paper_2302_01382_amd import mpq
from test_abi_host import FAKE16, needs_no_gpu
from test_serving_abi import kv


@needs_no_gpu
def test_outputs_that_overlap_are_refused():
    """Every pattern of few rows and heads against the elements that they cover.  A call that is taken ends at its missing
    workspace."""
    dim, taken = 16, 0
    for rows, heads in itertools.product((1, 2, 3, 5), (1, 2, 4)):
        c, b = kv({"heads": 1, "dim": dim}, {"rows": rows, "max_new": rows, "seqs": 1, "max_len": 100000, "table_pages": 7000})
        for ts, hs in itertools.product((0, 1, 8, 15, 16, 17, 31, 32, 33, 40, 48, 63, 64, 65, 80, 96, 160), repeat=2):
            cells = [i * ts + h * hs + d for i in range(rows) for h in range(heads) for d in range(dim)]
            rc = mpq.lib().mpq_kv_attention(c, b, 1, FAKE16, heads * dim, dim, heads, 0.125, 1, 0, FAKE16, ts, hs, None, 0, None)
            assert rc == (mpq.ERR_WORKSPACE if len(set(cells)) == len(cells) else mpq.ERR_SHAPE), (rows, heads, ts, hs)
            taken += rc == mpq.ERR_WORKSPACE
    assert taken > 500
