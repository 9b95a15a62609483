"""Chunks over the 4-bit cache beside many decode rows."""
import pytest

from q4_util import Batch, check

from parity_util import announce

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,dtype,rows", [(128, "bf16", 300), (64, "fp32", 200), (128, "bf16", 1100)])
def test_few_chunk_rows_beside_many_decode_rows(D, dtype, rows):
    """Long chunks in as many parts as the records' bytes leave."""
    announce(f"q4 varlen, 2 and 30 rows on 20000 and 9000 beside {rows} D={D} {dtype}")
    H_q, H_kv = (32, 8) if rows < 1000 else (16, 2)
    lens = [(1 + 7 * i % 60, 1) for i in range(rows)]
    lens[rows // 2] = (20000, 2)
    lens.append((9000, 30))
    b = Batch(lens, H_q, H_kv, D, dtype, seed=rows)
    check(b.attend(b.upload()).float().cpu(), b.expected_gpu(), 20000, dtype)
