"""What the library refuses of a cycle's batch is refused through the engine in the library's words, with rotary positions and without."""
import numpy as np
import pytest

from lr_workloads import Model, bf16_round
from paper_2506_19830_b200 import binding as B
from paper_2506_19830_b200.cycle import BranchInput, PagedCycleEngine, RequestInput

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kv_dtype,turned", [("bf16", False), ("bf16", True), ("mxfp4", True)])
@pytest.mark.parametrize("node,parents,own,q_len,words", [(5, (), 3, 2, "depth 5"), (-1, (), 3, 2, "depth -1"), (1, (3,), 3, 2, "continues 3"), (1, (-1,), 3, 2, "continues -1"),
                                                         (1, (), 3, 5, "own_len 3 < q_len 5"), (1, (), 0, 2, "own_len 0 < q_len 2")])
def test_a_batch_that_does_not_hold_together(node, parents, own, q_len, words, kv_dtype, turned):
    rng = np.random.default_rng(3)
    eng = PagedCycleEngine(Model(8, 2, 64, 16), 20, kv_dtype=kv_dtype, rope=B.Rope(64) if turned else None)
    rows = lambda n, h=2: bf16_round(rng.standard_normal((n, h, 64)).astype(np.float32))  # noqa: E731
    eng.add_request(rows(20), rows(20))
    x = RequestInput([(rows(5), rows(5))], [BranchInput(node, rows(own), rows(own), q_len, 1)], parents)
    with pytest.raises(B.LrError) as e:
        eng.run_cycle([x], rows(q_len, 8), np.zeros((2, 16), dtype=np.uint16), np.zeros(1, dtype=np.int32), np.ones(1, dtype=np.uint8))
    assert e.value.status == -1 and words in str(e.value)
