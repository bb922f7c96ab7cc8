"""4-bit products whose rows are long: two blocks of columns on their way, and columns split over workgroups, with every size of group, zeros or none, and both
types.  Bound and definition as in test_gpu_q4."""
import numpy as np
import pytest

import paper_2406_11674_amd as endor
from test_gpu_q4 import TYPES, check, make

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("zeros", [False, True], ids=["sym", "zeros"])
@pytest.mark.parametrize("group", [32, 64, 128, 256, 4096])
@pytest.mark.parametrize("rows,cols,batches,split", [(64, 8192, (1, 2, 16), False), (515, 9001, (1, 2), False), (17, 30001, (1, 3, 16), True),
                                                     (1024, 16640, (2,), True)], ids=str)
def test_long_rows(rows, cols, batches, split, group, zeros, dtype):
    print("q4 long", rows, cols, group, zeros, dtype, flush=True)
    m, w, g = make(rows, cols, group, zeros, seed=rows + group)
    for nb in batches:
        assert (endor.q4_scratch_bytes(m, nb) > 0) == split
        check(m, w, torch.from_numpy(g.standard_normal((nb, cols), dtype=np.float32)).to(TYPES[dtype]))
