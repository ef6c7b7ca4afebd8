"""The few-token layer in every geometry that its rules choose (test_decode_geometry.py checks that the cases get there):
1, 2 or 4 waves on the same features in the up- and the down-projection, K of whole units or not, rows that fit into
LDS at once or come in rounds, with a shared expert and without."""
import pytest

import test_gpu_decode as td
from paper_2607_18631_amd.workloads import MoEShape

pytestmark = pytest.mark.gpu
BASE = MoEShape(T=16, d=256, E=8, top_k=2, F=96, E_local=8)
CASES = [
    dict(d=32, F=14400),                            # many features to go up, long sums down
    dict(d=256, F=14592),
    dict(d=6400, F=32, F_shared=32),                # and the other way round
    dict(d=6400, F=256),
    dict(d=1600, F=640, F_shared=288),
    dict(d=1792, F=768, F_shared=512),
    dict(d=4096, F=96, E=2, E_local=2, top_k=1, T=64, F_shared=64),     # 16 rows of 4096 values: in rounds
    dict(d=96, F=4128, E=2, E_local=2, top_k=1, T=64, F_shared=4096),
    dict(d=288, F=160),
    dict(d=256, F=256),
]


@pytest.mark.parametrize("mixed", [False, True], ids=["bf16", "e2m1"])
@pytest.mark.parametrize("kw", CASES, ids=lambda kw: "-".join(f"{k}{v}" for k, v in kw.items()))
def test_every_geometry(kw, mixed):
    td.check(BASE.replace(**kw), mixed, seed=5)
