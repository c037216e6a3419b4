"""The 4-bit cache at the ends of what its calls take, on the GPU (bounds: see test_gpu_kv4.py)."""
import numpy as np
import pytest

import paper_2409_11155_amd as iso      # first: binds libiso to the HIP runtime it was built against
import iso_inputs
from oracle import kv4_oracle as ko
from test_gpu_kv4 import attend, check, device_cache, f64, make_ctx

pytestmark = pytest.mark.gpu
MOST_KEYS = 2 ** 31 - 1024


@pytest.mark.parametrize("dt,nq,d,fresh", [("bf16", 1, 64, 1), ("bf16", 4, 128, 5), ("f32", 1, 64, 1), ("bf16", 64, 64, 64)])
@pytest.mark.parametrize("kv", [MOST_KEYS, 2 ** 31 - 1])
def test_as_many_keys_as_a_table_may_have(dt, nq, d, fresh, kv):
    """Pages of the first and the last keys only, all others are missing: what is seen is known.  Of 2^31 - 1 keys the last 1023 have no
    place in the table."""
    page = 256
    width, n_pages = MOST_KEYS // page, 4
    cols = np.array([0, 1, width - 2, width - 1])
    table = np.full((1, width), -1, np.int32)
    table[0, cols] = [2, 0, 3, 1]
    rng = np.random.default_rng(3)
    codes, scales = zip(*(ko.encode(rng.standard_normal((n_pages, 1, page, d))) for _ in range(2)))
    q = iso_inputs.randn((fresh, nq, d), seed=5, dtype=dt)
    with make_ctx(nq, 1, d, dt) as ctx:
        got = f64(attend(ctx, q, device_cache(codes, scales, page), table, np.array([0, fresh]), [kv], dt, nq, d), dt)
    # the same keys, close together: a row sees as many fewer than the last as before
    gone = (width - 4) * page
    check(got, f64(q, dt), ko.decode(codes[0], scales[0]), ko.decode(codes[1], scales[1]), table[:, cols], page, [0, fresh], [kv - gone], nq, dt, n_pages)
