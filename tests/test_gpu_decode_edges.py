"""Cache attention and group-scaled linears where their kernels can go wrong
apart from ordinary inputs: numbers at the ends of their ranges, and the forms
that only some sizes reach. Tolerances are those derived in
test_gpu_decode.py.
"""

import numpy as np
import pytest
import torch

from oracle import decode as od
from tests.test_gpu_decode import Paged, attend, fill, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("page,D,H,Hkv,new", [(16, 128, 2, 1, 40), (64, 64, 6, 2, 61), (32, 128, 7, 1, 64),
                                              (64, 128, 8, 2, 2), (16, 64, 6, 3, 7), (32, 128, 2, 1, 19)])
@pytest.mark.parametrize("scale", [None, 1e-20])
@pytest.mark.parametrize("masked", [False, True])
def test_causal_zero_rows(abi, dtype, page, D, H, Hkv, new, scale, masked):
    """Each kernel, causal: query rows that are zero or tiny, key blocks that
    are zero (at the smallest scale and at none), as padding leaves them. The
    factor of a score may then be too small for a float, and the scores of
    keys that a row does not see are -inf."""
    rng = np.random.default_rng(new + D)
    lens = [23, new, new + 13, 203, 1201]
    count = [new, new, new - 1, new, new]
    pg = Paged(abi, rng, len(lens), max(lens), Hkv, page, D)
    fill(pg, rng, lens)
    for b, L in enumerate(lens):
        for blk in range((L + page - 1) // page):
            if blk % 3 != 1:                          # the last blocks among them
                p = pg.table[b, blk]
                pg.k[p], pg.ks[p] = 0, od.SCALE_FLOOR if blk % 3 == 0 else 0.0
    pg.cache.K.copy_(torch.from_numpy((pg.k + 128).astype(np.uint8)))
    pg.cache.k_scale.copy_(torch.from_numpy(pg.ks))
    q, _ = randn(rng, (sum(count), H * D), dtype)
    q[0::5] = 0
    q[1::5] *= 1e-30 if dtype is torch.bfloat16 else 2.0 ** -22
    q[2::5, :D] = 0                                   # one head of a row
    mask = (rng.random((len(lens), max(lens))) < 0.6).astype(np.uint8) if masked else None
    attend(abi, rng, pg, count, lens, H, dtype, causal=True, mask=mask, scale=scale, q=q)
