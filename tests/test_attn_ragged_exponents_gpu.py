"""Block exponents at the lower end of an E4M3 cache (ragged attention)."""
import numpy as np
import pytest

import paged_ref
from gpu_helpers import log
from paged_ref import Batch
from test_attn_ragged_gpu import run_paged

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,G", [([(1, 200), (3, 90)], 4), ([(70, 200)], 2)])
@pytest.mark.parametrize("exps", [(0, 1), (0, 6), (3, 9)])
def test_smallest_block_exponents(lens, G, exps):
    """Exponent bytes from 0 (2^-127) on against queries of up to 2^120: the codes from 0x40 on (2 to 448) decode to normal
    bf16 values down to 2^-126, which the scores of order 1 need."""
    import torch
    b = Batch(lens, 2 * G, 2, 128, 16, seed=5, fp8=True)
    g = torch.Generator().manual_seed(9)
    nan = (b.k & 0x7F) == 0x7F
    b.k = torch.randint(0x40, 0x7E, b.k.shape, generator=g, dtype=torch.uint8) | (torch.randint(0, 2, b.k.shape, generator=g, dtype=torch.uint8) << 7)
    b.k[nan] = 0x7F
    b.k_exp = torch.randint(exps[0], exps[1] + 1, b.k_exp.shape, generator=g, dtype=torch.uint8)
    b.q = (torch.randn(b.q.shape, generator=g) * 2.0 ** (118 - exps[1])).bfloat16()
    log(f"paged smallest exponents {lens} G={G} {exps}")
    o, a, mine = b.expected(1)
    got = run_paged(b, 1)
    assert np.all((np.abs(got - o) <= paged_ref.attention_tolerance(a))[mine])
