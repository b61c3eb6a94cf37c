"""How many bits of alpha paged_forward_mx keeps with bf16 queries: in every form its low part too,
so that outputs are off by little more than their own rounding."""
import pytest
import torch

from tests.mx_forms import PRECISE
from tests.seq_util import Bounds, near
from tests.test_gpu_paged_mx import Case

import numpy as np

from oracle import sequence as ref

import paper_2607_22696_amd as dsa

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dsa.load()
    yield


@pytest.mark.parametrize("bits", (8, 4))
@pytest.mark.parametrize("D", (64, 128))
@pytest.mark.parametrize("tile", PRECISE)
def test_alpha_has_16_bits(tile, D, bits):
    """Small queries give every key about the same weight and logits hardly an error; alpha may be
    off by 2^-17 of itself, where one bf16 number would be by 2^-9 to 2^-8."""
    c = Case(300 + tile, D=D, bits=bits, **PRECISE[tile])
    c.q, c.q64 = c.q / 16, c.q64 / 16  # exact
    out, lse = c.run()
    torch.cuda.synchronize()
    o, l, mag = ref.paged(c.q64, c.k64, c.v64, c.pages, c.held, c.new, True)
    k = np.concatenate([ref.gather(c.k64, c.v64, c.pages[b], m)[0] for b, m in enumerate(c.held)])
    bd = Bounds("bf16", True, c.q64, k, c.new, c.held, 0.0)
    near("out", out, o, bd.out(o, mag))
    near("lse", lse, l, bd.lse(l))
