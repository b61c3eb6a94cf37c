"""The calls on an 8- or 4-bit cache in forms that few calls take: every way of dealing the work out
and of joining it, in each type and width (tests/test_mx_forms.py checks that the calls take them),
and the write and reading back of very many tokens."""
import numpy as np
import pytest
import torch

from oracle import mx
from oracle import sequence as ref
from tests.mx_forms import FORMS
from tests.seq_util import TYPES
from tests.test_gpu_paged_mx import Case, ints, table_of, wide_numbers

import paper_2607_22696_amd as dsa

pytestmark = pytest.mark.gpu

KINDS = tuple((bits, dtype, D) for bits in (8, 4) for dtype in ("bf16", "f32") for D in (64, 128))


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dsa.load()
    yield


# the join of many rows, seconds of work for the oracle, does not see the bits
@pytest.mark.parametrize("name,bits,dtype,D", [
    (name, *kind) for name in FORMS for kind in KINDS
    if name != "many_rows_to_join" or (kind[0] == 8) == (kind[1] == "bf16")])
def test_attention(name, bits, dtype, D):
    Case(400 + len(name), D=D, bits=bits, dtype=dtype, **FORMS[name][0]).check()


@pytest.mark.parametrize("name", ("few_rows_in_few_parts", "drafts", "chunks", "66_drafts"))
@pytest.mark.parametrize("bits,dtype,D", ((8, "f32", 128), (4, "bf16", 64)))
def test_attention_with_bias(name, bits, dtype, D):
    Case(440 + len(name), D=D, bits=bits, dtype=dtype, bias=(32, 128, False),
         **FORMS[name][0]).check()


@pytest.mark.parametrize("bits,dtype,D", KINDS)
def test_write_and_read_of_many_tokens(bits, dtype, D):
    """More than 65,536 steps of 64 chunks of 8 channels (eight of them to a wave), and not a whole
    number of waves; the rows are some hundred different ones in turn."""
    KH, page, tail = 8, 48, 3
    count = 65536 * 64 // (2 * KH * D // 8) + 78
    new = [count // 2, 1, 0, count - count // 2 - 1]
    held = [new[0] + 5, 900, 70, new[3]]
    rows = count + tail
    steps = rows * (2 * KH * D // 8) / 64
    assert steps > 65536 and steps % 32
    r = np.random.default_rng(90)
    (k, k64), (v, v64) = (wide_numbers(r, (241, KH, D), dtype) for _ in range(2))
    at = np.arange(rows) * 7 % 241
    num = sum(-(-m // page) for m in held) + 3
    pages = table_of(r, held, page, num)
    pages[0, 40], pages[3, 9] = -1, num
    cache = tuple(torch.randint(0, 256, t.shape, dtype=torch.uint8).cuda()
                  for t in dsa.paged_cache_mx(num, page, KH, D, bits, device="cpu"))
    where = np.array(list(mx.places(pages, held, new, page, num)))
    assert len(where) == count - 2 * page
    row, p, j = (torch.tensor(x).cuda() for x in where.T)
    which = torch.tensor(at).cuda()
    want, back = [t.clone() for t in cache], []
    for i, x in enumerate((k64, v64)):
        code, scale = mx.quantise(x, bits)
        value = torch.tensor(mx.values(code, scale, bits).astype(np.float32)).cuda()
        for w, held_as in ((want[i], mx.pack(code, bits)), (want[2 + i], scale)):
            w[p, :, j] = torch.tensor(held_as).cuda()[which[row]]
        back.append(torch.zeros(rows, KH, D, device="cuda"))
        back[i][row] = value[which[row]]
    args = (ints(pages), ints(held), ints(ref.starts(new)))
    dsa.paged_append_mx(k.cuda()[which], v.cuda()[which], cache, *args)
    torch.cuda.synchronize()
    for got, w in zip(cache, want):
        assert torch.equal(got, w)
    for other in TYPES.values():
        for got, w in zip(dsa.paged_read_mx(cache, *args, rows, other), back):
            assert torch.equal(got.float().isnan(), w.isnan())
            assert torch.equal(got.float().nan_to_num(7.0), w.nan_to_num(7.0))
