"""Calls of the sequence kernels with more workgroups than a launch has in one dimension (2^32
threads): many sequences, most of them empty, give the bits of the same tokens without the empty
ones; a long write."""
import numpy as np
import pytest
import torch

import paper_2607_22696_amd as dsa

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dsa.load()
    yield


def starts(lengths):
    return torch.tensor(np.concatenate([[0], np.cumsum(lengths)]), dtype=torch.int32).cuda()


def spread_out(lengths, count, seed):
    """The lengths in their order among `count` sequences, the first and the last ones included,
    and where they stand."""
    r = np.random.default_rng(seed)
    at = np.sort(r.choice(np.arange(1, count - 1), len(lengths) - 2, replace=False))
    at = np.concatenate([[0], at, [count - 1]])
    many = np.zeros(count, np.int64)
    many[at] = lengths
    return many, at


@pytest.mark.parametrize("dtype,D,biased", ((torch.bfloat16, 128, False), (torch.bfloat16, 64, True),
                                            (torch.float32, 64, False)))
def test_many_sequences(dtype, D, biased):
    """1,100,000 sequences of 16 heads: 17.6 million workgroups."""
    lengths, H = [1 + 7 * i % 300 for i in range(70)], 16
    many, _ = spread_out(lengths, 1_100_000, 1)
    g = torch.Generator("cuda").manual_seed(2)
    q, k, v, dout = (torch.randn(sum(lengths), H, D, generator=g, device="cuda").to(dtype)
                     for _ in range(4))
    how = {}
    if biased:
        rel_buckets, rel_min = dsa.relative_buckets(4, 7, both=False)
        how = dict(rel_table=torch.randn(4, H, generator=g, device="cuda"), rel_min=rel_min,
                   rel_buckets=rel_buckets)
    got = []
    for cu in (starts(lengths), starts(many)):
        out, lse, res = dsa.seq_forward(q, k, v, cu, causal=True, need_residual=True, **how)
        grads = dsa.seq_backward(q, k, v, out, res, lse, dout, cu, causal=True, **how)
        got.append((out, lse, *grads[:3]))
        torch.cuda.synchronize()
        print(f"  {cu.numel() - 1} sequences", flush=True)
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_many_requests():
    """2,200,000 requests of 8 key heads."""
    new, held, page, H, KH, D = [1, 2, 1, 1, 5], [300, 40, 17, 1, 64], 16, 16, 8, 64
    many, at = spread_out(new, 2_200_000, 3)
    g = torch.Generator("cuda").manual_seed(4)
    counts = [-(-n // page) for n in held]
    kp, vp = (torch.randn(sum(counts), page, KH, D, generator=g, device="cuda").bfloat16()
              for _ in range(2))
    q = torch.randn(sum(new), H, D, generator=g, device="cuda").bfloat16()
    table = torch.full((len(new), max(counts)), -1, dtype=torch.int32)
    for b, c in enumerate(counts):
        table[b, :c] = torch.arange(c) + sum(counts[:b])
    lens = torch.tensor(held, dtype=torch.int32)
    wide, wide_lens = torch.zeros(len(many), max(counts), dtype=torch.int32), \
        torch.zeros(len(many), dtype=torch.int32)
    wide[at], wide_lens[at] = table, lens
    a = dsa.paged_forward(q, kp, vp, table.cuda(), lens.cuda(), starts(new), need_lse=True)
    b = dsa.paged_forward(q, kp, vp, wide.cuda(), wide_lens.cuda(), starts(many), need_lse=True)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_a_long_write():
    """67 million tokens, one wave each."""
    n, page, D = (1 << 26) + 5, 1 << 16, 64
    count = n // page + 1
    k = torch.empty(n, 1, D, dtype=torch.int16, device="cuda").random_().view(torch.bfloat16)
    kp, vp = (torch.zeros(count, page, 1, D, dtype=torch.bfloat16, device="cuda")
              for _ in range(2))
    table = torch.arange(count, dtype=torch.int32, device="cuda").flip(0).contiguous()[None]
    dsa.paged_append(k, k, kp, vp, table, torch.tensor([n], dtype=torch.int32).cuda(), starts([n]))
    for pages in (kp, vp):
        held = pages.flip(0).flatten(0, 1).view(torch.int16)
        assert torch.equal(held[:n], k.view(torch.int16)) and not held[n:].any()
