"""Kernels that only large batches reach: whole heads of fp32 backward between 65 and 128 positions, and short
sequences with shared heads in blocks that go through many of them."""
import math

import pytest
import torch

from paper_2407_15452_b200 import binding as B
from tests.attention_reference import check, reference

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
ALL, CAUSAL = (-1, -1), (-1, 0)
DEV = "cuda"


def tensors(b, lq, lk, hq, hk, d, dt, seed, row=None):
    gen = torch.Generator(device=DEV).manual_seed(seed)

    def make(n, h, gain=1.0):
        x = (torch.randn((b, n, h, d), generator=gen, device=DEV) * gain).to(dt)
        if row is None:
            return x
        room = torch.full((b, n, h, row), math.nan, dtype=dt, device=DEV)      # rows further apart, NaN in between
        room[..., :d] = x
        return room[..., :d]
    return make(lq, hq), make(lk, hk), make(lk, hk), make(lq, hq, 0.25)


def lengths(b, n, seed):
    values = torch.randint(0, n + 1, (b,), generator=torch.Generator().manual_seed(seed))
    values[:4] = torch.tensor([0, 1, n, n - 1])
    return values.to(torch.int32).to(DEV)


def pad_with_nan(lens, *ts):
    for t in ts:
        t[torch.arange(t.shape[1], device=DEV)[None, :] >= lens[:, None]] = math.nan


def call(q, k, v, do, window, ql, kl):
    out, lse = B.gs_attention_forward(q, k, v, window=window, q_lens=ql, k_lens=kl)
    return out, lse, *B.gs_attention_backward(do, q, k, v, out, lse, window=window, q_lens=ql, k_lens=kl)


def run(q, k, v, do, window, ql=None, kl=None, sample=24):
    """All sequences at once; a sample of them against the definition."""
    b, scale = q.shape[0], q.shape[3] ** -0.5
    got = call(q, k, v, do, window, ql, kl)
    some = torch.unique(torch.linspace(0, b - 1, min(b, sample)).round().long()).to(DEV)
    pick = lambda t: None if t is None else t[some]      # noqa: E731
    r = reference(pick(q), pick(k), pick(v), scale, window, pick(ql), pick(kl), pick(do))
    for name, t in zip(("out", "lse", "dq", "dk", "dv"), got):
        check(t[some], r, name)
    return got


def in_chunks(q, k, v, do, window, ql, kl, chunk):
    """The same in calls of `chunk` sequences: nothing that a sequence gets may depend on the others of its call."""
    cut = lambda t, i: None if t is None else t[i:i + chunk]      # noqa: E731
    parts = [call(*(cut(t, i) for t in (q, k, v, do)), window, cut(ql, i), cut(kl, i)) for i in range(0, q.shape[0], chunk)]
    return [torch.cat(p) for p in zip(*parts)]


@pytest.mark.parametrize("d,row", [(33, None), (64, None), (64, 65), (96, None), (128, None), (128, 132)])
@pytest.mark.parametrize("n", [65, 96, 97, 100, 127, 128])
def test_whole_heads_of_fp32_backward(n, d, row):
    b = 90                                                 # 180 key/value heads: more than there are SMs
    for seed, (window, hq, ragged) in enumerate(((CAUSAL, 2, True), (ALL, 4, False), ((10, 10), 2, True))):
        q, k, v, do = tensors(b, n, n, hq, 2, d, F32, seed=n + seed, row=row)
        m = None
        if ragged:
            m = lengths(b, n, n + d)
            pad_with_nan(m, q, k, v, do)
        run(q, k, v, do, window, m, m)


@pytest.mark.parametrize("lq,lk", [(70, 128), (128, 70)])
def test_whole_heads_of_fp32_backward_with_unequal_lengths(lq, lk):
    b = 90
    q, k, v, do = tensors(b, lq, lk, 2, 2, 64, F32, seed=lq)
    ql, kl = lengths(b, lq, 1), lengths(b, lk, 2)
    run(q, k, v, do, CAUSAL, ql, kl)


@pytest.mark.parametrize("dt", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("hq,hk", [(4, 2), (3, 1), (2, 2)])
@pytest.mark.parametrize("n,d,window", [(12, 16, (5, 5)), (24, 64, CAUSAL), (40, 32, (10, 10)), (40, 128, CAUSAL), (100, 16, ALL)])
def test_blocks_that_go_through_many_heads(n, d, window, hq, hk, dt):
    b = (6000 if n < 100 else 2500) // hk + 3
    for ragged in (False, True):
        q, k, v, do = tensors(b, n, n, hq, hk, d, dt, seed=n + d)
        do = (do * torch.logspace(-3, 1, b, base=2.0, device=DEV)[:, None, None, None]).to(dt)      # scales that differ from head to head
        m = None
        if ragged:
            m = lengths(b, n, n + d)
            pad_with_nan(m, q, k, v, do)
        got = run(q, k, v, do, window, m, m)
        # fp32 heads of few sequences go to other kernels; everything else has to agree to the last bit
        if dt != F32:
            assert all(torch.equal(x, y) for x, y in zip(got, in_chunks(q, k, v, do, window, m, m, 200)))


@pytest.mark.parametrize("dt", [F16, BF16], ids=["f16", "bf16"])
def test_many_unequal_lengths_with_shared_heads(dt):
    b, lq, lk = 3000, 30, 50
    q, k, v, do = tensors(b, lq, lk, 4, 2, 64, dt, seed=1)
    ql, kl = lengths(b, lq, 1), lengths(b, lk, 2)
    pad_with_nan(ql, q, do)
    pad_with_nan(kl, k, v)
    got = run(q, k, v, do, CAUSAL, ql, kl)
    assert all(torch.equal(x, y) for x, y in zip(got, in_chunks(q, k, v, do, CAUSAL, ql, kl, 200)))
