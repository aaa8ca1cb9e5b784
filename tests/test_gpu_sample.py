"""lapsum_sample against the definition in 64 bits, token for token."""
import numpy as np
import pytest
import torch

import paper_2608_06912_b200 as L
from tests.dense_util import sample_reference

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def check(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, by_row=True):
    rows = logits.shape[0]
    full = {}
    for name, v, dt in (("temperature", temperature, torch.float32), ("top_k", top_k, torch.int32), ("top_p", top_p, torch.float32),
                        ("min_p", min_p, torch.float32)):
        full[name] = torch.as_tensor(v, dtype=dt, device="cuda").expand(rows).contiguous()
    token, kept = (torch.full((rows,), -7, device="cuda", dtype=torch.int32) for _ in range(2))
    logprob = torch.full((rows,), 7.0, device="cuda")
    params = L.sample_params(io_dtype=L.IO_OF[logits.dtype])
    if by_row:
        L.lapsum_sample(logits, u, params, token, logprob, kept, **full)
    else:
        for name in full:
            setattr(params, name, full[name][0].item())
        L.lapsum_sample(logits, u, params, token, logprob, kept)
    t, lp, n = sample_reference(logits, u.cpu(), *(full[name].cpu() for name in ("temperature", "top_k", "top_p", "min_p")))
    assert np.array_equal(token.cpu().numpy(), t), (token.cpu().numpy()[token.cpu().numpy() != t], t[token.cpu().numpy() != t])
    assert np.array_equal(kept.cpu().numpy(), n)
    # the sum of all weights is off by at most vocab 2^-46 of the largest weight, the result by one rounding to fp32
    got = logprob.cpu().numpy().astype(np.float64)
    ok = np.isfinite(lp)
    assert np.array_equal(np.isnan(got), np.isnan(lp)) and np.array_equal(got[~ok & ~np.isnan(lp)], lp[~ok & ~np.isnan(lp)])
    assert np.all(np.abs(got - lp)[ok] <= 2.0 ** -24 * np.abs(lp[ok]) + logits.shape[1] * 2.0 ** -46 + 1e-13)
    return token, logprob, kept


def make(rows, vocab, dtype="f32", seed=0, spread=2.0, device="cuda"):
    gen = torch.Generator(device=device).manual_seed(seed)
    x = spread * torch.randn(rows, vocab, device=device, generator=gen)
    return x.to(DT[dtype]), torch.rand(rows, device=device, generator=gen)


def settings(rows, seed):
    rng = np.random.default_rng(seed)
    pick = lambda v: torch.tensor(rng.choice(v, rows))  # noqa: E731
    return dict(temperature=pick([0.0, 0.2, 0.7, 1.0, 1.5, 40.0]), top_k=pick([0, 1, 2, 7, 50, 300, 5000]), top_p=pick([1.0, 0.99, 0.9, 0.4, 1e-6]),
                min_p=pick([0.0, 0.0, 0.01, 0.3, 1.0]))


@pytest.mark.parametrize("vocab", [1, 2, 3, 31, 128, 129, 1000, 4097, 32001])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_rows_with_settings_of_their_own(vocab, dtype):
    rows = 40
    x, u = make(rows, vocab, dtype, seed=vocab)
    check(x, u, **settings(rows, vocab))


@pytest.mark.parametrize("rows,vocab,dtype", [(1, 131073, "f32"), (3, 262144, "bf16"), (1, 700001, "f32"), (2, 500000, "f32"), (300, 20000, "f32")])
def test_long_rows_and_many_rows(rows, vocab, dtype):
    x, u = make(rows, vocab, dtype, seed=rows)
    check(x, u, **settings(rows, rows))
    check(x, u, top_p=0.95)
    check(x, u)


@pytest.mark.parametrize("kw", [{}, dict(top_k=40), dict(top_p=0.9), dict(min_p=0.05), dict(top_k=600), dict(top_p=0.999),
                                dict(top_k=100, top_p=0.8, min_p=0.001, temperature=1.7), dict(temperature=0.0)])
def test_each_filter(kw):
    x, u = make(24, 50021, seed=3)
    a = check(x, u, **kw)
    b = check(x, u, by_row=False, **kw)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("vocab", [900, 30000])
@pytest.mark.parametrize("kw", [dict(top_k=17), dict(top_k=700), dict(top_p=0.5), dict(top_k=501, top_p=0.37), {}, dict(min_p=1.0), dict(temperature=0.0)])
def test_equal_logits_rank_by_index(vocab, kw):
    u = torch.rand(6, device="cuda", generator=torch.Generator(device="cuda").manual_seed(vocab))
    x = torch.zeros(6, vocab, device="cuda")
    x[1] = -0.0
    x[2, ::2] = -0.0                       # -0 and 0 are equal
    x[3, ::3] = 1.0                        # two values
    x[4] = torch.arange(vocab, device="cuda").remainder(5).float()
    x[5] = -1e30
    check(x, u, **kw)


def test_masks_infinities_and_nan():
    vocab = 5000
    x, u = make(12, vocab, seed=9)
    inf, nan, low = float("inf"), float("nan"), torch.finfo(torch.float32).min
    x[0] = -inf
    x[1] = nan
    x[2, 1:] = -inf
    x[3, :vocab - 1] = nan
    x[4, ::2] = -inf
    x[5, ::2] = low                        # a mask of the type's lowest value
    x[6] = low
    x[7, 17] = inf
    x[8, 17], x[8, 40], x[8, 4000] = inf, inf, inf
    x[9, ::3] = nan
    x[10] = low
    x[10, 77] = 3.0
    x[11, :10] = 3e38
    for kw in ({}, dict(top_k=3), dict(top_p=0.7), dict(top_k=4000, top_p=0.9), dict(min_p=0.2), dict(temperature=0.0), dict(top_k=2, top_p=0.3)):
        check(x, u, **kw)
    y = torch.where(x.isfinite(), x.clamp(-6e4, 6e4), x).half()
    y[5, ::2] = torch.finfo(torch.float16).min
    check(y, u, top_k=9, top_p=0.9)


def test_settings_out_of_range_void_their_row_alone():
    x, u = make(12, 300, seed=4)
    nan, inf = float("nan"), float("inf")
    t, k = torch.ones(12), torch.zeros(12, dtype=torch.int32)
    p, m = torch.ones(12), torch.zeros(12)
    t[0], t[1], t[2], p[3], p[4], m[5], m[6], m[7] = -1.0, nan, inf, 0.0, nan, 1.5, -0.1, nan
    u[8], u[9], u[10] = 1.0, -0.5, nan
    k[11] = -5
    token, logprob, kept = check(x, u, t, k, p, m)
    assert (token[:11] == -1).all() and token[11] >= 0 and kept[11] == 300


@pytest.mark.parametrize("temperature", [1e-30, 1e-3, 0.05, 30.0, 1e6])
def test_extreme_temperatures(temperature):
    x, u = make(10, 9000, seed=12)
    for kw in ({}, dict(top_k=25), dict(top_p=0.6), dict(top_k=3000, top_p=0.9), dict(min_p=0.5)):
        check(x, u, temperature=temperature, **kw)


def test_a_temperature_whose_reciprocal_is_infinite():
    x, u = make(5, 2000, seed=14)
    token, kept = (torch.full((5,), -7, device="cuda", dtype=torch.int32) for _ in range(2))
    for kw in (dict(min_p=0.5), dict(top_p=0.5), dict(top_k=9, min_p=1.0), {}):
        L.lapsum_sample(x, u, L.sample_params(temperature=1e-310, **kw), token, None, kept)
        assert torch.equal(token.long(), x.argmax(1)), kw
        if kw:
            assert (kept == 1).all() or "top_k" in kw


@pytest.mark.parametrize("scale,shift", [(1e-6, 0.0), (1e-3, 1000.0), (1e4, 0.0), (1.0, -1e5), (1e30, 0.0)])
def test_logits_of_any_size(scale, shift):
    x, u = make(8, 20000, seed=13)
    x = x * scale + shift
    for kw in (dict(top_k=50), dict(top_p=0.9), dict(top_k=5000, top_p=0.99)):
        check(x, u, **kw)


@pytest.mark.parametrize("offset,stride", [(0, 1001), (1, 1003), (3, 1024), (8, 1008)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_of_any_stride_and_alignment(offset, stride, dtype):
    vocab, rows = 1000, 9
    gen = torch.Generator(device="cuda").manual_seed(offset)
    buf = (2 * torch.randn(rows * stride + offset + 64, device="cuda", generator=gen)).to(DT[dtype])
    x = buf[offset:].as_strided((rows, vocab), (stride, 1))
    check(x, torch.rand(rows, device="cuda", generator=gen), **settings(rows, offset))


def test_a_vocabulary_beyond_the_cluster_s_memory_and_tokens_at_its_ends():
    vocab = 2_000_003
    x, u = make(3, vocab, "f32", seed=21)
    check(x, u, top_p=0.9)
    check(x, u, top_k=1000)
    x[:] = -50.0
    x[0, 0], x[1, vocab - 1], x[2, vocab - 2] = 9.0, 9.0, 9.0
    check(x, u, temperature=0.0)
    check(x, u, top_k=3, top_p=0.9)


def test_the_draws_follow_the_distribution():
    """100000 draws at stratified u count every token to within one of its share"""
    rows = 100_000
    x = torch.tensor([1.0, -0.5, 2.0, float("-inf"), 0.0, 2.0], device="cuda")
    u = (torch.arange(rows, device="cuda", dtype=torch.float64) + 0.5).div(rows).float()
    token = torch.empty(rows, device="cuda", dtype=torch.int32)
    L.lapsum_sample(x.expand(rows, 6).contiguous(), u, L.sample_params(temperature=0.9), token)
    share = torch.bincount(token.long(), minlength=6).double() / rows
    want = torch.softmax(x.double() / 0.9, 0)
    assert ((share - want).abs() <= 1.5 / rows).all()


def test_results_do_not_depend_on_scheduling():
    x, u = make(64, 60000, seed=30)
    s = {k: v.cuda() if k != "top_k" else v.to(torch.int32).cuda() for k, v in settings(64, 1).items()}
    s = {k: v.float() if k != "top_k" else v for k, v in s.items()}
    outs = []
    for _ in range(3):
        o = [torch.empty(64, device="cuda", dtype=torch.int32), torch.empty(64, device="cuda"), torch.empty(64, device="cuda", dtype=torch.int32)]
        L.lapsum_sample(x, u, L.sample_params(), *o, **s)
        outs.append(o)
    assert all(torch.equal(a, b) for o in outs[1:] for a, b in zip(outs[0], o))
