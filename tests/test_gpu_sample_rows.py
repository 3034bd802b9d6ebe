"""Draws with parameters per row (skd_sample, skd_logits_sample_rows) against 64 bits on the CPU."""
import math

import numpy as np
import pytest
import torch

import synth_inputs as S
from paper_2307_02628_amd import skd

pytestmark = pytest.mark.gpu


def reference(z, u, t=1.0, k=0, p=1.0, m=0.0):
    """The token of one row.  Masses are rounded to units of 2^-45 as documented (so that u = 0 draws no token without one); sums
    and comparisons are in float64: a draw could come out otherwise only where u * mass lies within about 2^-45 * len(z) of a
    running mass, which no test here does by chance (2^-27 at 2^18 tokens)."""
    z = np.where(np.isnan(z), -np.inf, z).astype(np.float64)
    top = z.max()
    if not np.isfinite(top) or not t > 0:
        return int(np.argmax(z)) if top > -np.inf else 0
    w = np.exp((z - top) / t)
    keep = z > -np.inf
    if m > 0:
        keep &= w >= min(m, 1.0)
    w = np.round(w * 2.0 ** 45)
    if 0 < k < len(z):
        keep &= z >= np.sort(z)[-k]
    if p < 1:
        order = np.sort(z[keep])[::-1]
        mass = np.cumsum(np.exp((order - top) / t))
        keep &= z >= order[min(int((mass < max(p, 0.0) * mass[-1]).sum()), len(order) - 1)]
    run = np.cumsum(np.where(keep, w, 0.0))
    return int((run <= float(u) * run[-1]).sum())


def draw(z, u, **params):
    t = {n: None if a is None else torch.as_tensor(a, dtype=torch.int32 if n == "top_k" else torch.float32).cuda() for n, a in params.items()}
    out = torch.full((z.shape[0],), -5, dtype=torch.int32, device="cuda")
    ws = torch.full((skd.sample_workspace(*z.shape),), 0xff, dtype=torch.uint8, device="cuda")
    skd.sample(z, torch.as_tensor(u, dtype=torch.float32).cuda(), out, **t, workspace=ws)
    return out.cpu().numpy()


def check(z, u, **params):
    zz, u = z.cpu().numpy(), np.float32(u)
    got = draw(z, u, **params)
    col = {n: np.float32(a) if n != "top_k" else np.int64(a) for n, a in params.items() if a is not None}
    names = {"temperature": "t", "top_k": "k", "top_p": "p", "min_p": "m"}
    for b in range(len(zz)):
        want = reference(zz[b], u[b], **{names[n]: float(a[b]) if n != "top_k" else int(a[b]) for n, a in col.items()})
        assert got[b] == want, (b, got[b], want, float(u[b]), {n: a[b] for n, a in col.items()})


def some(B, V, spread, seed):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(B, V, generator=g) * spread
    z[::2] = z[::2].bfloat16().float()
    r = torch.rand(5, B, generator=g).numpy()
    return z.cuda(), r


@pytest.mark.parametrize("V", [1, 2, 63, 256, 257, 1000, 4097, 50272, 131072, 262144])
@pytest.mark.parametrize("spread", [0.3, 3.0])
def test_every_filter(V, spread):
    B = 12
    z, r = some(B, V, spread, V)
    u = r[0]
    u[0], u[1] = 0.0, np.float32(1) - np.float32(2) ** -24
    t = 0.2 + r[1]
    k = np.array([0, 1, 2, 5, 40, 1000, V, V - 1, 3 * V, 0, 7, V // 2])
    p = np.array([1.0, 0.5, 0.999, 0.9, 1.0, 0.7, 0.01, 1.0, 0.6, 0.95, 1e-6, 0.99])
    m = np.array([0.0, 0.0, 0.5, 0.05, 0.0, 0.01, 0.0, 1.0, 1e-9, 0.1, 0.0, 0.0])
    check(z, u)
    check(z, u, temperature=t)
    check(z, u, temperature=t, top_k=k)
    check(z, u, temperature=t, top_p=p)
    check(z, u, temperature=t, min_p=m)
    check(z, u, temperature=t, top_k=k, top_p=p, min_p=m)
    check(z, u, top_k=k, top_p=p)


def test_equal_logits():
    """More equal logits than any list of candidates holds; the tied ones all stay in."""
    z = torch.zeros(6, 9000, device="cuda")
    z[1, 5000:] = -1.0
    z[2, ::3] = 1.0
    z[3, 0] = -0.0
    z[4] = -7.25
    z[5, 8999] = 2.0 ** -20
    u = [0.0, 0.9999, 0.5, 0.1, 0.73, 0.2]
    check(z, u, top_k=[1, 4999, 2999, 1, 5, 2])
    check(z, u, top_p=[0.1, 0.3, 0.2, 0.9, 0.5, 1e-4])
    check(z, u, temperature=[0.5] * 6, top_k=[1, 6000, 3001, 1, 5, 2], top_p=[0.1, 0.3, 0.2, 0.9, 0.5, 1e-4])


def test_values_that_are_not_finite():
    inf, nan = math.inf, math.nan
    z = torch.randn(9, 700, generator=torch.Generator().manual_seed(2))
    z[0, 13:] = -inf
    z[1] = -inf
    z[2, 99] = inf
    z[2, 100] = inf
    z[3] = nan
    z[4, ::2] = nan
    z[5, :699] = -inf
    z[6, 5], z[6, 6] = inf, nan
    z[7, 3] = 3.4e38
    z[7, 4] = -3.4e38
    z[8] *= 1e-42
    z = z.cuda()
    for kw in ({}, dict(top_k=[3] * 9), dict(top_p=[0.8] * 9), dict(min_p=[0.2] * 9), dict(top_k=[50] * 9, top_p=[0.9] * 9, min_p=[0.01] * 9)):
        check(z, [0.6] * 9, **kw)
        check(z, [0.6] * 9, temperature=[0.7] * 9, **kw)


@pytest.mark.parametrize("t", [0.0, 1e-30, 1e-3, 50.0, 1e30])
def test_temperatures(t):
    z, r = some(7, 3001, 2.0, 5)
    check(z, r[0], temperature=[t] * 7)
    check(z, r[0], temperature=[t] * 7, top_p=[0.8] * 7)
    check(z, r[0], temperature=[t] * 7, top_k=[20] * 7, min_p=[0.001] * 7)


@pytest.mark.parametrize("t", [1e-37, 1e-30, 1e-3, 1.0, 3e38, math.inf])
@pytest.mark.parametrize("offset", [-3e38, -1e10, -700.0, 1e4, 1e10])
def test_logits_far_from_zero(offset, t):
    """Places on the grid of bins that overflow, that are not distinct, or that are all the same."""
    z, r = some(4, 5003, 2.0, 15)
    z = z + offset
    check(z, r[0], temperature=[t] * 4)
    check(z, r[0], temperature=[t] * 4, top_p=[0.8, 0.3, 0.99, 0.0])
    check(z, r[0], temperature=[t] * 4, top_k=[20, 1, 3000, 5003], min_p=[0.001] * 4)
    check(z, r[0], temperature=[t] * 4, top_p=[0.8] * 4, min_p=[0.5] * 4)


@pytest.mark.parametrize("levels", [2, 40, 4000])
def test_long_lists_of_few_values(levels):
    """Thresholds among more tokens than are listed, and buckets with many equal ones."""
    B, V = 8, 100003
    g = torch.Generator().manual_seed(levels)
    z = (torch.randint(0, levels, (B, V), generator=g).float() / levels * 0.5).cuda()
    u = torch.rand(B, generator=g).numpy()
    k = np.array([0, 1, 9000, 50000, 99999, 8192, 8193, 3])
    p = np.array([0.5, 1.0, 0.9, 0.99, 0.05, 1.0, 0.3, 0.7])
    m = np.array([0.0, 0.0, 0.0, 0.5, 0.8, 0.9, 0.7, 0.99])
    check(z, u, top_k=k)
    check(z, u, top_p=p)
    check(z, u, min_p=m)
    check(z, u, top_k=k, top_p=p, min_p=m)
    check(z, u, temperature=[0.01] * B, top_k=k, top_p=p, min_p=m)


def test_values_outside_their_ranges():
    z, _ = some(6, 500, 2.0, 6)
    nan = math.nan
    u = [0.5] * 6
    off = draw(z, u)
    assert (draw(z, u, top_k=[-3] * 6, top_p=[2.0, nan, 1.0, 5.0, nan, 1.5], min_p=[-1.0, nan, 0.0, -0.5, nan, 0.0]) == off).all()
    best = z.argmax(-1).cpu().numpy()
    assert (draw(z, u, temperature=[-1.0, nan, 0.0, -2.0, nan, 0.0]) == best).all()
    assert (draw(z, u, top_p=[0.0, -1.0] * 3) == best).all() and (draw(z, u, min_p=[1.0, 2.0] * 3) == best).all()
    assert (draw(z, [-1.0, nan, -math.inf] * 2) == draw(z, [0.0] * 6)).all()
    assert (draw(z, [1.0, 2.0, math.inf] * 2) == draw(z, [float(np.float32(1) - np.float32(2) ** -24)] * 6)).all()


def test_strided_rows_and_rows_that_are_not_aligned():
    flat = torch.randn(5 * 1003 + 1, generator=torch.Generator().manual_seed(8)).cuda() * 2
    z = flat[1:].view(5, 1003)[:, :1001]
    u = torch.rand(5, generator=torch.Generator().manual_seed(9)).numpy()
    check(z, u, temperature=[0.6] * 5, top_k=[50] * 5, top_p=[0.9] * 5)
    assert skd.sample_workspace(5, 1003) >= 0


def test_captured_and_replayed():
    z, r = some(9, 20000, 2.0, 12)
    t, k, p, u = (torch.zeros(9, dtype=d, device="cuda") for d in (torch.float32, torch.int32, torch.float32, torch.float32))
    out = torch.zeros(9, dtype=torch.int32, device="cuda")
    ws = torch.empty(skd.sample_workspace(9, 20000), dtype=torch.uint8, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        skd.sample(z, u, out, t, k, p, workspace=ws, stream=torch.cuda.current_stream().cuda_stream)
    for step in range(4):
        gen = torch.Generator().manual_seed(step)
        z.copy_(torch.randn(9, 20000, generator=gen) * (1 + step))
        for x, lo, hi in ((t, 0.2, 1.2), (p, 0.5, 1.0), (u, 0.0, 1.0)):
            x.copy_(lo + (hi - lo) * torch.rand(9, generator=gen))
        k.copy_(torch.randint(0, 60, (9,), generator=gen))
        g.replay()
        torch.cuda.synchronize()
        want = draw(z, u.cpu(), temperature=t.cpu(), top_k=k.cpu(), top_p=p.cpu())
        assert (out.cpu().numpy() == want).all()
        check(z, u.cpu().numpy(), temperature=t.cpu(), top_k=k.cpu(), top_p=p.cpu())


@pytest.mark.parametrize("dtype", [skd.BF16, skd.FP32])
@pytest.mark.parametrize("io", [0, 1])
def test_head_of_a_state(dtype, io):
    """skd_logits_sample_rows draws from the logits that it returns, and the generation goes on from the tokens."""
    shape, B, P = S.ModelShape(L=2, d=256, H=4, f=512, V=1003, max_pos=16), 5, 4
    w = S.weights_to_bf16_values(S.make_weights(shape, 3))
    w["tok_emb"] = w["tok_emb"] * 16
    cfg = skd.make_config(shape, B, P, 12, 1, 2, dtype=dtype, io_on_device=io)
    g = np.random.default_rng(1)
    params = dict(temperature=g.uniform(0.3, 1.2, B).astype(np.float32), top_k=np.array([0, 5, 100, 0, 1], dtype=np.int32),
                  top_p=np.array([0.7, 1.0, 0.9, 1.0, 0.5], dtype=np.float32), min_p=np.array([0, 0.05, 0, 0.1, 0], dtype=np.float32))
    prompts = S.make_prompts(B, P, shape.V, 2)
    with skd.Decoder(cfg, w) as dec:
        assert skd.lib().skd_logits_sample_rows(dec._h, 1 << 20, None, None, None) == skd.ERR_ORDER
        dec.prefill(torch.from_numpy(np.ascontiguousarray(prompts.T)).cuda() if io else prompts)
        for step in range(3):
            u = g.random(B, dtype=np.float32).clip(0, 0.999)
            use = params if step else {}
            if io:
                dev = {n: torch.from_numpy(a).cuda() for n, a in use.items()}
                tok, lg = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, shape.V, device="cuda")
                dec.logits_sample_rows_device(torch.from_numpy(u).cuda(), **dev, tokens_out=tok, logits_out=lg)
                dec.synchronize()
                tok, lg = tok.cpu().numpy(), lg.cpu().numpy()
            else:
                tok, lg = dec.logits_sample_rows(u, **use)
            for b in range(B):
                a = {n: x[b] for n, x in use.items()}
                assert tok[b] == reference(lg[b], u[b], a.get("temperature", 1.0), int(a.get("top_k", 0)), a.get("top_p", 1.0), a.get("min_p", 0.0))
            dec.decode_step(P + step, None)
        if not io:
            bad = dict(temperature=-1.0, top_k=-1, top_p=0.0, min_p=1.5)
            dec.logits_argmax()
            for n, x in bad.items():
                a = {m: y.copy() for m, y in params.items()}
                a[n][3] = x
                assert dec.logits_sample_rows_rc(np.zeros(B), **a)[0] == skd.ERR_RANGE
            assert dec.logits_sample_rows_rc(np.full(B, 1.0))[0] == skd.ERR_RANGE
            assert dec.logits_sample_rows_rc(np.full(B, 0.5), **params)[0] == skd.OK
