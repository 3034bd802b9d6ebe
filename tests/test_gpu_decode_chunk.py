"""Several columns at once (skd_decode_chunk) and caches of 8 bits (SKD_BF16_KV8) against the decoder in float64 and against the
columns one by one."""
import numpy as np
import pytest
import torch

import decoder_reference as D
import kv_reference as R
import synth_inputs as S
from paper_2307_02628_amd import skd

pytestmark = pytest.mark.gpu
WIDE = S.ModelShape(L=3, d=256, H=2, f=544, V=777, max_pos=128)       # heads of 128, an FFN that no tile of 64 divides
NARROW = S.ModelShape(L=4, d=192, H=3, f=384, V=500, max_pos=400)     # heads of 64
BIG = S.ModelShape(L=2, d=1024, H=8, f=2048, V=1000, max_pos=256)
BAR = 2e-2  # of the range of the logits: the bar of this repository's bf16 path


def weights(shape, seed):
    w = S.weights_to_bf16_values(S.make_weights(shape, seed))
    w["wqkv"] = [a * 4 for a in w["wqkv"]]                             # scores that decide something
    return S.weights_to_bf16_values(w)


def off(got, ref):
    got = np.asarray(got, dtype=np.float64)
    return np.abs(got - ref).max() / (ref.max() - ref.min())


class Run:
    def __init__(self, shape, B, P, N, n_min, n_max, warmup=0, dtype=skd.BF16, io=0, ragged=False, seed=1, page=0):
        self.shape, self.B, self.P, self.N, self.io = shape, B, P, N, io
        self.w = weights(shape, seed)
        g = np.random.default_rng(seed)
        self.tokens = g.integers(0, shape.V, size=(B, N), dtype=np.int32)
        self.start = np.concatenate([[0], g.integers(0, P, size=B - 1)]) if ragged else np.zeros(B, dtype=int)
        self.mask = (np.arange(P)[None] >= self.start[:, None]).astype(np.uint8) if ragged else None
        self.cfg = skd.make_config(shape, B, P, N, n_min, n_max, warmup, dtype, page, io)
        self.warmup = warmup
        self.depth = [skd.skd_schedule(t, P, N, n_min, n_max, shape.L) for t in range(N)]
        self.dec = skd.Decoder(self.cfg, self.w)
        self.prefill()

    def prefill(self):
        self.dec.prefill(torch.from_numpy(self.tokens[:, :self.P].T.copy()).cuda() if self.io else self.tokens[:, :self.P].copy(), self.mask)

    def chunk(self, t, cols):
        c = self.tokens[:, t:t + cols]
        self.dec.decode_chunk(t, torch.from_numpy(c.T.copy()).cuda() if self.io else c.copy())

    def step(self, t):
        self.dec.decode_step(t, torch.from_numpy(self.tokens[:, t].copy()).cuda() if self.io else self.tokens[:, t].copy())

    def logits(self):
        if not self.io:
            return self.dec.logits_argmax()[1]
        z = torch.zeros(self.B, self.shape.V, device="cuda")
        self.dec.logits_argmax_device(None, z)
        self.dec.synchronize()
        return z.cpu().numpy()

    def reference(self, kv8=False, upto=None):
        n = upto or self.N
        return D.logits(self.shape, self.w, self.tokens[:, :n], self.depth, self.warmup, self.start, kv8, self.P - 1)

    def kv_lens(self):
        return [self.dec.kv_len(l) for l in range(self.shape.L)]


CHUNKS = [
    # shape, B, P, N, n_min, n_max, warmup, ragged, chunks (None: one step)
    (WIDE, 1, 5, 40, 1, 3, 0, False, [1, 7, None, 26]),
    (WIDE, 5, 9, 60, 1, 3, 0, True, [20, None, None, 29]),
    (NARROW, 3, 33, 120, 2, 4, 1, True, [87]),
    (NARROW, 2, 4, 90, 1, 4, 1, False, [2, 80]),                       # the last columns run the warm-up layer alone
    (NARROW, 17, 40, 80, 2, 3, 0, True, [39, None]),
    (BIG, 2, 16, 160, 1, 2, 0, False, [128, 5]),
]


@pytest.mark.parametrize("dtype", [skd.BF16, skd.BF16_KV8])
@pytest.mark.parametrize("case", CHUNKS, ids=lambda c: f"d{c[0].d}B{c[1]}P{c[2]}")
def test_chunks(case, dtype):
    shape, B, P, N, n_min, n_max, warmup, ragged, chunks = case
    kv8 = dtype == skd.BF16_KV8
    r = Run(shape, B, P, N, n_min, n_max, warmup, dtype, ragged=ragged)
    t, at = P, [P - 1]
    got = [r.logits()]
    for c in chunks:
        r.step(t) if c is None else r.chunk(t, c)
        t += c or 1
        at.append(t - 1)
        got.append(r.logits())
        # a layer holds the columns that it was active at
        active = [sum(1 for i in range(t) if l < warmup or l >= shape.L - (r.depth[i] - warmup)) for l in range(shape.L)]
        assert r.kv_lens() == active
    ref, cache = r.reference(kv8, t)
    # 8 bits: where a key differs by one bf16 step from the reference's, its code may too; that moves the logits by no more than
    # the rounding to 8 bits itself does
    bar = BAR + (off(D.logits(shape, r.w, r.tokens[:, :t], r.depth, warmup, r.start, False, P - 1)[0], ref) if kv8 else 0.0)
    for i, z in zip(at, got):
        assert off(z, ref[i - (P - 1)]) <= bar
    for l in range(shape.L):
        n = r.kv_lens()[l]
        for b in range(B):
            k, v = r.dec.kv_read(l, b)
            for x, y in ((k, cache[l][0]), (v, cache[l][1])):
                y = y[b, r.start[b]:n]
                assert x.shape[0] == n and off(x[r.start[b]:], y) <= (bar + 2.0 ** -4 if kv8 else bar)  # a step of e4m3
    r.dec.close()


@pytest.mark.parametrize("io", [0, 1])
@pytest.mark.parametrize("dtype", [skd.BF16, skd.FP32, skd.BF16_KV8])
def test_chunk_then_back_and_on(dtype, io):
    """Host and device buffers; columns taken back and processed again give the same logits; steps go on behind a chunk."""
    r = Run(NARROW, 4, 12, 60, 1, 4, 0, dtype, io, ragged=True)
    r.chunk(12, 20)
    first = r.logits()
    r.dec.rewind(12)
    r.chunk(12, 20)
    assert np.array_equal(first, r.logits())
    r.dec.rewind(20)
    for t in range(20, 32):
        r.step(t)
    assert off(r.logits(), first) <= BAR
    one_by_one = r.logits()
    r.step(32)
    behind = r.logits()
    r.dec.rewind(32)
    r.chunk(32, 1)
    assert off(r.logits(), behind) <= BAR
    assert off(one_by_one, r.reference(dtype == skd.BF16_KV8, 32)[0][-1]) <= 2 * BAR
    r.prefill()                                                        # a new generation in the same state
    r.chunk(12, 20)
    assert np.array_equal(first, r.logits())
    r.dec.close()


def test_more_rows_than_fit_at_once():
    r = Run(NARROW, 128, 4, 60, 1, 4, 0, skd.BF16, 1, ragged=True)
    r.chunk(4, 50)                                                     # 6400 rows: two parts
    z = r.logits()
    r.dec.rewind(4)
    r.chunk(4, 32)
    r.chunk(36, 18)
    assert np.array_equal(z, r.logits())
    ref = r.reference(False, 54)[0][-1]
    assert off(z, ref) <= BAR
    r.dec.close()


def test_refusals():
    r = Run(WIDE, 2, 5, 20, 1, 3)
    tok = r.tokens[:, 5:9].copy()
    assert skd.lib().skd_decode_chunk(None, 5, 1, tok.ctypes.data) == skd.ERR_NULL
    assert skd.lib().skd_decode_chunk(r.dec._h, 5, 1, None) == skd.ERR_NULL
    assert r.dec.decode_chunk_rc(6, tok) == skd.ERR_ORDER and r.dec.decode_chunk_rc(4, tok) == skd.ERR_ORDER
    assert r.dec.decode_chunk_rc(17, tok) == skd.ERR_RANGE and r.dec.decode_chunk_rc(-1, tok) == skd.ERR_RANGE
    assert skd.lib().skd_decode_chunk(r.dec._h, 5, 0, tok.ctypes.data) == skd.ERR_RANGE
    bad = tok.copy()
    bad[1, 3] = WIDE.V
    before = r.kv_lens()
    assert r.dec.decode_chunk_rc(5, bad) == skd.ERR_RANGE and r.kv_lens() == before
    assert r.dec.decode_chunk_rc(5, tok) == skd.OK
    with pytest.raises(ValueError):
        r.dec.decode_chunk(9, tok[:1])
    fresh = skd.Decoder(r.cfg, r.w)
    assert fresh.decode_chunk_rc(5, tok) == skd.ERR_ORDER
    fresh.close()
    r.dec.close()


@pytest.mark.parametrize("shape,B,P,ragged", [(WIDE, 3, 40, True), (NARROW, 2, 20, False), (BIG, 8, 128, True)], ids=["wide", "narrow", "big"])
def test_what_8_bits_hold(shape, B, P, ragged):
    """Keys and values of the first layer are the bf16 state's, rounded; pages take the bytes that they should; and the cache can be
    set from arrays."""
    N = P + 12
    a, b = (Run(shape, B, P, N, shape.L, shape.L, 0, t, ragged=ragged) for t in (skd.BF16, skd.BF16_KV8))
    for t in range(P, P + 4):
        a.step(t)
        b.step(t)
    for row in range(B):
        for x, y in zip(a.dec.kv_read(0, row), b.dec.kv_read(0, row)):
            x = x.reshape(len(x), shape.H, -1).astype(np.float64)
            s = a.start[row]
            np.testing.assert_array_equal(R.as_held(x, R.FP8)[s:], y.reshape(x.shape)[s:].astype(np.float64))
            assert (y[:s] == 0).all()
    assert a.dec.kv_pages() == b.dec.kv_pages()
    g = np.random.default_rng(4)
    K, V = ([D.R_round(g.standard_normal((B, P + 2, shape.d))).astype(np.float32) for _ in range(shape.L)] for _ in range(2))
    b.dec.kv_load(P + 2, K, V, b.start)
    for l in range(shape.L):
        for row in range(B):
            for x, y in zip(b.dec.kv_read(l, row), (K, V)):
                s = b.start[row]
                want = R.as_held(y[l][row].reshape(P + 2, shape.H, -1).astype(np.float64), R.FP8).reshape(P + 2, -1)
                np.testing.assert_array_equal(x[s:], want[s:])
    b.step(P + 2)
    assert np.isfinite(b.logits()).all()
    a.dec.close()
    b.dec.close()


def test_8_bits_one_column_at_a_time(monkeypatch):
    """The prompt column by column, padding columns among them, and a table that decays inside it."""
    r = Run(NARROW, 3, 20, 40, 2, 4, 0, skd.BF16_KV8, ragged=True)
    z = r.logits()
    monkeypatch.setenv("SKD_PREFILL_BATCHED", "0")
    s = Run(NARROW, 3, 20, 40, 2, 4, 0, skd.BF16_KV8, ragged=True)
    assert off(s.logits(), z) <= 2 * BAR
    for x in (r, s):
        x.dec.close()


def test_heads_of_a_state_with_8_bits():
    r = Run(WIDE, 3, 7, 30, 1, 3, 0, skd.BF16_KV8, io=1)
    tok, z = (torch.zeros(3, dtype=torch.int32, device="cuda") for _ in range(2)), torch.zeros(3, WIDE.V, device="cuda")
    t0, t1 = tok
    r.chunk(7, 9)
    r.dec.logits_argmax_device(t0, z)
    assert r.dec.logits_argmax_noalloc_rc(t1, None) == skd.OK
    r.dec.synchronize()
    assert torch.equal(t0, t1) and torch.equal(t0.long(), z.argmax(-1))
    u = torch.tensor([0.1, 0.5, 0.9], device="cuda")
    r.dec.logits_sample_rows_device(u, torch.full((3,), 0.7, device="cuda"), torch.full((3,), 20, dtype=torch.int32, device="cuda"), tokens_out=t0)
    r.dec.decode_step(16, None)
    r.dec.profile_enable(1)
    r.step(17)
    assert r.dec.profile_read()["attention"]["launches"] >= r.depth[17]
    r.dec.close()
