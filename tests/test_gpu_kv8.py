"""The 8-bit KV cache on the GPU: the append bit for bit, attention against fp64 over the values the codes stand for."""
import types

import numpy as np
import pytest
import torch

from oracle import kv8
from paper_2410_01228_amd import binding as cs
from paper_2410_01228_amd import synth

pytestmark = pytest.mark.gpu

NAN_CODE = 0x7F          # what slots that nobody has written hold here
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


class World:
    """A batch over an 8-bit pool on the CPU, its earlier tokens appended by the oracle."""

    def __init__(self, ctx, new, Hkv, D, seed, dtype=torch.bfloat16, stride=None, layers=1, layer=0, gain=1.0, spare=5):
        self.Hkv, self.D, self.dtype, self.layer, self.layers = Hkv, D, dtype, layer, layers
        self.rng = np.random.default_rng(seed)
        self.ctx, self.new = list(ctx), list(new)
        need = [-(-(c + q) // 16) for c, q in zip(ctx, new)]
        self.P = sum(need) + spare
        perm = self.rng.permutation(self.P).astype(np.int32)
        self.tables = np.full((max(len(ctx), 1), max(need + [1])), -1, np.int32)
        o = 0
        for s, n in enumerate(need):
            self.tables[s, :n] = perm[o:o + n]
            o += n
        self.spare = perm[o:]
        self.cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.stride = kv8.page_bytes(Hkv, D) if stride is None else stride
        self.pool = np.full((layers, self.P, self.stride), NAN_CODE, np.uint8)
        cu_old = np.concatenate([[0], np.cumsum(ctx)]).astype(np.int32)
        k, v = self.rows(int(cu_old[-1]), gain), self.rows(int(cu_old[-1]), gain)
        kv8.ref_append(self.pool, layer, self.tables, np.zeros(len(ctx), np.int32), cu_old, k, v, Hkv, D, dtype == torch.float16)

    @property
    def T(self):
        return int(self.cu[-1])

    def rows(self, n, gain=1.0):
        x = self.rng.standard_normal((n, self.Hkv, self.D)) * np.exp2(self.rng.standard_normal((n, 1, 1))) * gain
        return torch.from_numpy(x).to(self.dtype).double().numpy()

    def batch(self):
        return cs.Batch(torch.from_numpy(self.tables), torch.tensor(self.ctx, dtype=torch.int32), torch.from_numpy(self.cu))

    def handle(self, t):
        return cs.Pool8(t, self.layers, self.P, self.Hkv, self.D, page_stride=self.stride)

    def append(self, k, v):
        """(the pool after the GPU's append, after the oracle's)"""
        t = torch.from_numpy(self.pool).cuda()
        k, v = (torch.from_numpy(x).to(self.dtype) for x in (k, v))             # (what either side is given)
        fn = cs.cs_kv8_append_f16 if self.dtype == torch.float16 else cs.cs_kv8_append
        fn(self.handle(t), self.layer, self.batch(), k.cuda(), v.cuda())
        want = self.pool.copy()
        kv8.ref_append(want, self.layer, self.tables, self.ctx, self.cu, k.double().numpy(), v.double().numpy(), self.Hkv, self.D, self.dtype == torch.float16)
        return t.cpu().numpy(), want


def same_codes(got, want, Hkv, D):
    """Equal bytes, any NaN code for any other."""
    codes = 2 * Hkv * 16 * D
    g, w = got.copy(), want.copy()
    for a in (g, w):
        c = a[..., :codes]
        c[(c & 127) == 127] = 127
    return np.array_equal(g, w)


APPENDS = {
    "first_and_last_slots": ([0, 15, 16, 31, 7, 100], [1] * 6),
    "one_chunk": ([0], [37]),
    "inside_a_page": ([3], [5]),
    "over_a_border": ([15, 14], [2, 3]),
    "ragged_chunks": ([0, 5, 16, 47, 1], [16, 2, 33, 100, 300]),
    "mixed_with_idle": ([20, 9, 33, 0, 50, 4], [1, 0, 1, 40, 17, 0]),
    "chunks_first": ([4, 18, 7], [21, 1, 1]),
    "nothing": ([5, 6], [0, 0]),
}


@pytest.mark.parametrize("Hkv,D", [(1, 64), (2, 64), (3, 128), (8, 128)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("name", list(APPENDS))
def test_append_is_exact(name, dtype, Hkv, D):
    w = World(*APPENDS[name], Hkv, D, 17 + Hkv, dtype)
    got, want = w.append(w.rows(w.T), w.rows(w.T))
    assert same_codes(got, want, Hkv, D)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("new", [1, 3, 20])
def test_append_raises_scales(new, D, dtype):
    """New tokens far above and far below the ones that share their blocks: every second block's scale rises, some by more
    than the codes' whole range."""
    w = World([5, 9, 12, 1], [new] * 4, 4, D, 5, dtype)
    k, v = w.rows(w.T), w.rows(w.T)
    for s, gain in enumerate((64.0, 2.0 ** -12, 2.0 ** 10, 1.0)):
        k[w.cu[s]:w.cu[s + 1], ::2] *= gain
        v[w.cu[s]:w.cu[s + 1], 1::2] *= gain
    got, want = w.append(k, v)
    assert not np.array_equal(want, w.pool) and same_codes(got, want, 4, D)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("ctx,new", [([0, 6], [1, 1]), ([0, 6], [24, 9])])
def test_append_of_zeros_infinities_and_nans(ctx, new, dtype):
    w = World(ctx, new, 2, 128, 3, dtype)
    k, v = w.rows(w.T), w.rows(w.T)
    k[0] = 0.0
    v[0, 0], v[0, 1, 5], v[0, 1, 6] = np.nan, np.inf, -np.inf
    k[-1, 1, ::3] = -np.inf
    v[-1, :, 7] = np.nan
    if dtype == torch.float16:
        k[-1, 0, 3], v[-1, 0, 4] = 65504.0, -62000.0
    else:
        k[-1, 0, 3], v[-1, 0, 4] = 3.0e38, 1e-38
    w.pool[0, :, :] = np.where((w.pool[0] & 127) == 127, 0, w.pool[0])
    got, want = w.append(k, v)
    assert same_codes(got, want, 2, 128)


def test_append_in_a_strided_layer_of_a_larger_pool():
    w = World([3, 30], [18, 1], 2, 64, 8, stride=kv8.page_bytes(2, 64) + 48, layers=3, layer=1)
    got, want = w.append(w.rows(w.T), w.rows(w.T))
    assert np.array_equal(got[::2], w.pool[::2])                       # the other layers
    assert same_codes(got, want, 2, 64)


def test_append_skips_pages_outside_the_pool():
    w = World([0, 20, 3, 40], [20, 1, 1, 7], 2, 128, 9)
    w.tables[0, 1], w.tables[1, 1], w.tables[3, 2] = -1, w.P, 2 ** 31 - 1
    got, want = w.append(w.rows(w.T), w.rows(w.T))
    assert same_codes(got, want, 2, 128)


@pytest.mark.parametrize("D", [64, 128])
def test_tokens_one_by_one_give_the_scales_of_a_chunk(D):
    """Scales do not depend on how a sequence's tokens were dealt to steps; codes only where one fell below the smallest
    normal code in between."""
    w = World([0], [40], 2, D, 12)
    k, v = w.rows(40), w.rows(40)
    chunk, _ = w.append(k, v)
    t = torch.from_numpy(w.pool).cuda()
    for i in range(40):
        b = cs.Batch(torch.from_numpy(w.tables), torch.tensor([i], dtype=torch.int32), torch.tensor([0, 1], dtype=torch.int32))
        cs.cs_kv8_append(w.handle(t), 0, b, torch.from_numpy(k[i:i + 1]).bfloat16().cuda(), torch.from_numpy(v[i:i + 1]).bfloat16().cuda())
    single = t.cpu().numpy()
    codes = 2 * 2 * 16 * D
    assert np.array_equal(single[..., codes:codes + 16], chunk[..., codes:codes + 16])
    for a, b in zip(kv8.read_logical(single, 0, w.tables[0], 40, 2, D), kv8.read_logical(chunk, 0, w.tables[0], 40, 2, D)):
        assert np.abs(a - b).max() <= 2.0 ** -9 * single[..., codes:codes + 16].copy().view(np.float32).max()


# ------------------------------------------------------------------------------- attention

def check_attention(w, G, out, q, seqs=None):
    """Every element within what the roundings on the way can make of it.  The weights and the output are rounded to
    the 16-bit type (half a step h of either; the sum is that of the rounded weights, so their errors weigh |v_j - out|); an fp16 Q may
    be scaled before the product and rounded once more (h of the score's terms, as an error of the exponent); half
    precision cannot hold weights under 2^-14 of the largest to h, 2^-25 each; scores, sums and exponentials are
    fp32, 2^-20 of the score's terms and of the result over this many terms."""
    h = HALF_STEP[w.dtype]
    Hq = w.Hkv * G
    got, qf = out.double().cpu().numpy(), q.double().cpu().numpy()
    scale = 1.0 / np.sqrt(w.D)
    for s in range(len(w.ctx)) if seqs is None else seqs:
        c, n, t0 = w.ctx[s], w.new[s], int(w.cu[s])
        if n == 0:
            continue
        K, V = kv8.read_logical(w.pool, w.layer, w.tables[s], c + n, w.Hkv, w.D)
        ref, spread, reach = kv8.attention(qf[t0:t0 + n], K, V, c, scale)
        fold = h if w.dtype == torch.float16 else 0.0
        weights = 1.01 * (h + (fold + 2.0 ** -20) * reach[..., None] * 2) * spread
        tiny = (c + n) * 2.0 ** -25 * 2 * np.abs(V).max() if w.dtype == torch.float16 else 0.0
        bound = 1.01 * (h + 2.0 ** -20) * np.abs(ref) + weights + tiny + 2.0 ** -20 * np.abs(V).max()
        err = np.abs(got[t0:t0 + n] - ref)
        assert (err <= bound).all(), "sequence %d (%d + %d keys): error %.3g where %.3g is the bound" % (
            s, c, n, err[err > bound].max(), bound[err > bound].min())
    assert Hq == out.shape[1]


def attend(w, G, q, workspace=None):
    t = torch.from_numpy(w.pool).cuda()
    b = w.batch()
    out = torch.full((w.T, w.Hkv * G, w.D), float("nan"), dtype=w.dtype, device="cuda")
    fn = cs.cs_paged_attention_mixed_kv8_f16 if w.dtype == torch.float16 else cs.cs_paged_attention_mixed_kv8
    fn(w.handle(t), w.layer, b, q, out, w.Hkv * G, 1.0 / np.sqrt(w.D), cs.workspace_for_kv8(b, w.Hkv * G, w.Hkv, w.D))
    return out


def filled(ctx, new, Hkv, D, seed, dtype=torch.bfloat16, **more):
    """A world whose new tokens are in the pool too (the oracle's append), NaN codes behind every sequence."""
    w = World(ctx, new, Hkv, D, seed, dtype, **more)
    kv8.ref_append(w.pool, w.layer, w.tables, w.ctx, w.cu, w.rows(w.T), w.rows(w.T), Hkv, D, dtype == torch.float16)
    return w


def queries(w, G, gain=1.0):
    return torch.from_numpy(w.rng.standard_normal((w.T, w.Hkv * G, w.D)) * gain).to(w.dtype).cuda()


DECODES = [0, 1, 14, 15, 16, 17, 30, 31, 32, 33, 47, 62, 63, 64, 99, 127, 128, 129, 255, 256, 700, 1023]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("Hkv,G,D", [(1, 1, 64), (2, 2, 64), (1, 16, 128), (2, 7, 128), (3, 4, 128)])
def test_decode_of_every_length(Hkv, G, D, dtype):
    w = filled(DECODES, [1] * len(DECODES), Hkv, D, 21, dtype)
    q = queries(w, G)
    check_attention(w, G, attend(w, G, q), q)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("split,ahead", [(16, 1), (48, 2), (112, 1), (256, 2), (0, 1), (0, 2), (0, 0)])
def test_cut_decodes_at_every_depth(split, ahead, D, dtype):
    w = filled([3000, 17, 1500, 95, 2047], [1] * 5, 2, D, 22, dtype)
    q = queries(w, 4)
    try:
        cs.cs_set_decode_split_tokens(split)
        cs.cs_set_decode_pages_ahead(ahead)
        check_attention(w, 4, attend(w, 4, q), q)
    finally:
        cs.cs_set_decode_split_tokens(0)
        cs.cs_set_decode_pages_ahead(0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("Hkv,G,D", [(2, 2, 64), (1, 8, 128), (2, 5, 128)])
@pytest.mark.parametrize("ctx,new", [([0, 0, 0], [2, 16, 17]), ([5, 16, 31, 33], [3, 16, 31, 64]), ([100, 250], [70, 130]), ([1000], [33]), ([2, 1300], [200, 2])])
def test_chunks(ctx, new, Hkv, G, D, dtype):
    w = filled(ctx, new, Hkv, D, 23, dtype)
    q = queries(w, G)
    check_attention(w, G, attend(w, G, q), q)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("mode", [0, 1, 2, 3])
def test_mixed_batches_in_every_arrangement(mode, D, dtype):
    w = filled([40, 3, 500, 1100, 0, 77, 640, 20], [1, 1, 1, 1, 30, 0, 90, 1], 2, D, 24, dtype)
    q = queries(w, 3)
    try:
        cs.cs_set_mixed_fusion(mode)
        check_attention(w, 3, attend(w, 3, q), q)
    finally:
        cs.cs_set_mixed_fusion(1)


def test_arrangements_give_the_same_bits():
    w = filled([40, 3, 500, 1100, 0, 640], [1, 1, 1, 1, 30, 90], 2, 128, 25)
    q, outs = queries(w, 4), []
    try:
        for mode in (0, 2, 3):
            cs.cs_set_mixed_fusion(mode)
            outs.append(attend(w, 4, q))
    finally:
        cs.cs_set_mixed_fusion(1)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@pytest.mark.parametrize("gain", [8.0, 2.0 ** -14])
def test_peaked_and_flat_softmaxes(gain):
    w = filled([300, 77, 10], [1, 1, 40], 2, 128, 26)
    q = queries(w, 4, gain)
    check_attention(w, 4, attend(w, 4, q), q)


def test_blocks_of_very_different_scales():
    """Pages whose scales lie 2^40 apart: each code is widened with its own block's."""
    w = World([0], [160], 2, 128, 27)
    k, v = w.rows(160), w.rows(160)
    for p in range(10):
        v[p * 16:(p + 1) * 16] *= 2.0 ** (4 * p - 20)
        k[p * 16:(p + 1) * 16] *= 2.0 ** (p % 3 - 20 * (p % 2))
    kv8.ref_append(w.pool, 0, w.tables, [0], w.cu, k, v, 2, 128)
    q = queries(w, 4)
    check_attention(w, 4, attend(w, 4, q), q)
    d = World([159], [1], 2, 128, 27)                                   # the last of them as a decode
    d.pool, d.tables = w.pool, w.tables
    qd = q[-1:].contiguous()
    check_attention(d, 4, attend(d, 4, qd), qd)


def test_bad_page_ids_harm_no_other_sequence():
    w = filled([200, 60, 90, 33], [1, 1, 20, 40], 2, 128, 28)
    q = queries(w, 4)
    good = attend(w, 4, q)
    w.tables[0, 3], w.tables[2, 1] = -1, w.P + 7
    got = attend(w, 4, q)
    for s in (1, 3):
        assert torch.equal(got[w.cu[s]:w.cu[s + 1]], good[w.cu[s]:w.cu[s + 1]])
    # a decode without a single good page: zeros
    w.tables[0, :] = -1
    assert (attend(w, 4, q)[0] == 0).all()


def test_a_nan_key_stays_with_the_rows_that_see_it():
    w = filled([64, 0], [1, 40], 1, 64, 29)
    codes, _ = kv8.block(w.pool, 0, int(w.tables[1, 1]), 1, 0, 1, 64)
    codes[kv8.v_index(4, np.arange(64))] = NAN_CODE                      # V of token 20 of the chunk
    out = attend(w, 2, queries(w, 2)).float().cpu()
    assert torch.isfinite(out[:21]).all() and torch.isnan(out[21:]).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("split", [0, 64])
def test_what_is_no_number_stays_with_the_rows_that_see_it(split, D, dtype):
    """K, V and Q, in whole and cut decodes, whole and cut chunks: K spoils a kv head's rows, V a feature of them, Q its own row."""
    Hkv, G = 2, 3
    w = filled([3000, 500, 0, 1700, 900, 20], [1, 1, 70, 40, 1, 1], Hkv, D, 32, dtype)
    want = np.zeros((w.T, Hkv * G, D), bool)
    for s, token, g, kv, d in [(0, 1234, 1, 0, 7), (1, 500, 0, 1, D - 1), (2, 33, 0, 0, 20), (2, 50, 1, 1, 33), (3, 1100, 0, 1, 3), (3, 1739, 1, 0, 0), (5, 3, 0, 0, 1)]:
        codes, _ = kv8.block(w.pool, 0, int(w.tables[s, token // 16]), kv, g, Hkv, D)
        codes[(kv8.v_index if kv else kv8.k_index)(token % 16, np.arange(d, d + 1))] = NAN_CODE
        t0 = int(w.cu[s])
        for i in range(w.new[s]):
            if token <= w.ctx[s] + i:
                want[t0 + i, g * G:(g + 1) * G, d if kv else slice(None)] = True
    q = queries(w, G)
    for s, i, h, x in [(4, 0, 2, np.nan), (4, 0, 4, np.inf), (2, 9, 1, -np.inf), (3, 8, 5, np.nan)]:
        q[int(w.cu[s]) + i, h, D // 2] = x
        want[int(w.cu[s]) + i, h] = True
    try:
        cs.cs_set_decode_split_tokens(split)
        out = attend(w, G, q)
    finally:
        cs.cs_set_decode_split_tokens(0)
    assert np.array_equal(torch.isnan(out).cpu().numpy(), want) and not torch.isinf(out).any()


def test_rows_behind_the_last_sequence_and_outside_the_batch_are_left():
    w = filled([20, 40, 8], [1, 5, 0], 2, 64, 30)
    q = queries(w, 2)
    t, b = torch.from_numpy(w.pool).cuda(), w.batch()
    before = t.clone()
    out = torch.full((w.T + 3, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    cs.cs_paged_attention_mixed_kv8(w.handle(t), 0, b.truncated(1), q, out, 4, 0.125, cs.workspace_for_kv8(b, 4, 2, 64))
    assert (out[1:] == 7.0).all()
    cs.cs_paged_attention_mixed_kv8(w.handle(t), 0, b, q, out, 4, 0.125, cs.workspace_for_kv8(b, 4, 2, 64))
    assert (out[w.T:] == 7.0).all() and torch.equal(t, before)


def test_a_pool_beyond_32_bits():
    """Pages 4 GiB and more into the pool, in either path."""
    stride, Hkv, D = 1 << 16, 2, 128
    w = filled([70, 5], [1, 40], Hkv, D, 31, stride=None)
    far = (1 << 32) // stride + 1000
    t = torch.empty((far + w.P) * stride, dtype=torch.uint8, device="cuda")
    view = t.view(-1, stride)
    view[far:, :w.stride] = torch.from_numpy(w.pool[0]).cuda()
    b = cs.Batch(torch.from_numpy(np.where(w.tables >= 0, w.tables + far, -1).astype(np.int32)), torch.tensor(w.ctx, dtype=torch.int32), torch.from_numpy(w.cu))
    pool = cs.Pool8(t, 1, far + w.P, Hkv, D, page_stride=stride)
    q = queries(w, 4)
    out = torch.empty_like(q)
    cs.cs_paged_attention_mixed_kv8(pool, 0, b, q, out, 8, 1.0 / np.sqrt(D), cs.workspace_for_kv8(b, 8, Hkv, D))
    check_attention(w, 4, out, q)
    k, v = w.rows(w.T), w.rows(w.T)
    cs.cs_kv8_append(pool, 0, b, torch.from_numpy(k).bfloat16().cuda(), torch.from_numpy(v).bfloat16().cuda())
    kv8.ref_append(w.pool, 0, w.tables, w.ctx, w.cu, k, v, Hkv, D)
    assert same_codes(view[far:, :w.stride].cpu().numpy()[None], w.pool, Hkv, D)


def test_another_stream_and_replays_of_a_graph():
    """Captured append + attention with cut sequences, replayed with eager work between; each replay against the eager result."""
    w = filled([3000, 40, 700], [1, 1, 50], 2, 128, 32)
    q, k, v = queries(w, 4), torch.from_numpy(w.rows(w.T)).bfloat16().cuda(), torch.from_numpy(w.rows(w.T)).bfloat16().cuda()
    b = w.batch()
    start = torch.from_numpy(w.pool).cuda()
    ws, out = cs.workspace_for_kv8(b, 8, 2, 128), torch.empty_like(q)
    pool = w.handle(start.clone())

    def step(stream=None):
        cs.cs_kv8_append(pool, 0, b, k, v, stream)
        cs.cs_paged_attention_mixed_kv8(pool, 0, b, q, out, 8, 0.09, ws, stream)

    step()
    torch.cuda.synchronize()
    want_out, want_pool = out.clone(), pool.tensor.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    pool.tensor.copy_(start)
    out.zero_()
    torch.cuda.synchronize()
    step(side)
    side.synchronize()
    assert torch.equal(out, want_out) and torch.equal(pool.tensor, want_pool)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(4):
        pool.tensor.copy_(start)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want_out) and torch.equal(pool.tensor, want_pool)
        step()                                                            # eager work of the same kind between the replays
        torch.cuda.synchronize()


@pytest.mark.parametrize("Hq,Hkv", [(32, 8), (28, 4)])
def test_many_sequences_of_the_model_shapes(Hq, Hkv):
    """More work items than the kernel arguments hold, and a full decode batch: random rows against the oracle."""
    for S, hi in ((1000, 60), (64, 900)):
        r = np.random.default_rng(S)
        w = filled(list(r.integers(1, hi, S)), [1] * S, Hkv, 128, 33)
        q = queries(w, Hq // Hkv)
        out = attend(w, Hq // Hkv, q)
        check_attention(w, Hq // Hkv, out, q, seqs=r.choice(S, 12, replace=False))
        assert torch.isfinite(out.float()).all()


def test_synth_batches_run_in_both_caches():
    """The tiny workload of the 16-bit path through the 8-bit one: the 16-bit result on the widened values is within the roundings."""
    b = synth.config_tiny()
    ctx, new = [int(x) for x in b.ctx_lens], [int(x) for x in b.q_lens]
    w = filled(ctx, new, b.shape.Hkv, b.shape.D, 34)
    q = queries(w, b.shape.G)
    check_attention(w, b.shape.G, attend(w, b.shape.G, q), q)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("ctx,new", [([5000, 16], [40, 700]), ([4200], [600])])
def test_chunks_over_many_windows_of_pages(ctx, new, D, dtype):
    w = filled(ctx, new, 1, D, 33, dtype)
    q = queries(w, 4)
    check_attention(w, 4, attend(w, 4, q), q)


def drawn_pool(ctx, new, Hkv, D, seed, dtype):
    """A world whose codes are drawn, not appended: for batches too large for the oracle's append."""
    w = World([], [], Hkv, D, seed, dtype)
    need = [-(-(c + n) // 16) for c, n in zip(ctx, new)]
    w.ctx, w.new, w.P = list(ctx), list(new), sum(need)
    w.cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    w.tables, perm, o = np.full((len(ctx), max(need)), -1, np.int32), w.rng.permutation(w.P).astype(np.int32), 0
    for s, n in enumerate(need):
        w.tables[s, :n] = perm[o:o + n]
        o += n
    w.pool = w.rng.integers(0, 256, (1, w.P, w.stride), np.uint8)
    w.pool[(w.pool & 127) == 127] = 0
    codes = 2 * Hkv * 16 * D
    scales = np.exp2(w.rng.integers(-9, -6, (w.P, 2 * Hkv))).astype(np.float32)      # (values up to 3.5)
    w.pool[0, :, codes:codes + 8 * Hkv] = scales.view(np.uint8)
    return w


@pytest.mark.parametrize("Hq,Hkv,decodes,chunks,dtype", [
    (28, 4, (64, 1024, 8192), [(3276, 512), (9712, 512), (10901, 512), (6220, 512)], torch.bfloat16),    # tiles whole, decode work behind them
    (40, 8, (10, 239, 956), [(6461, 576), (768, 861), (232, 761), (3545, 984)], torch.float16),          # two kernels
    (40, 8, (10, 239, 956), [(6461, 576), (768, 861), (232, 761), (3545, 984)], torch.bfloat16),
    (64, 8, (60, 500, 2000), [(3000, 300)], torch.float16)])
def test_mixes_in_the_arrangement_that_the_host_takes(Hq, Hkv, decodes, chunks, dtype):
    """Some decodes and the last rows of every chunk against the oracle; the other rows are numbers."""
    r = np.random.default_rng(40)
    n, lo, hi = decodes
    w = drawn_pool([int(x) for x in r.integers(lo, hi, n)] + [c for c, _ in chunks], [1] * n + [q for _, q in chunks], Hkv, 128, 41, dtype)
    q = queries(w, Hq // Hkv)
    out = attend(w, Hq // Hkv, q)
    assert torch.isfinite(out.float()).all()
    check_attention(w, Hq // Hkv, out, q, seqs=[0, n // 2, n - 1])
    for s in range(n, n + len(chunks)):                                  # a chunk's last rows: a shorter chunk on more context
        t = w.new[s] - 6
        tail = types.SimpleNamespace(Hkv=Hkv, D=128, dtype=dtype, pool=w.pool, layer=0, tables=w.tables[s:s + 1], ctx=[w.ctx[s] + t], new=[6], cu=np.array([0, 6]))
        rows = slice(int(w.cu[s]) + t, int(w.cu[s + 1]))
        check_attention(tail, Hq // Hkv, out[rows], q[rows])


def test_two_graphs_share_a_workspace():
    """One batch with cut decodes and cut chunks in bf16, one in fp16, replayed in turn in one workspace with an eager call between."""
    runs = []
    for seed, dtype, ctx, new in ((34, torch.bfloat16, [2900, 30, 1500], [1, 1, 60]), (35, torch.float16, [1, 2600, 4000], [1, 1, 33])):
        w = filled(ctx, new, 2, 128, seed, dtype)
        q, b = queries(w, 4), w.batch()
        pool = w.handle(torch.from_numpy(w.pool).cuda())
        runs.append((cs.cs_paged_attention_mixed_kv8 if dtype == torch.bfloat16 else cs.cs_paged_attention_mixed_kv8_f16, pool, b, q, torch.empty_like(q)))
    ws = torch.empty(max(cs.cs_paged_attention_kv8_workspace_bytes(r[2], 8, 2, 128) for r in runs), dtype=torch.uint8, device="cuda")
    want, graphs = [], []
    for fn, pool, b, q, out in runs:
        fn(pool, 0, b, q, out, 8, 0.09, ws)
        torch.cuda.synchronize()
        want.append(out.clone())
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            fn(pool, 0, b, q, out, 8, 0.09, ws)
    for i in range(6):
        for r, g, x in zip(runs, graphs, want):
            r[4].zero_()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(r[4], x)
        if i % 2:
            fn, pool, b, q, out = runs[i // 2 % 2]
            fn(pool, 0, b, q, out, 8, 0.09, ws)
            torch.cuda.synchronize()


def test_two_threads_on_streams_of_their_own():
    import threading
    ws, got, failed = [filled([2000, 30, 700], [1, 1, 50], 2, 128, s) for s in (36, 37)], [None, None], []
    qs = [queries(w, 4) for w in ws]
    want = [attend(w, 4, q) for w, q in zip(ws, qs)]
    torch.cuda.synchronize()

    def work(i):
        try:
            w, b, stream = ws[i], ws[i].batch(), torch.cuda.Stream()
            with torch.cuda.stream(stream):
                pool, space = w.handle(torch.from_numpy(w.pool).cuda()), cs.workspace_for_kv8(b, 8, 2, 128)
                outs = [torch.empty_like(qs[i]) for _ in range(20)]
                for out in outs:
                    cs.cs_paged_attention_mixed_kv8(pool, 0, b, qs[i], out, 8, 1.0 / np.sqrt(128), space, stream)
            stream.synchronize()
            got[i] = outs
        except Exception as e:                                            # (a thread's own failure would go unseen)
            failed.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed
    for x, outs in zip(want, got):
        assert all(torch.equal(out, x) for out in outs)


def nans_of_v_in_every_step(w, G):
    """A V that is not a number in every 32 keys of every sequence, each in a feature of its own (a step's kv head and feature are not
    used again); which outputs see one.  Rows before the first token of a step keep its feature."""
    want = np.zeros((w.T, w.Hkv * G, w.D), bool)
    for s, (c, n) in enumerate(zip(w.ctx, w.new)):
        for step in range(-(-(c + n) // 32)):
            assert step < w.Hkv * w.D
            token, g, d = min(32 * step + int(w.rng.integers(32)), c + n - 1), step % w.Hkv, step // w.Hkv
            codes, _ = kv8.block(w.pool, 0, int(w.tables[s, token // 16]), 1, g, w.Hkv, w.D)
            codes[kv8.v_index(token % 16, np.arange(d, d + 1))] = NAN_CODE | (128 if step & 1 else 0)
            t0 = int(w.cu[s])
            want[t0 + max(token - c, 0):t0 + n, g * G:(g + 1) * G, d] = True
    return want


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("cus", [2, 256])
@pytest.mark.parametrize("ctx,new", [(64, 40), (100, 40), (0, 40), (500, 40), (1700, 40), (1733, 40), (991, 300), (3000, 33), (3021, 17)])
def test_a_v_that_is_no_number_at_every_place_of_a_tile(ctx, new, cus, D, dtype):
    """Tiles whole (2 CUs need no cuts) and cut into ranges (256): edges at odd and even steps, ranges of odd and even length."""
    w = filled([ctx], [new], 2, D, 50, dtype)
    want, q = nans_of_v_in_every_step(w, 3), queries(w, 3)
    try:
        cs.cs_debug_set_cu_count(cus)
        out = attend(w, 3, q)
    finally:
        cs.cs_debug_set_cu_count(0)
    assert np.array_equal(torch.isnan(out).cpu().numpy(), want) and not torch.isinf(out).any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("mode", [0, 2, 3])
def test_a_v_that_is_no_number_in_every_step_of_a_mix(mode, D, dtype):
    w = filled([40, 500, 1700, 2100, 65, 960, 300], [1, 1, 40, 1, 70, 33, 1], 2, D, 51, dtype)
    want, q = nans_of_v_in_every_step(w, 4), queries(w, 4)
    try:
        cs.cs_set_mixed_fusion(mode)
        out = attend(w, 4, q)
    finally:
        cs.cs_set_mixed_fusion(1)
    assert np.array_equal(torch.isnan(out).cpu().numpy(), want) and not torch.isinf(out).any()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("ctx,new", [([6, 0, 16], [1, 1, 1]), ([0, 6, 33], [24, 9, 2])])
def test_append_of_the_largest_values_of_bf16(ctx, new, D):
    """From 248 * 2^120 on the nearest code at the block's scale, 256, would stand for 2^128, an infinity: 240 it is.  The rows
    that do not see such a V stay what they are (0 * infinity would be no number)."""
    w = World(ctx, new, 2, D, 52)
    k, v = w.rows(w.T), w.rows(w.T)
    most = float(torch.finfo(torch.bfloat16).max)
    for s in range(3):
        row = int(w.cu[s + 1]) - 1                                       # a sequence's last token
        v[row, 0, 0], v[row, 0, 3], v[row, 0, 5], v[row, 0, 6] = most, -most, 248 * 2.0 ** 120, 240 * 2.0 ** 120
        v[row, 0, 7] = np.inf
    w.pool[0] = np.where((w.pool[0] & 127) == 127, 0, w.pool[0])
    got, want = w.append(k, v)
    assert same_codes(got, want, 2, D)
    w.pool = got
    for s in range(3):
        _, V = kv8.read_logical(got, 0, w.tables[s], ctx[s] + new[s], 2, D)
        assert list(V[-1, 0, [0, 3, 5, 6, 7]]) == [240 * 2.0 ** 120 * sign for sign in (1, -1, 1, 1, 1)]
    q = queries(w, 2)
    out = attend(w, 2, q)
    for s in range(3):
        # A chunk's weights are relative to a maximum that may lie 2^6 below the scores', and its sums are normalised at the end: 2^6 * 240 *
        # 2^120 is beyond fp32, so the one row that sees these values may say so, in their features.  All others, and
        # decodes (whose weights are at most 1, with one such value a feature), are within the roundings.
        rows = slice(int(w.cu[s]), int(w.cu[s + 1]) - (new[s] > 1))
        few = types.SimpleNamespace(Hkv=2, D=D, dtype=w.dtype, pool=w.pool, layer=0, tables=w.tables[s:s + 1], ctx=[ctx[s]], new=[rows.stop - rows.start], cu=np.array([0]))
        check_attention(few, 2, out[rows], q[rows])
        large = out[int(w.cu[s + 1]) - 1].clone()
        large[:2, [0, 3, 5, 6, 7]] = 0
        assert torch.isfinite(large).all()


@pytest.mark.parametrize("new", [1, 5])
def test_what_an_infinity_becomes(new):
    """bf16: the largest code at the scale of the block's other values; fp16: 61440, whatever the others are."""
    for dtype, exponent, value in ((torch.bfloat16, -8, 448 * 2.0 ** -8), (torch.float16, 8, 61440.0)):
        w = World([0], [new], 1, 64, 53, dtype)
        k = np.ones((new, 1, 64))
        k[-1, 0, 9] = -np.inf
        got, _ = w.append(k, np.ones((new, 1, 64)))
        assert kv8.block(got, 0, int(w.tables[0, 0]), 0, 0, 1, 64)[1][0] == 2.0 ** exponent
        K, V = kv8.read_logical(got, 0, w.tables[0], new, 1, 64)
        want = np.ones((new, 1, 64))
        assert np.array_equal(V, want)
        want[-1, 0, 9] = -value
        assert np.array_equal(K, want)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype,above", [(torch.bfloat16, 2.0 ** 4), (torch.bfloat16, 2.0 ** 12), (torch.bfloat16, 2.0 ** 15), (torch.bfloat16, 2.0 ** 17),
                                         (torch.float16, 2.0 ** 4), (torch.float16, 2.0 ** 12)])
def test_a_feature_of_q_far_above_the_others_where_k_is_zero(above, D, dtype):
    """The scores come from the small values alone.  Under bf16 a chunk's Q is two codes a value: 2^-21.8 of the row's largest may be
    missing from each, top * 2^-21.8 * sum |K_j| from a score; an error of d in the exponents makes at most e^(2d) - 1 of a
    weight.  (fp16 ends at 65504.)"""
    w = filled([300, 9], [40, 33], 2, D, 54, dtype)
    G, far = 3, 11
    for page in range(w.P):
        for h in range(2):
            codes, _ = kv8.block(w.pool, 0, page, 0, h, 2, D)
            codes[kv8.k_index(np.arange(16), far)] = 0
    q = queries(w, G)
    q[:, :, far] *= above
    got, qf, h16, scale = attend(w, G, q).double().cpu().numpy(), q.double().cpu().numpy(), HALF_STEP[dtype], 1.0 / np.sqrt(D)
    for s in range(2):
        c, n, t0 = w.ctx[s], w.new[s], int(w.cu[s])
        K, V = kv8.read_logical(w.pool, 0, w.tables[s], c + n, 2, D)
        ref, spread, reach = kv8.attention(qf[t0:t0 + n], K, V, c, scale)
        top = np.abs(qf[t0:t0 + n]).max(-1)
        most = np.repeat(np.abs(K).sum(-1).max(0), G)                    # of a kv head's keys
        off = scale * top * 2.0 ** -21.8 * most[None] if dtype == torch.bfloat16 else 0.0 * top
        fold = h16 if dtype == torch.float16 else 0.0
        weights = 1.01 * (h16 + np.expm1(2 * (off + (fold + 2.0 ** -20) * reach)))[..., None] * spread
        tiny = (c + n) * 2.0 ** -25 * 2 * np.abs(V).max() if dtype == torch.float16 else 0.0
        bound = 1.01 * (h16 + 2.0 ** -20) * np.abs(ref) + weights + tiny + 2.0 ** -20 * np.abs(V).max()
        assert (np.abs(got[t0:t0 + n] - ref) <= bound).all()


@pytest.mark.parametrize("D", [64, 128])
def test_half_precision_blocks_of_very_small_values(D):
    """fp16 values down to its subnormal ones, 2^-24, in pages of different scales, in decodes and chunks: the codes of such a value are
    multiples of 2^-24, so widening them to half precision rounds nothing."""
    w = World([0, 0], [160, 160], 2, D, 55, torch.float16)
    k, v = w.rows(w.T), w.rows(w.T)
    for p in range(20):
        v[p * 16:(p + 1) * 16] *= 2.0 ** -(p % 10 + 8)
        k[p * 16:(p + 1) * 16] *= 2.0 ** -(p % 7 + 8)
    k, v = (torch.from_numpy(x).half().double().numpy() for x in (k, v))
    kv8.ref_append(w.pool, 0, w.tables, [0, 0], w.cu, k, v, 2, D, True)
    for s in range(2):
        for x in kv8.read_logical(w.pool, 0, w.tables[s], 160, 2, D):
            assert np.array_equal(x, x.astype(np.float16)) and (np.abs(x[x != 0]) < 2.0 ** -14).any()
    q = queries(w, 4, 2.0 ** 9)
    check_attention(w, 4, attend(w, 4, q), q)
    d = World([159, 159], [1, 1], 2, D, 55, torch.float16)               # the last of either as decodes
    d.pool, d.tables, d.P = w.pool, w.tables, w.P
    qd = q[[159, 319]].contiguous()
    check_attention(d, 4, attend(d, 4, qd), qd)


@pytest.mark.parametrize("which,dtype", [(0, torch.bfloat16), (1, torch.float16), (1, torch.bfloat16), (2, torch.bfloat16), (2, torch.float16)])
def test_mixes_at_model_shapes_run_as_planned_and_are_right_in_every_part_of_a_chunk(which, dtype):
    """The arrangement is asked for first (tiles whole with decode work behind them; two kernels; cut tiles): then rows of the
    first, a middle and the last tile of each chunk against the oracle."""
    from test_kv8_host import ARRANGED, arranged_batch
    Hq, Hkv, decodes, chunks, want = ARRANGED[which]
    ctx, new = arranged_batch(decodes, chunks)
    w = drawn_pool(ctx, new, Hkv, 128, 56, dtype)
    q = queries(w, Hq // Hkv)
    try:
        cs.cs_debug_set_cu_count(256)
        assert cs.cs_debug_mixed_kv8(w.batch(), Hq, Hkv, 128) == want
        out = attend(w, Hq // Hkv, q)
    finally:
        cs.cs_debug_set_cu_count(0)
    assert torch.isfinite(out.float()).all()
    check_attention(w, Hq // Hkv, out, q, seqs=[1, decodes[0] // 3])
    for s in range(decodes[0], len(ctx)):
        for t in (0, new[s] // 2 - 1, new[s] - 3):
            part = types.SimpleNamespace(Hkv=Hkv, D=128, dtype=dtype, pool=w.pool, layer=0, tables=w.tables[s:s + 1], ctx=[ctx[s] + t], new=[3], cu=np.array([0, 3]))
            rows = slice(int(w.cu[s]) + t, int(w.cu[s]) + t + 3)
            check_attention(part, Hq // Hkv, out[rows], q[rows])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("Hq,Hkv,decodes,chunks", [(32, 8, (100, 100, 3000), [(2000, 300), (50, 700)]), (4, 2, (64, 1000, 8000), [(5000, 512)])])
def test_mixes_of_head_dim_64_at_model_sizes(Hq, Hkv, decodes, chunks, dtype):
    from test_kv8_host import arranged_batch
    ctx, new = arranged_batch(decodes, chunks)
    w = drawn_pool(ctx, new, Hkv, 64, 57, dtype)
    q = queries(w, Hq // Hkv)
    for mode in (0, 2, 3):
        try:
            cs.cs_set_mixed_fusion(mode)
            out = attend(w, Hq // Hkv, q)
        finally:
            cs.cs_set_mixed_fusion(1)
        assert torch.isfinite(out.float()).all()
        check_attention(w, Hq // Hkv, out, q, seqs=[0, decodes[0] - 1])
        for s in range(decodes[0], len(ctx)):
            for t in (0, new[s] // 2, new[s] - 3):
                part = types.SimpleNamespace(Hkv=Hkv, D=64, dtype=dtype, pool=w.pool, layer=0, tables=w.tables[s:s + 1], ctx=[ctx[s] + t], new=[3], cu=np.array([0, 3]))
                rows = slice(int(w.cu[s]) + t, int(w.cu[s]) + t + 3)
                check_attention(part, Hq // Hkv, out[rows], q[rows])
