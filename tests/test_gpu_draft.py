"""The speculative step on the GPU: norm, rotation and append, attention of trees, verification and commit, each against fp64."""
import numpy as np
import pytest
import torch

from oracle import draft, kv_layout
from paper_2410_01228_amd import binding as cs

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16
HALF_STEP = {BF16: 2.0 ** -8, F16: 2.0 ** -11}
NAN_BITS = {BF16: 0x7FC0, F16: 0x7E00}


def bits(t):
    return t.detach().contiguous().cpu().view(torch.int16).numpy().view(np.uint16)


def tensor(b, dtype):
    return torch.from_numpy(np.ascontiguousarray(b).view(np.int16)).view(dtype)


def values(b, dtype):
    return tensor(b, dtype).double().numpy()


def fn(name, dtype):
    return getattr(cs, name + ("_f16" if dtype == F16 else ""))


class World:
    """A batch over a 16-bit pool on the CPU: earlier tokens written by the oracle, all other slots NaN."""

    def __init__(self, ctx, new, Hkv, D, seed, dtype=BF16, page_size=16, layers=1, layer=0, pad=0, gain=1.0):
        self.ctx, self.new, self.Hkv, self.D, self.dtype, self.ps, self.layer, self.layers = list(ctx), list(new), Hkv, D, dtype, page_size, layer, layers
        self.rng = np.random.default_rng(seed)
        need = [-(-(c + q) // page_size) for c, q in zip(ctx, new)]
        self.P = sum(need) + 3
        perm = self.rng.permutation(self.P).astype(np.int32)
        self.tables = np.full((max(1, len(ctx)), max(need + [1])), -1, np.int32)
        o = 0
        for s, n in enumerate(need):
            self.tables[s, :n] = perm[o:o + n]
            o += n
        self.cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.pad, self.elems = pad, 2 * Hkv * page_size * D
        self.pool = kv_layout.new_pool(layers, self.P, Hkv, D, NAN_BITS[dtype], page_size=page_size)
        cu_old = np.concatenate([[0], np.cumsum(ctx)]).astype(np.int32)
        self.k_old, self.v_old = self.rows(int(cu_old[-1]), Hkv, gain), self.rows(int(cu_old[-1]), Hkv, gain)
        self.cu_old = cu_old
        self.put(layer, np.zeros(len(ctx), np.int32), cu_old, self.k_old, self.v_old)

    @property
    def T(self):
        return int(self.cu[-1])

    def rows(self, n, heads, gain=1.0):
        return bits(torch.from_numpy(self.rng.standard_normal((n, heads, self.D)) * gain).to(self.dtype))

    def put(self, layer, ctx, cu, k, v):
        kv_layout.ref_append(self.pool, layer, self.tables, ctx, cu, k, v, page_size=self.ps)

    def append(self, k, v, layer=None):
        self.put(self.layer if layer is None else layer, self.ctx, self.cu, k, v)

    def batch(self):
        return cs.Batch(torch.from_numpy(self.tables), torch.tensor(self.ctx, dtype=torch.int32), torch.from_numpy(self.cu))

    def device_pool(self):
        """(handle, tensor [layers, P, elems + pad]) of the pool as it is now; the padding NaN."""
        t = torch.from_numpy(np.full((self.layers, self.P, self.elems + self.pad), NAN_BITS[self.dtype], np.uint16).view(np.int16))
        t[..., :self.elems] = torch.from_numpy(self.pool.reshape(self.layers, self.P, -1).view(np.int16))
        t = t.cuda()
        return cs.Pool(t, self.layers, self.P, self.Hkv, self.D, page_stride=self.elems + self.pad, page_size=self.ps), t

    def host_pool(self, t):
        a = t.cpu().numpy().view(np.uint16)
        assert np.all(a[..., self.elems:] == NAN_BITS[self.dtype])
        return a[..., :self.elems].reshape(self.pool.shape)

    def logical(self, s, layer=None):
        n = self.ctx[s] + self.new[s]
        k, v = kv_layout.read_logical(self.pool, self.layer if layer is None else layer, self.tables[s], n, page_size=self.ps)
        return values(k, self.dtype), values(v, self.dtype)


# ------------------------------------------------------------------------------- norm, rotation, append

def rope_tolerance(want, size, dtype, angle):
    """Half a step of the type, fp32 arithmetic in the chain (norm: a sum of at most 128 squares, a root, a quotient and two products, under 2^-18 in all)
    and the angle's own error (2^-24 of half a turn, and 2^-52 of itself)."""
    small = 2.0 ** -25 if dtype == F16 else 0.0
    return HALF_STEP[dtype] * np.abs(want) + size * (2.0 ** -18 + 2.0 ** -21 + angle * 2.0 ** -51) + small


ROPES = [
    # Hq, Hkv, D, rotary, interleaved, norm, axes
    (4, 2, 64, 64, False, False, 1), (4, 2, 64, 32, True, True, 1), (8, 1, 128, 128, False, True, 3), (28, 4, 128, 64, False, False, 2), (3, 3, 128, 128, True, False, 3),
    (40, 8, 128, 8, False, True, 1), (2, 1, 64, 0, False, True, 1), (5, 5, 64, 16, True, True, 2), (16, 8, 128, 128, False, False, 1),
]
STEPS = [((5, 0, 33), (1, 1, 1)), ((0, 15, 16, 31, 100), (1, 17, 0, 2, 40)), ((7,), (1,)), ((9, 70), (16, 1)), ((0,), (64,))]


def make_rope(rng, T, D, rotary, interleaved, norm, axes, dtype, positions=None, eps=1e-5):
    pairs = rotary // 2
    inv = (500000.0 ** (-np.arange(pairs) / max(pairs, 1))).astype(np.float32)
    split = None if axes == 1 else [pairs - pairs // 4 * (axes - 1)] + [pairs // 4] * (axes - 1)
    at = rng.integers(0, 100000, (axes, T)).astype(np.int32) if positions is None else positions
    weights = [bits(torch.from_numpy(1 + rng.standard_normal(D) / 4).to(dtype)) if norm else None for _ in range(2)]
    wide = torch.zeros((axes, T + 5), dtype=torch.int32)                       # (a longer list than the step's)
    wide[:, :T] = torch.from_numpy(at)
    rope = cs.Rope(torch.from_numpy(inv).cuda(), rotary, wide.cuda(), split, interleaved, *(None if w is None else tensor(w, dtype).cuda() for w in weights), eps)
    ref = lambda x, w: draft.ref_rope(values(x, dtype), at, inv, rotary, interleaved, None if w is None else values(w, dtype), eps, split)  # noqa: E731
    return rope, ref, weights, float(np.abs(at).max(initial=0))


def near(got, want, tol, what):
    off = np.abs(got - want) - tol
    assert np.all(np.isfinite(got)) and off.max(initial=-1.0) <= 0, (what, float(off.max()), np.unravel_index(np.argmax(off), off.shape))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("shape", ROPES)
@pytest.mark.parametrize("T", [1, 15, 17, 200])
def test_rotated_rows(shape, T, dtype):
    Hq, Hkv, D, rotary, interleaved, norm, axes = shape
    rng = np.random.default_rng(T)
    rope, ref, weights, far = make_rope(rng, T, D, rotary, interleaved, norm, axes, dtype)
    fused = torch.from_numpy(rng.standard_normal((T, Hq + Hkv + 2, D)) * 2).to(dtype)
    dev = fused.cuda()
    q, k = dev[:, 1:1 + Hq], dev[:, 1 + Hq:1 + Hq + Hkv]
    q_out, k_out = torch.full((T + 1, Hq, D), 7.0, dtype=dtype, device="cuda"), torch.full((T + 1, Hkv, D), 7.0, dtype=dtype, device="cuda")
    fn("cs_qk_rope", dtype)(rope, q, k, q_out, k_out)
    for got, x, w in ((q_out, q, weights[0]), (k_out, k, weights[1])):
        assert torch.all(got[T:] == 7.0)
        want, size = ref(bits(x), w)
        near(got[:T].double().cpu().numpy(), want, rope_tolerance(want, size, dtype, far), shape)
        if not norm:
            assert torch.equal(got[:T, :, rotary:], x[..., rotary:])
    assert torch.equal(dev.cpu(), fused)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("page_size", [16, 8])
@pytest.mark.parametrize("shape", ROPES)
@pytest.mark.parametrize("ctx,new", STEPS)
def test_rotated_append(ctx, new, shape, page_size, dtype):
    Hq, Hkv, D, rotary, interleaved, norm, axes = shape
    w = World(ctx, new, Hkv, D, 11, dtype, page_size, layers=2, layer=1, pad=8)
    rope, ref, weights, far = make_rope(w.rng, w.T, D, rotary, interleaved, norm, axes, dtype)
    fused = torch.from_numpy(w.rng.standard_normal((w.T, Hq + 2 * Hkv, D)) * 2).to(dtype)
    dev = fused.cuda()
    q, k, v = dev[:, :Hq], dev[:, Hq:Hq + Hkv], dev[:, Hq + Hkv:]
    q_out = torch.empty((w.T, Hq, D), dtype=dtype, device="cuda")
    pool, t = w.device_pool()
    fn("cs_kv_append_rope", dtype)(pool, 1, w.batch(), rope, q, k, v, q_out)
    want, size = ref(bits(q), weights[0])
    near(q_out.double().cpu().numpy(), want, rope_tolerance(want, size, dtype, far), shape)
    got = w.host_pool(t)
    # K's rows are what cs_qk_rope makes of them, bit for bit; everything else is as the plain append leaves it
    q2, k2 = torch.empty_like(q_out), torch.empty((w.T, Hkv, D), dtype=dtype, device="cuda")
    fn("cs_qk_rope", dtype)(rope, q, k, q2, k2)
    assert torch.equal(q2, q_out)
    w.append(bits(k2), bits(v))
    assert np.array_equal(got, w.pool)


@pytest.mark.parametrize("ctx,new", STEPS)
def test_rotated_append_counts_positions_by_itself(ctx, new):
    w = World(ctx, new, 2, 64, 12)
    at = np.concatenate([c + np.arange(n) for c, n in zip(ctx, new)]).astype(np.int32)[None]
    inv = torch.from_numpy((1e4 ** (-np.arange(32) / 32)).astype(np.float32)).cuda()
    q, k, v = (torch.randn(w.T, h, 64, generator=torch.Generator().manual_seed(h)).to(BF16).cuda() for h in (4, 2, 2))
    out = []
    for rope in (cs.Rope(inv, 64, torch.from_numpy(at).cuda()), cs.Rope(inv, 64)):
        pool, t = w.device_pool()
        q_out = torch.empty_like(q)
        cs.cs_kv_append_rope(pool, 0, w.batch(), rope, q, k, v, q_out)
        out.append((q_out, t))
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_far_positions_and_outputs_in_place(dtype):
    rng = np.random.default_rng(13)
    T, Hq, Hkv, D = 40, 6, 2, 128
    at = (2 ** 31 - 1 - rng.integers(0, 1000, (1, T))).astype(np.int32)
    at[0, ::3] *= -1
    rope, ref, weights, far = make_rope(rng, T, D, 128, False, True, 1, dtype, positions=at)
    q, k = (torch.from_numpy(rng.standard_normal((T, h, D))).to(dtype) for h in (Hq, Hkv))
    dq, dk = q.cuda(), k.cuda()
    fn("cs_qk_rope", dtype)(rope, dq, dk, dq, dk)
    for got, x, w in ((dq, q, weights[0]), (dk, k, weights[1])):
        want, size = ref(bits(x), w)
        near(got.double().cpu().numpy(), want, rope_tolerance(want, size, dtype, far), "far")


def test_large_append_of_many_sequences():
    """More workgroups than one trip of the search for a workgroup's sequence; lengths of zero among them."""
    rng = np.random.default_rng(14)
    new = rng.choice([0, 1, 1, 2, 5, 33], 500).tolist()
    w = World(rng.integers(0, 40, 500).tolist(), new, 1, 64, 15)
    rope, _, _, _ = make_rope(rng, w.T, 64, 64, False, False, 1, BF16)
    q, k, v = (torch.from_numpy(rng.standard_normal((w.T, h, 64))).to(BF16).cuda() for h in (2, 1, 1))
    pool, t = w.device_pool()
    q_out, q2, k2 = torch.empty_like(q), torch.empty_like(q), torch.empty_like(k)
    cs.cs_kv_append_rope(pool, 0, w.batch(), rope, q, k, v, q_out)
    cs.cs_qk_rope(rope, q, k, q2, k2)
    w.append(bits(k2), bits(v))
    assert torch.equal(q_out, q2) and np.array_equal(w.host_pool(t), w.pool)


def test_rotated_append_skips_bad_pages():
    w = World((20, 5, 40), (20, 1, 30), 2, 64, 16)
    rope, _, _, _ = make_rope(w.rng, w.T, 64, 64, False, True, 1, BF16)
    q, k, v = (torch.from_numpy(w.rng.standard_normal((w.T, h, 64))).to(BF16).cuda() for h in (4, 2, 2))
    good = w.tables.copy()
    w.tables[0, 1], w.tables[1, 0], w.tables[2, 3] = -1, w.P, 2 ** 31 - 1
    pool, t = w.device_pool()
    q_out, q2, k2 = torch.empty_like(q), torch.empty_like(q), torch.empty_like(k)
    cs.cs_kv_append_rope(pool, 0, w.batch(), rope, q, k, v, q_out)
    cs.cs_qk_rope(rope, q, k, q2, k2)
    assert torch.equal(q_out, q2)
    before = w.pool.copy()
    w.tables = good
    w.append(bits(k2), bits(v))
    for s, b in ((0, 1), (1, 0), (2, 3)):
        w.pool[:, good[s, b]] = before[:, good[s, b]]
    assert np.array_equal(w.host_pool(t), w.pool)


# ------------------------------------------------------------------------------------- trees

def random_tree(rng, n, width):
    return [-1] + [int(rng.integers(max(0, i - 1 - width), i)) for i in range(1, n)]


def tree_step(w, Hq, rng, q_gain=1.0):
    """Appends a step's K and V, and returns its queries."""
    w.append(w.rows(w.T, w.Hkv), w.rows(w.T, w.Hkv))
    return tensor(w.rows(w.T, Hq, q_gain), w.dtype)


def run_tree(w, q, Hq, masks, scale, batch=None, words=None, poison=True):
    """masks: bool [n, n or more] per sequence, or None."""
    batch = batch or w.batch()
    pool, t = w.device_pool()
    mask = None
    if masks is not None:
        words = words or max(1, -(-max(m.shape[1] for m in masks) // 64))
        mask = torch.from_numpy(np.concatenate([draft.mask_words(m, words) for m in masks])).cuda()
    out = torch.full((q.shape[0] + 2, Hq, w.D), 9.0, dtype=w.dtype, device="cuda")
    ws = cs.workspace_for_tree(batch, Hq, w.Hkv, w.D)
    if poison:
        ws.fill_(255)
    fn("cs_paged_attention_tree", w.dtype)(pool, w.layer, batch, q.cuda(), out, Hq, scale, mask, ws)
    out = out.cpu()
    assert torch.all(out[batch.num_tokens:] == 9.0)
    return out[:batch.num_tokens]


def check_tree(w, q, Hq, masks, scale, got):
    for s in range(len(w.ctx)):
        n, t0 = w.new[s], int(w.cu[s])
        if n == 0:
            continue
        k, v = w.logical(s)
        seen = np.tril(np.ones((n, n), bool)) if masks is None else masks[s][:, :n]
        want, tol = draft.ref_tree_attention(q[t0:t0 + n].double().numpy(), k, v, seen, scale, HALF_STEP[w.dtype], w.dtype == F16)
        near(got[t0:t0 + n].double().numpy(), want, tol, (s, w.ctx[s], n))


TREES = [
    # Hq, Hkv, D, contexts, nodes
    (4, 2, 64, (17, 100), (5, 8)),
    (4, 2, 64, (0, 1, 31, 32, 33, 15), (1, 2, 1, 7, 31, 3)),
    (28, 4, 128, (129, 0, 700), (24, 64, 1)),
    (8, 8, 128, (5, 300), (65, 33)),
    (16, 1, 128, (64, 127), (4, 9)),
    (5, 1, 64, (40, 250), (256, 129)),
    (32, 8, 128, (3000, 0, 5), (6, 0, 5)),
    (64, 8, 128, (2100,), (16,)),
    (2, 2, 64, (6000, 90), (3, 2)),
]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("page_size", [16, 8])
@pytest.mark.parametrize("shape", TREES)
def test_trees(shape, page_size, dtype):
    Hq, Hkv, D, ctx, new = shape
    w = World(ctx, new, Hkv, D, 21, dtype, page_size, layers=2, layer=1, pad=16)
    q = tree_step(w, Hq, w.rng)
    masks = [draft.ancestors(random_tree(w.rng, n, 4)) if n else np.zeros((0, 1), bool) for n in new]
    check_tree(w, q, Hq, masks, D ** -0.5, run_tree(w, q, Hq, masks, D ** -0.5))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("shape", TREES[:6])
def test_any_masks(shape, dtype):
    """Masks that no tree has: rows that see nothing (zeros where there is no context), bits of nodes that are not there, more words than needed."""
    Hq, Hkv, D, ctx, new = shape
    w = World(ctx, new, Hkv, D, 22, dtype)
    q = tree_step(w, Hq, w.rng, 4.0)
    masks = [w.rng.random((n, 256)) < 0.3 for n in new]
    for m in masks:
        m[::3, :] = False
        m[::3, m.shape[0]:] = True
    got = run_tree(w, q, Hq, masks, D ** -0.5, words=4)
    check_tree(w, q, Hq, masks, D ** -0.5, got)
    for s, c in enumerate(ctx):
        if c == 0:
            assert torch.all(got[int(w.cu[s]):int(w.cu[s + 1]):3] == 0)


@pytest.mark.parametrize("shape", [TREES[1], TREES[5], TREES[6]])
def test_chains_need_no_mask(shape):
    Hq, Hkv, D, ctx, new = shape
    w = World(ctx, new, Hkv, D, 23)
    q = tree_step(w, Hq, w.rng)
    got = run_tree(w, q, Hq, None, D ** -0.5)
    check_tree(w, q, Hq, None, D ** -0.5, got)
    chains = [np.tril(np.ones((n, max(n, 1)), bool)) for n in new]
    assert torch.equal(got, run_tree(w, q, Hq, chains, D ** -0.5))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("what", ["k nan", "k inf", "v nan", "v inf", "v -inf"])
def test_what_a_row_does_not_see_has_no_effect_on_it(what, dtype):
    Hq, Hkv, D, ctx, new = 8, 2, 64, (70, 0), (40, 12)
    w = World(ctx, new, Hkv, D, 24, dtype)
    q = tree_step(w, Hq, w.rng)
    masks = [draft.ancestors(random_tree(w.rng, n, 3)) for n in new]
    clean = run_tree(w, q, Hq, masks, 0.1)
    bad = {"nan": NAN_BITS[dtype], "inf": 0x7F80 if dtype == BF16 else 0x7C00}[what.split()[1].strip("-")] | (0x8000 if "-" in what else 0)
    node = [17, 5]
    kv = 0 if what[0] == "k" else 1
    index = (kv_layout.k_index, kv_layout.v_index)[kv]
    for s in range(2):
        at = ctx[s] + node[s]
        w.pool[0, w.tables[s, at // 16], kv, 1, index(at % 16, np.arange(D), D)] = bad     # kv head 1 of one node
    got = run_tree(w, q, Hq, masks, 0.1)
    for s in range(2):
        for i in range(new[s]):
            row, was = got[int(w.cu[s]) + i], clean[int(w.cu[s]) + i]
            assert torch.equal(row[:4], was[:4])
            if not masks[s][i, node[s]]:
                assert torch.equal(row[4:], was[4:]), (s, i)
            elif what == "k nan" or what == "v nan":
                assert torch.all(torch.isnan(row[4:]))
            elif what[0] == "v":
                assert torch.all(row[4:] == (float("inf") if "-" not in what else float("-inf")))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("page_size", [16, 8])
@pytest.mark.parametrize("D", [64, 128])
def test_every_number_of_row_tiles(D, page_size, dtype):
    """Rows that fill 1 to 27 tiles of 16, the last one partly, beside a sequence with fewer; contexts from none to some rounds of keys."""
    G, rng = 5, np.random.default_rng(31)
    for tiles in range(1, 28):
        n = -(-(16 * (tiles - 1) + 1) // G)
        ctx, new = (int(rng.integers(0, 600)), int(rng.integers(0, 300))), (n, int(rng.integers(0, n + 1)))
        w = World(ctx, new, 1, D, tiles, dtype, page_size)
        q = tree_step(w, G, w.rng)
        masks = [draft.ancestors(random_tree(w.rng, m, 6)) if m else np.zeros((0, 1), bool) for m in new]
        check_tree(w, q, G, masks, D ** -0.5, run_tree(w, q, G, masks, D ** -0.5))


@pytest.mark.parametrize("S", [1, 2, 5, 9, 17])
@pytest.mark.parametrize("Hkv", [1, 2, 3, 4, 6])
def test_blocks_of_few_kv_heads(Hkv, S):
    """Work items are dealt to the XCDs in whole rounds where the kv heads divide their number: counts that fill no round, blocks and pieces among them."""
    G, D, rng = 4, 64, np.random.default_rng(100 * Hkv + S)
    new = rng.integers(17, 130, S).tolist()
    w = World(rng.integers(0, 1500, S).tolist(), new, Hkv, D, 10 * Hkv + S)
    q = tree_step(w, Hkv * G, w.rng)
    masks = [draft.ancestors(random_tree(w.rng, n, 5)) for n in new]
    check_tree(w, q, Hkv * G, masks, D ** -0.5, run_tree(w, q, Hkv * G, masks, D ** -0.5))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("page_size", [16, 8])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("nodes", [3, 7, 10, 20, 40])
def test_long_walks_over_shared_pages(nodes, D, page_size, dtype):
    """As many sequences as the chip has room for, so that none is cut, all behind one prefix whose page table is longer than a wavefront."""
    S, ctx, Hkv, Hq, pages = 16, 1216, 32, 128, 1216 // page_size
    w = World([ctx] + [0] * (S - 1), [nodes] * S, Hkv, D, nodes, dtype, page_size)
    own = w.tables[1:, :w.tables.shape[1] - pages].copy()
    w.tables[1:, :pages] = w.tables[0, :pages]
    w.tables[1:, pages:] = own
    w.ctx = [ctx] * S
    q = tree_step(w, Hq, w.rng)
    masks = [draft.ancestors(random_tree(w.rng, nodes, 3)) for _ in range(S)]
    got = run_tree(w, q, Hq, masks, D ** -0.5)
    for s in (0, 7, 15):
        k, v = w.logical(s)
        t0 = s * nodes
        want, tol = draft.ref_tree_attention(q[t0:t0 + nodes].double().numpy(), k, v, masks[s], D ** -0.5, HALF_STEP[dtype], dtype == F16)
        near(got[t0:t0 + nodes].double().numpy(), want, tol, s)


def test_trees_agree_with_the_mixed_call_on_chains_and_tokens():
    Hq, Hkv, D, ctx, new = 32, 8, 128, (100, 900, 33, 0), (1, 6, 40, 3)
    w = World(ctx, new, Hkv, D, 25)
    q = tree_step(w, Hq, w.rng)
    pool, _ = w.device_pool()
    batch = w.batch()
    out = torch.empty_like(q).cuda()
    cs.cs_paged_attention_mixed(pool, 0, batch, q.cuda(), out, Hq, 0.1, cs.workspace_for(batch, Hq, Hkv, D))
    check_tree(w, q, Hq, None, 0.1, run_tree(w, q, Hq, None, 0.1))
    check_tree(w, q, Hq, None, 0.1, out.cpu())


def test_more_items_than_a_launch_takes_and_prefixes():
    rng = np.random.default_rng(26)
    ctx, new = rng.integers(0, 70, 1000).tolist(), rng.integers(0, 4, 1000).tolist()
    ctx[500], new[500] = 9000, 30
    w = World(ctx, new, 1, 64, 27)
    q = tree_step(w, 4, rng)
    masks = [draft.ancestors(random_tree(rng, n, 2)) if n else np.zeros((0, 1), bool) for n in new]
    got = run_tree(w, q, 4, masks, 0.125)
    check_tree(w, q, 4, masks, 0.125, got)
    half = w.batch().truncated(501)
    part = run_tree(w, q, 4, masks, 0.125, batch=half)
    w.ctx, w.new, w.cu = ctx[:501], new[:501], w.cu[:502]
    check_tree(w, q, 4, masks, 0.125, part)


def test_a_bad_page_harms_no_other_sequence():
    w = World((50, 60, 20), (9, 12, 3), 2, 64, 28)
    q = tree_step(w, 4, w.rng)
    masks = [draft.ancestors(random_tree(w.rng, n, 2)) for n in w.new]
    want = run_tree(w, q, 4, masks, 0.125)
    for bad in (-1, w.P, 2 ** 31 - 1, -2 ** 31):
        keep = w.tables[1, 2]
        w.tables[1, 2] = bad
        got = run_tree(w, q, 4, masks, 0.125)
        w.tables[1, 2] = keep
        assert torch.equal(got[:9], want[:9]) and torch.equal(got[21:], want[21:])


def test_large_scores_and_long_lags():
    """Scores that climb along the cache, so that the running maximum moves often, and some far below it."""
    w = World((2000,), (7,), 2, 128, 29)
    w.pool[:] = kv_layout.new_pool(1, w.P, 2, 128, NAN_BITS[BF16])
    ramp = (np.linspace(0.05, 6, 2000) * np.where(np.arange(2000) % 5, 1, 0.3))[:, None, None]
    k = bits(torch.from_numpy(w.rng.standard_normal((2000, 2, 128)) * 0.3 + ramp).to(BF16))
    w.put(0, [0], [0, 2000], k, w.v_old)
    q = tree_step(w, 6, w.rng, 1.0) + 0.5
    masks = [draft.ancestors(random_tree(w.rng, 7, 3))]
    check_tree(w, q, 6, masks, 128 ** -0.5, run_tree(w, q, 6, masks, 128 ** -0.5))


# ------------------------------------------------------------------------------ verification

class Drafts:
    """Trees of drafts with the target's and the draft model's rows."""

    def __init__(self, new, vocab, drawn, seed, width=3, sharp=3.0, stride=None, chains=False):
        self.rng = rng = np.random.default_rng(seed)
        self.new, self.vocab, self.drawn = list(new), vocab, drawn
        self.cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        T = int(self.cu[-1])
        soft = lambda x: (np.exp(x - x.max(-1, keepdims=True)) / np.exp(x - x.max(-1, keepdims=True)).sum(-1, keepdims=True)).astype(np.float32)  # noqa: E731
        x = rng.standard_normal((T, vocab)) * sharp
        self.p, self.q = soft(x), soft(x + rng.standard_normal((T, vocab)))
        self.parents = np.concatenate([[]] + [[-1, *range(n - 1)] if chains else random_tree(rng, n, width) for n in new if n]).astype(np.int32)
        self.tokens = np.zeros(T, np.int32)
        for s, n in enumerate(new):
            for i in range(1, n):
                row = self.q[self.cu[s] + self.parents[self.cu[s] + i]].astype(np.float64)
                order = np.argsort(-row)
                self.tokens[self.cu[s] + i] = rng.choice(vocab, p=row / row.sum()) if drawn else order[min(vocab - 1, int(rng.integers(0, 4)))]
        self.u, self.u_next = rng.random(T).astype(np.float32), rng.random(len(new)).astype(np.float32)
        self.stride = stride or vocab

    def rows(self, x):
        wide = torch.full((x.shape[0], self.stride), float("nan"))
        wide[:, :self.vocab] = torch.from_numpy(x)
        return wide.cuda()[:, :self.vocab]

    def batch(self):
        S = len(self.new)
        return cs.Batch(torch.zeros((S, 64), dtype=torch.int32), torch.zeros(S, dtype=torch.int32), torch.from_numpy(self.cu))

    def device(self, chains=False):
        T, S = len(self.tokens), len(self.new)
        full = lambda n: torch.full((n + 2,), -9, dtype=torch.int32, device="cuda")  # noqa: E731
        ints = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
        batch = self.batch()
        ws = cs.workspace_for_verify(batch, self.vocab)
        ws.fill_(255)
        return [batch, ints(self.tokens), None if chains else ints(self.parents), self.rows(self.p), self.rows(self.q) if self.drawn else None, ints(self.u), ints(self.u_next),
                full(T), full(T), full(S), ws]

    def check(self, args):
        tokens, path, count = (x.cpu().numpy() for x in args[7:10])
        T, S = len(self.tokens), len(self.new)
        assert np.all(tokens[T:] == -9) and np.all(path[T:] == -9) and np.all(count[S:] == -9)
        lens = []
        for s, n in enumerate(self.new):
            a, b = self.cu[s], self.cu[s + 1]
            if n == 0:
                assert count[s] == 0
                continue
            want_path, want = draft.ref_verify(self.tokens[a:b], self.parents[a:b], self.p[a:b], self.q[a:b] if self.drawn else None, self.u[a:b], self.u_next[s])
            assert count[s] == len(want), (s, path[a:b], want_path)
            assert path[a:b].tolist() == want_path + [-1] * (n - len(want)), s
            assert tokens[a:b].tolist() == want + [-1] * (n - len(want)), s
            lens.append(len(want))
        return lens

    def run(self, chains=False):
        args = self.device(chains)
        cs.cs_spec_verify(*args)
        return self.check(args)


@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("vocab", [1, 3, 1000, 1024, 1025, 8193, 50257])
def test_verification(vocab, drawn):
    d = Drafts((1, 7, 0, 16, 2, 30), vocab, drawn, vocab, sharp=1.0 if vocab < 10 else 3.0)
    d.run()


@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("new", [(1,), (64,), (65,), (256, 3), (130, 200)])
def test_verification_of_large_trees(new, drawn):
    Drafts(new, 700, drawn, 31, width=6, sharp=1.5).run()


@pytest.mark.parametrize("drawn", [False, True])
def test_verification_of_many_sequences_and_rows_that_lie_apart(drawn):
    lens = Drafts(np.random.default_rng(32).integers(0, 7, 3000).tolist(), 130, drawn, 33, sharp=1.0).run()
    assert len(set(lens)) > 2                                    # walks of several lengths
    Drafts((5, 1, 9), 5001, drawn, 34, stride=5003).run()
    Drafts([6] * 40, 1027, drawn, 35, stride=1031, chains=True).run(chains=True)


@pytest.mark.parametrize("drawn", [False, True])
def test_verification_on_borders(drawn):
    """Probabilities and random numbers that are eighths: every sum is exact, and comparisons meet their borders."""
    for seed in range(4):
        d = Drafts([9] * 60, 11, drawn, 40 + seed, width=2)
        eighths = lambda n: (np.stack([d.rng.multinomial(8, np.ones(11) / 11) for _ in range(n)]) / 8).astype(np.float32)  # noqa: E731
        d.p, d.q = eighths(540), eighths(540)
        d.u, d.u_next = (d.rng.integers(0, 8, 540) / 8).astype(np.float32), (d.rng.integers(0, 8, 60) / 8).astype(np.float32)
        d.run()


@pytest.mark.parametrize("drawn", [False, True])
def test_verification_of_rows_with_little_in_them(drawn):
    vocab = 4000
    d = Drafts([4] * 24, vocab, drawn, 50)
    p = d.p.reshape(24, 4, vocab)
    p[0] = 0                                                      # nothing: no token
    p[1] = np.nan
    p[2, :, 100:] = 0                                             # the end of the row has nothing
    p[3, :, :vocab - 1] = 0
    p[4, :, 7] = np.nan
    p[5] = -1
    p[6, :, ::2] = -0.5
    d.q.reshape(24, 4, vocab)[7] = p[7]                           # the same rows: nothing is left after a refusal
    d.u.reshape(24, 4)[7] = 2.0
    d.u_next[8], d.u_next[9], d.u_next[10] = 0.0, 1.0, 5.0
    d.tokens.reshape(24, 4)[11] = [0, -1, vocab, 2 ** 31 - 1]     # outside the vocabulary
    d.tokens.reshape(24, 4)[12] = 17                              # the same token again and again
    d.parents.reshape(24, 4)[12] = [-1, 0, 0, 0]
    d.parents.reshape(24, 4)[13] = [-1, 1, 3, 2 ** 31 - 1]        # no parents: never reached
    d.parents.reshape(24, 4)[14] = [5, 0, -7, 2]                  # (node 0's entry is not read)
    d.u[52:60] = 0.0
    args = d.device()
    cs.cs_spec_verify(*args)
    d.parents.reshape(24, 4)[13] = [-1, -1, -1, -1]               # as the oracle knows them
    d.parents.reshape(24, 4)[14] = [-1, 0, -1, -1]
    d.check(args)


@pytest.mark.parametrize("vocab", [900, 50257])
def test_verification_leaves_unread_what_a_leaf_has_no_drafts_from(vocab):
    """Rows of q behind nodes without children were never filled; neither were rows of p that no walk reaches."""
    d = Drafts((6, 1, 30, 2), vocab, True, 58)
    leaf = np.ones(len(d.tokens), bool)
    for s, n in enumerate(d.new):
        leaf[[d.cu[s] + p for p in d.parents[d.cu[s] + 1:d.cu[s] + n]]] = False
    d.u[::2] = 0.0                                                # walks that end at leaves
    d.q[leaf] = np.nan
    assert max(d.run()) > 2


# ------------------------------------------------------------------------------------ commit

@pytest.mark.parametrize("page_size", [16, 8])
@pytest.mark.parametrize("Hkv,D", [(2, 64), (1, 64), (3, 128), (8, 128)])
def test_commit(Hkv, D, page_size):
    ctx, new = (0, 5, 16, 40, 7, 100, 3), (1, 17, 64, 0, 256, 9, 30)
    w = World(ctx, new, Hkv, D, 61, BF16, page_size, layers=3, pad=8)
    for layer in range(3):
        w.append(w.rows(w.T, Hkv), w.rows(w.T, Hkv), layer)
    paths = [[0], sorted([0, *w.rng.choice(np.arange(1, 17), 9, replace=False)]), [0, *range(2, 64)], [], sorted([0, *w.rng.choice(np.arange(1, 256), 150, replace=False)]), list(range(9)), [0, 29]]
    path = np.full(w.T, -1, np.int32)
    for t0, p in zip(w.cu, paths):
        path[t0:t0 + len(p)] = p
    count = torch.tensor([len(p) for p in paths], dtype=torch.int32).cuda()
    pool, t = w.device_pool()
    cs.cs_kv_tree_commit(pool, 1, 3, w.batch(), torch.from_numpy(path).cuda(), count)
    slot = lambda s, i: int(w.tables[s, (ctx[s] + i) // page_size]) * page_size + (ctx[s] + i) % page_size  # noqa: E731
    src = [slot(s, n) for s, p in enumerate(paths) for n in p]
    dst = [slot(s, k) for s, p in enumerate(paths) for k in range(len(p))]
    rows = kv_layout.ref_gather_tokens(w.pool, 1, 3, src, page_size=page_size)
    kv_layout.ref_restore_tokens(w.pool, 1, 3, dst, rows, page_size=page_size)
    assert np.array_equal(w.host_pool(t), w.pool)


def test_commit_leaves_out_what_is_not_there():
    w = World((20, 20, 20), (40, 12, 12), 2, 64, 62)
    w.append(w.rows(w.T, 2), w.rows(w.T, 2))
    path = np.full(w.T, -1, np.int32)
    path[:4] = [0, 2, 40, 2 ** 31 - 1]                             # nodes that the sequence does not have
    path[40:43] = [0, -5, 3]
    path[52:54] = [0, 11]
    keep = w.tables[2, 1]
    w.tables[2, 1] = w.P                                           # the last node's page is no page
    pool, t = w.device_pool()
    cs.cs_kv_tree_commit(pool, 0, 1, w.batch(), torch.from_numpy(path).cuda(), torch.tensor([99, 3, 2], dtype=torch.int32).cuda())
    w.tables[2, 1] = keep
    slot = lambda s, i: int(w.tables[s, (20 + i) // 16]) * 16 + (20 + i) % 16  # noqa: E731
    rows = kv_layout.ref_gather_tokens(w.pool, 0, 1, [slot(0, 2), slot(1, 3)])
    kv_layout.ref_restore_tokens(w.pool, 0, 1, [slot(0, 1), slot(1, 2)], rows)
    assert np.array_equal(w.host_pool(t), w.pool)


# ------------------------------------------------------------------------------- a run of them

@pytest.mark.parametrize("dtype", [BF16, F16])
def test_steps_of_speculation_leave_the_cache_of_plain_decoding(dtype):
    """Three steps, two layers, all five calls: the accepted tokens' keys, values and attention are those of tokens appended one after another, and trees
    after a commit see nothing of what was refused."""
    L, Hq, Hkv, D, vocab, steps = 2, 8, 2, 64, 300, 3
    rng = np.random.default_rng(71)
    ctx, S = np.array([37, 5, 64]), 3
    blocks = 16
    tables = rng.permutation(S * blocks).astype(np.int32).reshape(S, blocks)
    inv = torch.from_numpy((1e4 ** (-np.arange(32) / 32)).astype(np.float32)).cuda()
    # a model of tables: a token's Q, K, V rows in each layer, and the distribution behind it
    emb = torch.from_numpy(rng.standard_normal((L, vocab, Hq + 2 * Hkv, D))).to(dtype).cuda()
    rows = torch.softmax(torch.from_numpy(rng.standard_normal((vocab, vocab)) * 3).float(), -1).cuda()
    drafts = torch.softmax(torch.log(rows) + torch.from_numpy(rng.standard_normal((vocab, vocab))).float().cuda(), -1)
    def fresh():
        return cs.Pool(torch.full((L, S * blocks, 2, Hkv, 16 * D), float("nan"), dtype=dtype, device="cuda"), L, S * blocks, Hkv, D)
    pool, plain = fresh(), fresh()
    said = [rng.integers(0, vocab, c + 1).tolist() for c in ctx]      # the last one is not cached yet
    def batch_of(c, n):
        cu = torch.zeros(S + 1, dtype=torch.int32)
        cu[1:] = torch.cumsum(torch.tensor(n), 0)
        return cs.Batch(torch.from_numpy(tables), torch.tensor(c, dtype=torch.int32), cu)
    def append(pool, layer, batch, rope, x):
        q_out = torch.empty((x.shape[0], Hq, D), dtype=dtype, device="cuda")
        fn("cs_kv_append_rope", dtype)(pool, layer, batch, rope, x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], q_out)
        return q_out
    for p in (pool, plain):
        first = torch.tensor([t for s in said for t in s[:-1]]).cuda()
        for layer in range(L):
            append(p, layer, batch_of([0] * S, ctx.tolist()), cs.Rope(inv, D), emb[layer, first])
    done = ctx.copy()
    for step in range(steps):
        new = rng.integers(2, 20, S)
        trees = [random_tree(rng, int(n), 3) for n in new]
        batch = batch_of(done.tolist(), new.tolist())
        cu = batch.h_cu.tolist()
        tokens = np.zeros(cu[-1], np.int64)
        for s, t in enumerate(trees):
            tokens[cu[s]] = said[s][-1]
            for i in range(1, len(t)):
                row = drafts[tokens[cu[s] + t[i]]].double().cpu().numpy()
                tokens[cu[s] + i] = rng.choice(vocab, p=row / row.sum())
        depth = [[len(np.nonzero(r)[0]) - 1 for r in draft.ancestors(t)] for t in trees]
        at = torch.tensor([int(done[s]) + d for s in range(S) for d in depth[s]], dtype=torch.int32).cuda()
        ids = torch.from_numpy(tokens).cuda()
        mask = torch.from_numpy(np.concatenate([draft.mask_words(draft.ancestors(t), 1) for t in trees])).cuda()
        rope, ws, outs = cs.Rope(inv, D, at), cs.workspace_for_tree(batch, Hq, Hkv, D), []
        for layer in range(L):
            q_out = append(pool, layer, batch, rope, emb[layer, ids])
            out = torch.empty_like(q_out)
            fn("cs_paged_attention_tree", dtype)(pool, layer, batch, q_out, out, Hq, 0.125, mask, ws)
            outs.append(out)
        path, got, count = (torch.empty(n, dtype=torch.int32, device="cuda") for n in (cu[-1], cu[-1], S))
        cs.cs_spec_verify(batch, ids.to(torch.int32), torch.tensor([p for t in trees for p in t], dtype=torch.int32).cuda(), rows[ids], drafts[ids], torch.from_numpy(rng.random(cu[-1])).float().cuda(),
                          torch.from_numpy(rng.random(S)).float().cuda(), got, path, count, cs.workspace_for_verify(batch, vocab))
        cs.cs_kv_tree_commit(pool, 0, L, batch, path, count)
        path, got, count = path.cpu().numpy(), got.cpu().numpy(), count.cpu().numpy()
        # the same tokens one after another
        chain = [[said[s][-1], *got[cu[s]:cu[s] + count[s] - 1].tolist()] for s in range(S)]
        b2 = batch_of(done.tolist(), count.tolist())
        ids2 = torch.tensor([t for c in chain for t in c]).cuda()
        for layer in range(L):
            q_out = append(plain, layer, b2, cs.Rope(inv, D), emb[layer, ids2])
            want = torch.empty_like(q_out)
            fn("cs_paged_attention_mixed", dtype)(plain, layer, b2, q_out, want, Hq, 0.125, cs.workspace_for(b2, Hq, Hkv, D))
            kept = torch.cat([outs[layer][cu[s] + torch.from_numpy(path[cu[s]:cu[s] + count[s]]).long().cuda()] for s in range(S)])
            # either rounds weights and results once: twice the bound of one, with |V| at most 5 and weights that sum to 1
            assert (kept.double() - want.double()).abs().max() <= 2 * (2 * HALF_STEP[dtype] + HALF_STEP[dtype]) * 5
        for s in range(S):
            said[s] += got[cu[s]:cu[s] + count[s]].tolist()
        done += count
        assert [len(x) - 1 for x in said] == done.tolist()
        a, b = bits(pool.tensor), bits(plain.tensor)
        for layer in range(L):
            for s in range(S):
                for x, y in zip(*(kv_layout.read_logical(z, layer, tables[s], int(done[s])) for z in (a, b))):
                    assert np.array_equal(x, y), (step, layer, s)
    assert done.sum() > ctx.sum() + S * steps                     # some drafts were accepted


# -------------------------------------------------------------------- streams, graphs, repetition

def all_calls(seed, like=None):
    """One step's five calls on prepared memory, and its outputs.  like: another one's, whose workspaces it takes."""
    w = World((2500, 40, 9), (12, 5, 1), 2, 64, seed)
    rng = w.rng
    rope, _, _, _ = make_rope(rng, w.T, 64, 64, False, True, 1, BF16)
    x = torch.from_numpy(rng.standard_normal((w.T, 12, 64))).to(BF16).cuda()
    pool, t = w.device_pool()
    batch, q_out, k_out = w.batch(), torch.zeros((w.T, 8, 64), dtype=BF16, device="cuda"), torch.zeros((w.T, 2, 64), dtype=BF16, device="cuda")
    out, ws = torch.zeros_like(q_out), cs.workspace_for_tree(batch, 8, 2, 64) if like is None else like[2][4]
    if like is None:
        ws.fill_(255)
    mask = torch.from_numpy(np.concatenate([draft.mask_words(draft.ancestors(random_tree(rng, n, 3)), 1) for n in w.new])).cuda()
    d = Drafts(w.new, 40000, True, seed)                          # (rows that several workgroups sum)
    v = d.device()
    if like is not None:
        v[10] = like[2][3][10]

    def step():
        cs.cs_qk_rope(rope, x[:, :8], x[:, 8:10], q_out, k_out)
        cs.cs_kv_append_rope(pool, 0, batch, rope, x[:, :8], x[:, 8:10], x[:, 10:], q_out)
        cs.cs_paged_attention_tree(pool, 0, batch, q_out, out, 8, 0.125, mask, ws)
        cs.cs_spec_verify(*v)
        cs.cs_kv_tree_commit(pool, 0, 1, batch, v[8], v[9])
    return step, [q_out, k_out, out, v[7][:w.T], v[8][:w.T], v[9][:3], t], (w, batch, d, v, ws)


def clear(outs):
    for o in outs[:-1]:
        o.zero_()


def test_captured_and_replayed():
    step, outs, keep = all_calls(81)
    step()
    torch.cuda.synchronize()
    want = [o.clone() for o in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(4):
        clear(outs)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
        clear(outs)
        step()                                                    # the program's own work between replays
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
    keep[2].check(keep[3])


def test_two_graphs_that_share_their_workspaces():
    first = all_calls(85)
    runs = [first, all_calls(86, first)]
    want, graphs = [], []
    for step, outs, _ in runs:
        step()
        torch.cuda.synchronize()
        want.append([o.clone() for o in outs])
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            step()
    for i in (0, 1, 1, 0, 0, 1, 0, 1):
        clear(runs[i][1])
        graphs[i].replay()
        runs[1 - i][0]()                                          # and the other one's calls behind it
        torch.cuda.synchronize()
        for (_, outs, _), w in zip(runs, want):
            assert all(torch.equal(a, b) for a, b in zip(outs, w))


def test_two_streams_at_once():
    runs = [all_calls(82), all_calls(83)]
    for step, _, _ in runs:
        step()
    torch.cuda.synchronize()
    want = [[o.clone() for o in outs] for _, outs, _ in runs]
    for _, outs, _ in runs:
        clear(outs)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for (step, _, _), stream in zip(runs, streams):
            with torch.cuda.stream(stream):
                step()
    torch.cuda.synchronize()
    for (_, outs, _), w in zip(runs, want):
        assert all(torch.equal(a, b) for a, b in zip(outs, w))


def test_the_same_bits_every_time():
    step, outs, _ = all_calls(84)
    step()
    want = [o.clone() for o in outs]
    for _ in range(20):
        step()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))


@pytest.mark.parametrize("vocab", [6, 40, 3000, 50257])
def test_verification_takes_malformed_elements_of_either_row_as_nothing(vocab):
    """Negative elements, infinities below zero and NaN (signalling ones among them), in p and in q, at drafted tokens and elsewhere: as if they were 0."""
    d = Drafts([9] * (40 if vocab < 5000 else 6), vocab, True, 90 + vocab, width=2, sharp=1.0)
    clean = []
    for x in (d.p, d.q):
        kind, at = d.rng.integers(0, 6, x.shape), d.rng.random(x.shape) < 0.3
        for s, n in enumerate(d.new):                             # half of the drafts' own elements
            for i in range(1, n):
                t = d.cu[s] + i
                at[d.cu[s] + d.parents[t], d.tokens[t]] = d.rng.random() < 0.5
        for k, bad in enumerate((np.float32(-0.0), np.float32(-np.inf), np.float32(np.nan), np.uint32(0x7FA00001).view(np.float32))):
            x.view(np.uint32)[at & (kind == k)] = np.asarray(bad).view(np.uint32)
        x[at & (kind > 3)] *= -2
        clean.append(np.where(at, np.float32(0), x))
    args = d.device()
    cs.cs_spec_verify(*args)
    lens = d.check(args)                                          # as the header has it
    d.p, d.q = clean
    assert lens == d.check(args) and sum(lens) > len(lens)           # and as rows that hold zeros there


def test_a_draft_that_the_target_never_has_is_refused_however_negative_q_is():
    d = Drafts([3] * 8, 20, True, 91)
    d.p[:], d.q[:] = 0.0, 1.0 / 20
    d.p[:, 7] = 1.0
    d.tokens[:], d.parents[:] = 3, np.tile([-1, 0, 1], 8)
    d.q[::3, 3] = [-1.0, -0.25, -1e-30, -np.inf, -3e38, -0.0, np.nan, 0.25]
    args = d.device()
    cs.cs_spec_verify(*args)
    assert args[9][:8].tolist() == [1] * 8 and args[7][:24:3].tolist() == [7] * 8


@pytest.mark.parametrize("drawn", [False, True])
def test_what_has_no_probability_is_refused_whatever_the_random_number_is(drawn):
    """Random numbers below 0, and guesses whose refusals take more than 1 from a row: the bar is negative, and nothing is left of the token."""
    vocab, outside = 9, [-1, 9, 2 ** 31 - 1, -2 ** 31]
    d = Drafts([2] * 5 + [4] * 4, vocab, drawn, 92)
    d.p[:], d.q[:] = 0.0, 1.0 / vocab
    d.p[:, 2] = 1.0
    d.u[:] = -1.0
    for s in range(5):
        d.tokens[2 * s + 1] = outside[s] if s < 4 else 5          # 5: inside, but the target never has it
        d.parents[2 * s:2 * s + 2] = [-1, 0]
    for s in range(4):                                            # children 2 and 4 have 0.75 each of a row, the third one nothing
        t = 10 + 4 * s
        d.p[t] = 0.0
        d.p[t, [2, 4]] = 0.75
        d.tokens[t:t + 4] = [0, 2, 4, outside[s]]
        d.parents[t:t + 4] = [-1, 0, 0, 0]
        d.u[t:t + 4] = 20.0
    d.u_next[:] = 0.0
    args = d.device()
    cs.cs_spec_verify(*args)
    assert args[9][:9].tolist() == [1] * 9
    assert args[7][:10:2].tolist() == [2] * 5 and args[7][10:26:4].tolist() == [2] * 4
    d.check(args)


def infinitely_far(w, s, first, end, value):
    """K of the keys first .. end - 1 of sequence s gets `value` as its first feature, in every head: all of their scores are -infinity for queries
    with a positive one there."""
    for key in range(first, end):
        w.pool[w.layer, w.tables[s, key // w.ps], 0, :, kv_layout.k_index(key % w.ps, 0, w.D, page_size=w.ps)] = value


def near_without(w, q, Hq, masks, scale, got, first, end):
    """The keys first .. end - 1 of each sequence's cached ones weigh nothing: exp(-infinity - m) for a finite m."""
    for s in range(len(w.ctx)):
        n, t0 = w.new[s], int(w.cu[s])
        k, v = (np.concatenate([x[:first[s]], x[end[s]:]]) for x in w.logical(s))
        seen = np.tril(np.ones((n, n), bool)) if masks is None else masks[s][:, :n]
        want, tol = draft.ref_tree_attention(q[t0:t0 + n].double().numpy(), k, v, seen, scale, HALF_STEP[w.dtype], w.dtype == F16)
        near(got[t0:t0 + n].double().numpy(), want, tol, (s, w.ctx[s], n))


# -infinity, and for bf16 a finite one whose products with q are below the least float
NEGATIVE = [(BF16, 0xFF80), (F16, 0xFC00), (BF16, 0xFF7F)]


@pytest.mark.parametrize("dtype,value", NEGATIVE)
@pytest.mark.parametrize("page_size", [16, 8])
@pytest.mark.parametrize("Hq,Hkv,D,ctx,new,first,end", [
    (4, 2, 64, (400, 300), (4, 2), (0, 0), (200, 160)),           # wavefronts that share the keys, whose first steps hold nothing else
    (16, 2, 128, (400, 300), (3, 1), (0, 40), (200, 290)),
    (8, 2, 64, (400, 90), (40, 9), (0, 3), (200, 90)),            # that share the rows
    (16, 2, 128, (300, 0), (60, 5), (0, 0), (300, 0)),            # one to three tiles each; nodes see nothing else but nodes
    (4, 2, 128, (9000, 3), (4, 1), (0, 0), (6000, 3)),            # whole pieces of a cut sequence
    (32, 2, 64, (9000,), (30,), (100,), (8990,)),
])
def test_keys_infinitely_far_weigh_nothing(Hq, Hkv, D, ctx, new, first, end, page_size, dtype, value):
    w = World(ctx, new, Hkv, D, 93, dtype, page_size)
    q = tree_step(w, Hq, w.rng)
    q[..., 0] = q[..., 0].abs() + 1.5
    for s in range(len(ctx)):
        infinitely_far(w, s, first[s], end[s], value)
    masks = [draft.ancestors(random_tree(w.rng, n, 4)) for n in new]
    near_without(w, q, Hq, masks, 2.0, run_tree(w, q, Hq, masks, 2.0), first, end)


@pytest.mark.parametrize("dtype,value", NEGATIVE)
@pytest.mark.parametrize("page_size", [16, 8])
@pytest.mark.parametrize("Hq,Hkv,D,ctx,new,first,end", [
    (4, 2, 64, (400, 300, 5), (1, 1, 1), (0, 0, 0), (200, 160, 5)),
    (16, 2, 128, (400, 77), (1, 1), (0, 3), (390, 70)),
    (4, 2, 128, (20000, 3), (1, 1), (0, 0), (15000, 2)),          # whole pieces
    (4, 2, 128, (400, 300), (1, 1), (0, 0), (200, 300)),          # nothing but the token itself is left
    (4, 2, 128, (400, 900, 300), (1, 1, 40), (0, 20, 0), (200, 880, 0)),   # beside a chunk
])
def test_decode_gives_keys_infinitely_far_no_weight(Hq, Hkv, D, ctx, new, first, end, page_size, dtype, value):
    w = World(ctx, new, Hkv, D, 94, dtype, page_size)
    q = tree_step(w, Hq, w.rng)
    q[..., 0] = q[..., 0].abs() + 1.5
    for s in range(len(ctx)):
        infinitely_far(w, s, first[s], end[s], value)
    pool, _ = w.device_pool()
    batch, out = w.batch(), torch.full_like(q, 9.0).cuda()
    fn("cs_paged_attention_mixed", dtype)(pool, 0, batch, q.cuda(), out, Hq, 2.0, cs.workspace_for(batch, Hq, Hkv, D))
    w.ctx, w.new = ([x for x, n in zip(y, new) if n == 1] for y in (ctx, new))   # (the chunk's Q is scaled before it is rounded: a bound of its own)
    near_without(w, q, Hq, None, 2.0, out.cpu(), first, end)


@pytest.mark.parametrize("Hq,D,ctx", [(4, 64, (400, 192)), (16, 128, (400, 250)), (4, 128, (20000, 192))])
def test_decode_over_8_bits_gives_keys_infinitely_far_no_weight(Hq, D, ctx):
    """Codes hold no infinity: K near the greatest bf16, whose products with q are below the least float."""
    import test_gpu_kv8
    w, first = test_gpu_kv8.World(ctx, [1] * len(ctx), 2, D, 97), 192
    cu = np.concatenate([[0], np.cumsum(ctx)]).astype(np.int32)
    k, v = w.rows(int(cu[-1])), w.rows(int(cu[-1]))
    for t in cu[:-1]:
        k[t:t + first, :, 0] = -3.0e38
    w.pool[:] = test_gpu_kv8.NAN_CODE
    test_gpu_kv8.kv8.ref_append(w.pool, 0, w.tables, [0] * len(ctx), cu, k, v, 2, D)
    _, w.pool = w.append(w.rows(w.T), w.rows(w.T))
    q = torch.from_numpy(w.rng.standard_normal((w.T, Hq, D))).to(BF16)
    q[..., 0] = q[..., 0].abs() + 1.5
    batch, out = w.batch(), torch.full_like(q, 9.0).cuda()
    cs.cs_paged_attention_mixed_kv8(w.handle(torch.from_numpy(w.pool).cuda()), 0, batch, q.cuda(), out, Hq, 0.5, cs.workspace_for_kv8(batch, Hq, 2, D))
    for s, c in enumerate(ctx):
        K, V = (x[first:] for x in test_gpu_kv8.kv8.read_logical(w.pool, 0, w.tables[s], c + 1, 2, D))
        want, tol = draft.ref_tree_attention(q[s:s + 1].double().numpy(), K, V, np.ones((1, 1), bool), 0.5, HALF_STEP[BF16], False)
        near(out[s:s + 1].cpu().double().numpy(), want, tol, (s, c))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("Hq,Hkv,D,ctx,new", [
    (4, 2, 64, (70, 0, 133), (8, 6, 5)), (16, 2, 128, (70, 200), (4, 3)), (8, 2, 64, (70, 0), (40, 30)), (8, 2, 128, (100, 260), (70, 100)), (8, 1, 128, (6000,), (60,)), (4, 2, 64, (5000,), (8,)),
])
def test_keys_that_a_row_does_not_see_change_no_bit_of_it(Hq, Hkv, D, ctx, new, dtype):
    """Nodes whose K lies far out, finite or infinite in one feature: their descendants' scores climb, and rows beside them in the same tile stay as they were."""
    w = World(ctx, new, Hkv, D, 95, dtype)
    q = tree_step(w, Hq, w.rng, 2.0)
    masks = [draft.ancestors(random_tree(w.rng, n, 6)) for n in new]
    scale = 0.7 * D ** -0.5
    clean, tables, pool = run_tree(w, q, Hq, masks, scale), w.tables, w.pool.copy()
    apart = 0
    for node in range(1, max(new), 3):
        for what in ("large", "infinite"):
            w.pool = pool.copy()
            for s, n in enumerate(new):
                if node < n:
                    at = ctx[s] + node
                    block, index = w.pool[0, tables[s, at // 16], 0], kv_layout.k_index(at % 16, np.arange(D), D)
                    if what == "large":
                        block[:, index] = bits(tensor(block[:, index], dtype) * 30)
                    else:
                        block[:, index[3]] = 0x7F80 if dtype == BF16 else 0x7C00
            got = run_tree(w, q, Hq, masks, scale)
            for s, n in enumerate(new):
                for i in range(n):
                    if node >= n or not masks[s][i, node]:
                        assert torch.equal(got[int(w.cu[s]) + i], clean[int(w.cu[s]) + i]), (node, what, s, i)
                        apart += 1
    assert apart >= sum(new)                                      # (there were such rows)


@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("vocab", [65536, 65537, 128256, 151936, 1 << 20])
def test_verification_of_long_rows(vocab, drawn):
    """More than 64 blocks of 1024 elements: draws that fall into every group of 64 and on their borders, rows that have something in one group only, and
    random numbers that no running sum passes."""
    groups = -(-vocab // 65536)
    d = Drafts([2] * 7, vocab, drawn, 96, sharp=1.0)
    d.u_next[:] = [0.0, 0.02, 0.51, 0.97, 1.0 - 2.0 ** -24, 1.0, 3.0]
    d.run()
    d.u[:] = 2.0                                                  # every draft is refused
    d.run()
    # a few elements, of weights that are exact, on both sides of the groups' borders
    at = sorted({x for g in range(groups + 1) for x in (65536 * g - 1024, 65536 * g - 1, 65536 * g, 65536 * g + 1023) if 0 <= x < vocab} | {0, vocab - 1})
    d.p[:], d.q[:] = 0.0, 0.0
    d.q[:, 5] = 1.0
    d.p[:, at] = 1.0 / 64
    d.tokens[:] = 5
    d.u_next[:] = [0.0, *((np.arange(1, 6) * len(at) // 6 + 0.0) / len(at)), 1.0 - 2.0 ** -24]
    d.run()
    for only in at[::5] + [vocab - 1]:                            # all of it at one place
        d.p[:] = 0.0
        d.p[:, only] = 0.5
        d.u_next[:] = [0.0, 0.3, 0.5, 0.9, 1.0, 2.0, 0.1]
        args = d.device()
        cs.cs_spec_verify(*args)
        d.check(args)
        assert args[7][:14:2].tolist() == [only] * 7


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_trees_beside_prompt_chunks_take_a_batch_each(dtype):
    """A step of online trees and offline chunks: one append, the trees' attention on a prefix of the batch, the chunks' on a batch of the rest."""
    Hq, Hkv, D, ctx, new, trees = 8, 2, 64, (70, 5, 0, 40), (12, 1, 300, 260), 2
    w = World(ctx, new, Hkv, D, 98, dtype)
    rope, _, _, _ = make_rope(w.rng, w.T, D, D, False, False, 1, dtype)
    x = torch.from_numpy(w.rng.standard_normal((w.T, Hq + 2 * Hkv, D))).to(dtype).cuda()
    pool, t = w.device_pool()
    batch, t0 = w.batch(), int(w.cu[trees])
    q, out = (torch.full((w.T, Hq, D), 9.0, dtype=dtype, device="cuda") for _ in range(2))
    fn("cs_kv_append_rope", dtype)(pool, 0, batch, rope, x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], q)
    online = batch.truncated(trees)
    offline = cs.Batch(torch.from_numpy(w.tables[trees:]), torch.tensor(ctx[trees:]), torch.from_numpy(w.cu[trees:] - t0))
    masks = [draft.ancestors(random_tree(w.rng, n, 3)) for n in new[:trees]] + [np.tril(np.ones((n, n), bool)) for n in new[trees:]]
    words = torch.from_numpy(np.concatenate([draft.mask_words(m, 1) for m in masks[:trees]])).cuda()
    with pytest.raises(cs.CsError) as refused:
        fn("cs_paged_attention_tree", dtype)(pool, 0, batch, q, out, Hq, 0.1, None, None)
    assert refused.value.status == cs.CS_ERR_UNSUPPORTED
    fn("cs_paged_attention_tree", dtype)(pool, 0, online, q, out, Hq, 0.1, words, cs.workspace_for_tree(online, Hq, Hkv, D))
    assert torch.all(out[t0:] == 9.0)
    fn("cs_paged_attention_mixed", dtype)(pool, 0, offline, q[t0:], out[t0:], Hq, 0.1, cs.workspace_for(offline, Hq, Hkv, D))
    w.pool = w.host_pool(t)
    check_tree(w, q.cpu(), Hq, masks, 0.1, out.cpu())
