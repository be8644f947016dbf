"""Page copies, forks, frees and compaction on the GPU against plain loops, byte for byte; and a serving loop that uses them
with the 8-bit append and attention."""
import numpy as np
import pytest
import torch

from oracle import kv8
from paper_2410_01228_amd import binding as cs

pytestmark = pytest.mark.gpu


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


def space_of(array, page_bytes):
    """(PageSpace over a device copy of uint8 [layers][pages][stride], that copy)"""
    t = torch.from_numpy(array).cuda()
    L, P, stride = array.shape
    return cs.PageSpace(t, cs.cs_page_space(t.data_ptr(), L, P, page_bytes, P * stride, stride)), t


def noise(r, L, P, stride):
    return r.integers(0, 256, (L, P, stride), dtype=np.uint8)


@pytest.mark.parametrize("page_bytes,stride", [(16, 16), (16, 64), (1024, 1024), (1040, 1056), (4112, 4224), (32832, 32896)])
@pytest.mark.parametrize("n", [1, 2, 37])
def test_copies(n, page_bytes, stride):
    r = np.random.default_rng(n)
    a, b = noise(r, 3, 90, stride), noise(r, 4, 50, stride + 32)
    src, _ = space_of(a, page_bytes)
    dst, t = space_of(b, page_bytes)
    si, di = r.choice(90, n), r.permutation(50)[:n]
    cs.cs_kv_pages_copy(src, 1, dev(si), dst, 2, dev(di), 2)
    b[2:4, di, :page_bytes] = a[1:3, si, :page_bytes]
    assert np.array_equal(t.cpu().numpy(), b)


def test_copies_inside_a_pool_without_lists_and_past_bad_ids():
    r = np.random.default_rng(5)
    a = noise(r, 2, 40, 2048)
    s, t = space_of(a, 2048)
    cs.cs_kv_pages_copy(s, 0, dev([3, -1, 40, 5, 6, 2 ** 31 - 1]), s, 0, dev([20, 21, 22, -7, 24, 25]), 2)
    a[:, 20], a[:, 24] = a[:, 3], a[:, 6]
    assert np.array_equal(t.cpu().numpy(), a)
    # a checkpoint to a staging buffer and back into other pages
    stage = torch.zeros((2, 7, 2048), dtype=torch.uint8, device="cuda")
    ids = r.permutation(20)[:7]
    cs.cs_kv_pages_copy(s, 0, dev(ids), cs.PageSpace.staging(stage), 0, None, 2)
    assert np.array_equal(stage.cpu().numpy(), a[:, ids])
    cs.cs_kv_pages_copy(cs.PageSpace.staging(stage), 0, None, s, 0, dev(30 + np.arange(7)), 2)
    a[:, 30:37] = a[:, ids]
    assert np.array_equal(t.cpu().numpy(), a)
    cs.cs_kv_pages_copy(s, 0, None, s, 0, None, 2, n=0)
    assert np.array_equal(t.cpu().numpy(), a)


def test_an_16_bit_pool_with_pages_of_8():
    pool = cs.Pool.empty(2, 12, 2, 64, page_size=8)
    pool.tensor.normal_()
    before = pool.tensor.clone()
    s = cs.PageSpace.of(pool)
    cs.cs_kv_pages_copy(s, 0, dev([1, 2]), s, 0, dev([8, 9]), 2)
    before[:, 8:10] = before[:, 1:3]
    assert torch.equal(pool.tensor, before)


def world(r, lens, pages, blocks, size=16, shared=0):
    """(tables, lens, counts): rows of these lengths on random pages, the first `shared` pages the same for all that are long enough."""
    perm = list(r.permutation(pages))
    tables = np.full((len(lens), blocks), -1, np.int32)
    common = [perm.pop() for _ in range(shared)]
    for i, n in enumerate(lens):
        for e in range(-(-n // size)):
            tables[i, e] = common[e] if e < shared and (e + 1) * size <= n else perm.pop()
    counts = np.zeros(pages, np.int32)
    np.add.at(counts, tables[tables >= 0], 1)
    return tables, np.array(lens, np.int32), counts, np.array(perm, np.int32)


@pytest.mark.parametrize("size", [8, 16])
@pytest.mark.parametrize("page_bytes", [64, 5008])
def test_forks_and_frees(page_bytes, size):
    r = np.random.default_rng(page_bytes + size)
    lens = [0, 1, size - 1, size, size + 1, 5 * size, 133, 400] + [0] * 14
    tables, lens, counts, spare = world(r, lens, 200, 60, size)
    a = noise(r, 3, 200, page_bytes)
    s, t = space_of(a, page_bytes)
    d = cs.PageTables(dev(tables), dev(lens), dev(counts), size)
    parents = np.array([0, 1, 2, 3, 4, 5, 6, 7, 7, 7, 6], np.int32)
    children = (8 + r.permutation(14)[:11]).astype(np.int32)
    cs.cs_kv_pages_fork(s, 1, 3, d, dev(parents), dev(children), dev(spare[:11]))
    kv8.ref_fork(a, 1, 3, tables, lens, counts, parents, children, spare[:11], size)

    def same():
        assert np.array_equal(t.cpu().numpy(), a)
        for got, want in ((d.block_tables, tables), (d.lens, lens), (d.ref_counts, counts)):
            assert np.array_equal(got.cpu().numpy(), want)
    same()
    freed, number = torch.full((200,), -9, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    for rows in ([children[3]], list(children[5:9]) + [7], [0], [], list(range(8)), list(children)):
        freed.fill_(-9)
        cs.cs_kv_pages_free(d, dev(rows), freed, number)
        want = kv8.ref_free(tables, lens, counts, rows, size)
        same()
        assert int(number) == len(want) and freed.cpu().tolist() == want + [-9] * (200 - len(want))
    assert counts.max() == 0


def test_misused_rows_and_counts_stay_in_bounds():
    r = np.random.default_rng(4)
    tables, lens, counts, spare = world(r, [100, 50, 0, 0], 40, 8)
    d = cs.PageTables(dev(tables), dev(lens), dev(counts))
    a = noise(r, 1, 40, 256)
    s, t = space_of(a, 256)
    freed, number = torch.full((40,), -9, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    # rows that are not there: skipped; no page for the unfinished one: the child ends at its last full page
    cs.cs_kv_pages_fork(s, 0, 1, d, dev([0, 9, 1, -1]), dev([7, 2, 3, 2]), dev([spare[0], spare[1], 40, spare[2]]))
    assert d.lens.cpu().tolist() == [100, 50, 0, 48] and np.array_equal(t.cpu().numpy(), a)
    assert d.block_tables[3].cpu().tolist() == list(tables[1, :3]) + [-1] * 5
    # a row listed twice is freed once
    cs.cs_kv_pages_free(d, dev([3, 3, 17, -2, 3]), freed, number)
    assert int(number) == 0 and np.array_equal(d.ref_counts.cpu().numpy(), counts)
    # entries outside the pool and pages that are free already: left out, whatever else the row holds
    d.block_tables[1, 0], d.block_tables[1, 1] = 40, int(spare[3])
    cs.cs_kv_pages_free(d, dev([1]), freed, number)
    assert freed.cpu().tolist()[:int(number)] == sorted(tables[1, 2:4]) and int(d.ref_counts[int(spare[3])]) == 0
    # a length beyond the row counts as the row
    d.lens[0] = 2 ** 31 - 1
    cs.cs_kv_pages_free(d, dev([0]), freed, number)
    assert freed.cpu().tolist()[:int(number)] == sorted(tables[0, :7]) and d.lens.cpu().tolist() == [0, 0, 0, 0]


@pytest.mark.parametrize("pages,rows,hi,shared", [(1, 1, 16, 0), (7, 1, 50, 0), (64, 3, 200, 1), (3000, 40, 900, 7), (20000, 60, 1500, 3), (20000, 2, 30, 0)])
def test_compaction(pages, rows, hi, shared):
    r = np.random.default_rng(pages + rows)
    lens = [int(x) for x in r.integers(0, hi + 1, rows)]
    tables, lens, counts, _ = world(r, lens, pages, -(-hi // 16) + 1, 16, shared)
    counts[counts == 0] = -(np.arange((counts == 0).sum()) % 2)          # (a count below zero is a free page too)
    a = noise(r, 2, pages, 272)
    s, t = space_of(a, 272)
    want = kv8.ref_compact(a, 0, 2, tables, lens, counts)
    for in_place in (False, True):
        if in_place:
            s, t = space_of(a0, 272)
        else:
            a0 = t.cpu().numpy().copy()
        d = cs.PageTables(dev(tables), dev(lens), dev(counts))
        n = d if in_place else cs.PageTables(torch.full_like(d.block_tables, 77), d.lens, torch.full_like(d.ref_counts, 77))
        ids, used = torch.full((pages,), 77, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        cs.cs_kv_pages_compact(s, 0, 2, d, n, ids, used, cs.compact_workspace_for(s))
        assert np.array_equal(t.cpu().numpy(), a)
        for got, w in zip((n.block_tables, n.ref_counts, ids), want):
            assert np.array_equal(got.cpu().numpy(), w)
        assert int(used) == want[3]
        if not in_place:                                                  # the inputs are as they were
            assert np.array_equal(d.block_tables.cpu().numpy(), tables) and np.array_equal(d.ref_counts.cpu().numpy(), counts)


def test_full_and_empty_pools_do_not_move():
    for counts in (np.ones(9000, np.int32), np.zeros(9000, np.int32)):
        a = noise(np.random.default_rng(1), 1, 9000, 16)
        s, t = space_of(a, 16)
        d = cs.PageTables(dev(np.full((2, 3), -1)), dev([0, 0]), dev(counts))
        ids, used = torch.empty(9000, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        cs.cs_kv_pages_compact(s, 0, 1, d, d, ids, used, cs.compact_workspace_for(s))
        assert int(used) == counts.sum() and np.array_equal(t.cpu().numpy(), a)
        assert np.array_equal(ids.cpu().numpy(), np.where(counts > 0, np.arange(9000), -1)) and np.array_equal(d.ref_counts.cpu().numpy(), counts)


def test_a_pool_beyond_32_bits():
    stride, pages = 1 << 22, 1100                                         # 4.3 GiB
    t = torch.zeros(pages * stride, dtype=torch.uint8, device="cuda")
    view = t.view(pages, stride)
    view[3], view[1090] = 7, 9
    s = cs.PageSpace(t, cs.cs_page_space(t.data_ptr(), 1, pages, stride, pages * stride, stride))
    cs.cs_kv_pages_copy(s, 0, dev([3, 1090]), s, 0, dev([1099, 5]), 1)
    assert (view[1099] == 7).all() and (view[5] == 9).all()
    counts = np.zeros(pages, np.int32)
    counts[[1099, 3]] = 1
    d = cs.PageTables(dev([[3], [1099]]), dev([5, 16]), dev(counts))
    ids, used = torch.empty(pages, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    cs.cs_kv_pages_compact(s, 0, 1, d, d, ids, used, cs.compact_workspace_for(s))
    assert int(used) == 2 and sorted(d.block_tables.view(-1).cpu().tolist()) == [0, 1]
    assert (view[0] == 7).all() and (view[1] == 7).all()


def test_replays_of_a_graph_and_another_stream():
    r = np.random.default_rng(9)
    tables, lens, counts, spare = world(r, [100, 333, 0, 0, 0], 90, 24)
    a = noise(r, 2, 90, 528)
    s, t = space_of(a, 528)
    start = [dev(x) for x in (tables, lens, counts)]
    d = cs.PageTables(*[x.clone() for x in start])
    n = cs.PageTables(torch.zeros_like(d.block_tables), d.lens, torch.zeros_like(d.ref_counts))
    freed, one = torch.full((90,), -9, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    ids, ws = torch.empty(90, dtype=torch.int32, device="cuda"), cs.compact_workspace_for(s)
    lists = [dev(x) for x in ([1, 1, 0], [2, 3, 4], spare[:3], [3, 0])]

    def work(stream=None):
        cs.cs_kv_pages_fork(s, 0, 2, d, *lists[:3], stream)
        cs.cs_kv_pages_free(d, lists[3], freed, one[:1], stream)
        cs.cs_kv_pages_compact(s, 0, 2, d, n, ids, one[1:], ws, stream)

    def reset():
        t.copy_(torch.from_numpy(a))
        for x, y in zip((d.block_tables, d.lens, d.ref_counts), start):
            x.copy_(y)
        freed.fill_(-9)
        torch.cuda.synchronize()

    def seen():
        torch.cuda.synchronize()
        return [x.clone() for x in (t, d.block_tables, d.lens, d.ref_counts, n.block_tables, n.ref_counts, freed, one, ids)]
    work()
    want = seen()
    kv8.ref_fork(ref := a.copy(), 0, 2, tables, lens, counts, [1, 1, 0], [2, 3, 4], spare[:3])
    gone = kv8.ref_free(tables, lens, counts, [3, 0])
    new = kv8.ref_compact(ref, 0, 2, tables, lens, counts)
    assert np.array_equal(want[0].cpu().numpy(), ref) and want[6].cpu().tolist()[:len(gone)] == gone and int(want[7][0]) == len(gone)
    assert np.array_equal(want[4].cpu().numpy(), new[0]) and int(want[7][1]) == new[3]
    side = torch.cuda.Stream()
    reset()
    work(side)
    assert all(torch.equal(x, y) for x, y in zip(seen(), want))
    graph = torch.cuda.CUDAGraph()
    reset()
    with torch.cuda.graph(graph):
        work()
    for _ in range(4):
        reset()
        graph.replay()
        assert all(torch.equal(x, y) for x, y in zip(seen(), want))


# --------------------------------------------------------------------- all of it together

class Sequences:
    """A serving loop's sequences: logical K/V by the oracle's append into a pool of their own, one row each."""

    def __init__(self, Hkv, D, blocks):
        self.Hkv, self.D, self.blocks, self.pools, self.lens = Hkv, D, blocks, {}, {}

    def new(self, row):
        self.pools[row] = np.zeros((1, self.blocks, kv8.page_bytes(self.Hkv, self.D)), np.uint8)
        self.lens[row] = 0

    def fork(self, parent, child):
        self.pools[child], self.lens[child] = self.pools[parent].copy(), self.lens[parent]

    def append(self, row, k, v):
        kv8.ref_append(self.pools[row], 0, np.arange(self.blocks)[None], [self.lens[row]], [0, len(k)], k, v, self.Hkv, self.D)
        self.lens[row] += len(k)

    def check(self, row, q, out):
        n = len(q)
        K, V = kv8.read_logical(self.pools[row], 0, np.arange(self.blocks), self.lens[row], self.Hkv, self.D)
        ref, spread, reach = kv8.attention(q, K, V, self.lens[row] - n, 1 / np.sqrt(self.D))
        # half a bf16 step of the weights and of the output; fp32 scores and sums
        bound = 1.01 * (2.0 ** -8 + 2.0 ** -19 * reach[..., None]) * spread + 1.01 * 2.0 ** -8 * np.abs(ref) + 2.0 ** -20 * np.abs(V).max()
        assert (np.abs(out - ref) <= bound).all()


@pytest.mark.parametrize("D", [64, 128])
def test_a_serving_loop(D):
    """Prompts in chunks, forks, decodes of the samples, a preemption through a staging buffer, frees, compaction into a
    smaller pool, decodes again: every attention output against the oracle's own sequences."""
    Hkv, G, P, blocks, rows, L = 2, 4, 60, 12, 8, 2
    r = np.random.default_rng(D)
    pool = cs.Pool8.empty(L, P, Hkv, D)
    pool.tensor.fill_(0x7F)
    space = cs.PageSpace.of(pool)
    tables = cs.PageTables(torch.full((rows, blocks), -1, dtype=torch.int32, device="cuda"), torch.zeros(rows, dtype=torch.int32, device="cuda"),
                           torch.zeros(P, dtype=torch.int32, device="cuda"))
    free = list(r.permutation(P))
    logical = [Sequences(Hkv, D, blocks) for _ in range(L)]
    freed, number = torch.full((P,), -1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")

    def step(work):
        """work: {row: new tokens}; every row's pages are extended, appended to and attended over, in every layer."""
        nonlocal free
        order = sorted(work)
        bt, lens, counts = tables.block_tables.cpu(), tables.lens.cpu(), tables.ref_counts.cpu()
        for row in order:
            for e in range(-(-int(lens[row]) // 16), -(-(int(lens[row]) + work[row]) // 16)):
                p = int(free.pop())
                bt[row, e], counts[p] = p, 1
        tables.block_tables.copy_(bt)
        tables.ref_counts.copy_(counts)
        cu = torch.tensor(np.concatenate([[0], np.cumsum([work[x] for x in order])]), dtype=torch.int32)
        b = cs.Batch(bt[order], lens[order], cu)
        T = int(cu[-1])
        for layer in range(L):
            k, v, q = (torch.from_numpy(r.standard_normal((T, h, D))).bfloat16() for h in (Hkv, Hkv, Hkv * G))
            out = torch.empty((T, Hkv * G, D), dtype=torch.bfloat16, device="cuda")
            cs.cs_kv8_append(pool, layer, b, k.cuda(), v.cuda())
            cs.cs_paged_attention_mixed_kv8(pool, layer, b, q.cuda(), out, Hkv * G, 1 / np.sqrt(D), cs.workspace_for_kv8(b, Hkv * G, Hkv, D))
            got = out.double().cpu().numpy()
            for i, row in enumerate(order):
                at = slice(int(cu[i]), int(cu[i + 1]))
                logical[layer].append(row, k[at].double().numpy(), v[at].double().numpy())
                logical[layer].check(row, q[at].double().numpy(), got[at])
        for i, row in enumerate(order):
            tables.lens[row] += work[row]

    def fork(parent, children):
        fresh = [int(free.pop()) for _ in children]
        tail = int(tables.lens[parent]) % 16 != 0
        cs.cs_kv_pages_fork(space, 0, L, tables, dev([parent] * len(children)), dev(children), dev(fresh))
        if not tail:
            free.extend(fresh)
        for s in logical:
            for c in children:
                s.fork(parent, c)

    def release(rows_):
        cs.cs_kv_pages_free(tables, dev(rows_), freed, number)
        free.extend(freed.cpu().tolist()[:int(number)])

    for s in logical:
        for row in (0, 1):
            s.new(row)
    step({0: 37, 1: 20})
    step({0: 1, 1: 12})                                                   # row 1 ends with a full page
    fork(0, [2, 3])
    fork(1, [4])
    step({0: 1, 1: 1, 2: 1, 3: 20, 4: 1})
    # preempt row 3: its pages to a staging buffer, other ones back
    ids = tables.block_tables[3, :4].clone()
    stage = torch.zeros((L, 4, pool.page_bytes), dtype=torch.uint8, device="cuda")
    cs.cs_kv_pages_copy(space, 0, ids, cs.PageSpace.staging(stage), 0, None, L)
    n3 = int(tables.lens[3])
    release([3])
    back = [int(free.pop()) for _ in range(4)]
    cs.cs_kv_pages_copy(cs.PageSpace.staging(stage), 0, None, space, 0, dev(back), L)
    tables.block_tables[3, :4] = dev(back)
    tables.ref_counts[dev(back).long()] = 1
    tables.lens[3] = n3
    step({2: 1, 3: 2})
    release([0, 4])
    new = cs.PageTables(torch.empty_like(tables.block_tables), tables.lens, torch.empty_like(tables.ref_counts))
    new_ids, used = torch.empty(P, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    cs.cs_kv_pages_compact(space, 0, L, tables, new, new_ids, used, cs.compact_workspace_for(space))
    tables = new
    u = int(used)
    assert u == P - len(free) and int(tables.block_tables.max()) < u and (tables.ref_counts[u:] == 0).all()
    pool.tensor[:, u:] = 0x7F                                              # the tail is given back
    free = list(range(u, P))
    step({1: 3, 2: 1, 3: 17})
    release([1, 2, 3])
    assert int(tables.ref_counts.abs().max()) == 0 and sorted(free) == list(range(P))


@pytest.mark.parametrize("bad", [-1, 40, 2 ** 31 - 1])
def test_a_fork_of_an_unfinished_page_that_is_not_there(bad):
    """The child ends at the parent's last full page: the fresh page holds nothing of the parent's, and stays free."""
    r = np.random.default_rng(6)
    tables, lens, counts, spare = world(r, [50, 9, 33, 0, 0, 0], 40, 8)
    a = noise(r, 2, 40, 256)
    tables[0, 3], tables[1, 0] = bad, bad                                # both unfinished
    counts[:] = 0
    np.add.at(counts, tables[(tables >= 0) & (tables < 40)], 1)
    s, t = space_of(a, 256)
    d = cs.PageTables(dev(tables), dev(lens), dev(counts))
    cs.cs_kv_pages_fork(s, 0, 2, d, dev([0, 1, 2]), dev([3, 4, 5]), dev(spare[:3]))
    kv8.ref_fork(a, 0, 2, tables, lens, counts, [2], [5], spare[2:3])    # the third is an ordinary one
    counts[tables[0, :3]] += 1
    tables[3, :3] = tables[0, :3]
    lens[3], lens[4] = 48, 0
    assert np.array_equal(t.cpu().numpy(), a)
    for got, want in ((d.block_tables, tables), (d.lens, lens), (d.ref_counts, counts)):
        assert np.array_equal(got.cpu().numpy(), want)
