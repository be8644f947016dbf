"""The speculative step's calls without a GPU: the oracle against what is known of it, and what the calls refuse before anything
would be enqueued."""
import ctypes
import os
import re
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle import draft
from paper_2410_01228_amd import binding as cs
import test_asm_hazards

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DEV = 0x10000                       # stands for device memory: nothing here gets as far as reading it


# ------------------------------------------------------------------------------------- oracle

def test_oracle_rotation_is_a_rotation():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((3, 2, 8))
    inv = [1.0, 0.25]
    y, _ = draft.ref_rope(x, [[0, 5, 7]], inv, 4)
    assert np.array_equal(y[0], x[0]) and np.array_equal(y[..., 4:], x[..., 4:])
    for i, (a, b) in enumerate(((0, 2), (1, 3))):
        z = (x[..., a] + 1j * x[..., b]) * np.exp(1j * np.array([0, 5, 7]) * inv[i])[:, None]
        assert np.allclose(y[..., a] + 1j * y[..., b], z)
    z, _ = draft.ref_rope(x[..., [0, 2, 1, 3, 4, 5, 6, 7]], [[0, 5, 7]], inv, 4, interleaved=True)
    assert np.allclose(z[..., [0, 2, 1, 3]], y[..., :4])
    # products of rotated rows depend on the distance of their positions alone
    q, k = rng.standard_normal((1, 1, 8)), rng.standard_normal((1, 1, 8))
    at = lambda r, p: draft.ref_rope(r, [[p]], inv, 4)[0][0, 0]  # noqa: E731
    assert np.isclose(at(q, 9) @ at(k, 4), at(q, 105) @ at(k, 100))
    n, _ = draft.ref_rope(x, [[0, 0, 0]], inv, 4, norm=np.full(8, 2.0))
    assert np.allclose((n * n).mean(-1), 4.0)


@pytest.mark.parametrize("drawn", [False, True])
def test_oracle_verification_keeps_the_distribution(drawn):
    """One node with two children and their leaves: the first token is distributed as p, whatever the drafts were."""
    rng = np.random.default_rng(2)
    vocab, n = 4, 40000
    p, q = rng.dirichlet(np.ones(vocab), 3).astype(np.float32), rng.dirichlet(np.ones(vocab), 3).astype(np.float32)
    seen = np.zeros(vocab)
    for _ in range(n):
        x = rng.choice(vocab, 2, p=q[0] / q[0].sum(dtype=np.float64)) if drawn else (2, 1)
        _, out = draft.ref_verify([0, *x], [-1, 0, 0], p, q if drawn else None, rng.random(3), rng.random())
        seen[out[0]] += 1
    # five standard deviations of a share of n draws
    assert np.all(np.abs(seen / n - p[0]) < 5 * np.sqrt(p[0] * (1 - p[0]) / n) + 1e-6)


def test_oracle_masks():
    seen = draft.ancestors([-1, 0, 0, 1, 3])
    assert seen.astype(int).tolist() == [[1, 0, 0, 0, 0], [1, 1, 0, 0, 0], [1, 0, 1, 0, 0], [1, 1, 0, 1, 0], [1, 1, 0, 1, 1]]
    assert draft.mask_words(seen, 1)[:, 0].tolist() == [1, 3, 5, 11, 27]
    wide = np.zeros((1, 70), bool)
    wide[0, [63, 64]] = True
    assert draft.mask_words(wide, 2).tolist() == [[-2 ** 63, 1]]


# ----------------------------------------------------------------------------------- refusals

def _pool(Hkv=2, D=64, L=2, P=8, ps=16):
    e = 2 * Hkv * ps * D
    return cs.cs_kv_pool(DEV, L, P, ps, Hkv, D, P * e, e)


def _batch(ctx=(3, 0), new=(2, 5), blocks=4):
    h = torch.tensor(ctx, dtype=torch.int32)
    cu = torch.zeros(len(new) + 1, dtype=torch.int32)
    cu[1:] = torch.cumsum(torch.tensor(new, dtype=torch.int32), 0)
    b = cs.cs_batch(len(ctx), int(cu[-1]), DEV, blocks, DEV, DEV, h.data_ptr(), cu.data_ptr())
    b.keep = (h, cu)
    return b


def _rope(**kw):
    d = dict(inv_freq=DEV, rotary_dim=64, interleaved=0, positions=DEV, position_stride=100, num_axes=1, axis_pairs=(ctypes.c_int32 * 3)(0, 0, 0), q_norm=None, k_norm=None, eps=0.0)
    d.update(kw)
    if not isinstance(d["axis_pairs"], ctypes.Array):
        d["axis_pairs"] = (ctypes.c_int32 * 3)(*d["axis_pairs"])
    return cs.cs_rope(**d)


def _qk(rope, f16=False, T=7, Hq=4, Hkv=2, D=64, q=DEV, qs=256, k=DEV, ks=128, qo=DEV, ko=DEV):
    fn = cs.lib().cs_qk_rope_f16 if f16 else cs.lib().cs_qk_rope
    return fn(ctypes.byref(rope) if rope else None, T, Hq, Hkv, D, q, qs, k, ks, qo, ko, None)


def _append(rope, f16=False, pool=None, layer=0, batch=None, Hq=4, q=DEV, qs=256, k=DEV, ks=128, v=DEV, vs=128, qo=DEV):
    fn = cs.lib().cs_kv_append_rope_f16 if f16 else cs.lib().cs_kv_append_rope
    pool, batch = pool or _pool(), batch or _batch()
    return fn(ctypes.byref(pool), layer, ctypes.byref(batch), ctypes.byref(rope) if rope else None, Hq, q, qs, k, ks, v, vs, qo, None)


INV, UNS, SMALL = cs.CS_ERR_INVALID_ARG, cs.CS_ERR_UNSUPPORTED, cs.CS_ERR_WORKSPACE_TOO_SMALL

BAD_ROPES = [
    (dict(rotary_dim=72), INV), (dict(rotary_dim=-8), INV), (dict(rotary_dim=12), UNS), (dict(num_axes=0), INV), (dict(num_axes=4), INV), (dict(eps=-1e-6), INV),
    (dict(eps=float("nan")), INV), (dict(eps=float("inf")), INV), (dict(inv_freq=None), INV), (dict(inv_freq=DEV + 2), INV), (dict(positions=DEV + 1), INV),
    (dict(num_axes=2, axis_pairs=(16, 15, 0)), INV), (dict(num_axes=3, axis_pairs=(16, 32, -16)), INV), (dict(num_axes=3, axis_pairs=(8, 8, 16), position_stride=6), INV),
    (dict(num_axes=2, axis_pairs=(2 ** 31 - 1, 2 ** 31 - 1, 0)), INV), (dict(q_norm=DEV + 4), INV), (dict(k_norm=DEV + 2), INV), (dict(num_axes=2, axis_pairs=(16, 16, 0), positions=None), INV),
]


@pytest.mark.parametrize("f16", [False, True])
@pytest.mark.parametrize("kw,status", BAD_ROPES)
def test_ropes_refused(kw, status, f16):
    assert _qk(_rope(**kw), f16) == status
    assert _append(_rope(**kw), f16) == status


@pytest.mark.parametrize("f16", [False, True])
def test_rotation_refused(f16):
    ok = _rope()
    assert _qk(None, f16) == INV and _append(None, f16) == INV
    assert _qk(_rope(positions=None), f16) == INV                      # (the append has positions of its own)
    for kw in (dict(T=-1), dict(Hq=0), dict(Hkv=0), dict(Hq=3), dict(q=None), dict(k=None), dict(qo=None), dict(ko=None), dict(qs=255), dict(qs=248), dict(qs=260), dict(ks=120), dict(ks=132),
               dict(q=DEV + 8), dict(k=DEV + 2), dict(qo=DEV + 8), dict(ko=DEV + 8)):
        assert _qk(ok, f16, **kw) == INV, kw
    assert _qk(ok, f16, D=96, qs=512, ks=512) == UNS
    assert _qk(ok, f16, T=0) == cs.CS_OK
    for kw in (dict(layer=-1), dict(layer=2), dict(Hq=3), dict(q=None), dict(k=None), dict(v=None), dict(qo=None), dict(qs=128), dict(ks=64), dict(vs=120), dict(vs=132), dict(v=DEV + 8),
               dict(pool=_pool(Hkv=0)), dict(batch=_batch(blocks=0)), dict(batch=_batch(ctx=(63, 0)))):
        assert _append(ok, f16, **kw) == INV, kw
    assert _append(ok, f16, pool=_pool(ps=4)) == UNS
    assert _append(ok, f16, batch=_batch(ctx=(3, 0), new=(0, 0))) == cs.CS_OK


def _tree(f16=False, pool=None, layer=0, batch=None, Hq=4, q=DEV, out=DEV, scale=0.1, mask=DEV, words=1, ws=DEV, wb=1 << 40):
    fn = cs.lib().cs_paged_attention_tree_f16 if f16 else cs.lib().cs_paged_attention_tree
    pool, batch = pool or _pool(), batch or _batch()
    return fn(ctypes.byref(pool), layer, ctypes.byref(batch), q, out, Hq, scale, mask, words, ws, wb, None)


@pytest.mark.parametrize("f16", [False, True])
def test_trees_refused(f16):
    for kw in (dict(layer=2), dict(Hq=0), dict(Hq=3), dict(q=None), dict(out=None), dict(q=DEV + 8), dict(out=DEV + 2), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")),
               dict(scale=float("nan")), dict(mask=DEV + 4), dict(words=0), dict(words=-1), dict(words=5), dict(batch=_batch((0,), (65,), 5)), dict(batch=_batch((0,), (256,), 16), words=3)):
        assert _tree(f16, **kw) == INV, kw
    assert _tree(f16, batch=_batch((0,), (257,), 32), words=4) == UNS
    assert _tree(f16, Hq=34) == UNS and _tree(f16, pool=_pool(D=96)) == UNS
    assert _tree(f16, batch=_batch((3,), (0,))) == cs.CS_OK
    # cut sequences need room
    long = _batch((30000,), (4,), 2000)
    need = cs.lib().cs_paged_attention_tree_workspace_bytes(ctypes.byref(long), 4, 2, 64)
    assert need > 0
    assert _tree(f16, batch=long, wb=need - 1) == SMALL and _tree(f16, batch=long, ws=None) == INV and _tree(f16, batch=long, ws=DEV + 8) == INV


def test_tree_workspaces():
    ask = lambda b, *shape: cs.lib().cs_paged_attention_tree_workspace_bytes(ctypes.byref(b), *shape)  # noqa: E731
    assert ask(_batch(), 4, 2, 64) == 0
    assert ask(_batch((0,), (257,), 32), 4, 2, 64) == 0 and ask(_batch((30000,), (4,), 2000), 5, 2, 64) == 0
    # whatever the lengths, a plan is made and grows with what is cut, not with the cache alone
    rng = np.random.default_rng(3)
    for S in (1, 3, 900, 3000):
        b = _batch(rng.integers(0, 60000, S).tolist(), rng.integers(1, 257, S).tolist(), 4000)
        assert 0 <= ask(b, 32, 2, 128) < 1 << 36


def _verify(batch=None, vocab=100, tokens=DEV, parents=DEV, p=DEV, ps=100, q=DEV, qs=100, u=DEV, un=DEV, o=DEV, path=DEV, count=DEV, ws=DEV, wb=1 << 30):
    batch = batch or _batch()
    return cs.lib().cs_spec_verify(ctypes.byref(batch), vocab, tokens, parents, p, ps, q, qs, u, un, o, path, count, ws, wb, None)


def test_verification_refused():
    for kw in (dict(vocab=0), dict(vocab=-1), dict(tokens=None), dict(p=None), dict(u=None), dict(un=None), dict(o=None), dict(path=None), dict(count=None), dict(ps=99), dict(qs=99),
               dict(p=DEV + 2), dict(count=DEV + 1), dict(batch=_batch(ctx=(0, 100), blocks=2))):
        assert _verify(**kw) == INV, kw
    assert _verify(vocab=(1 << 20) + 1, ps=1 << 21, qs=1 << 21) == UNS
    assert _verify(batch=_batch((0,), (257,), 32)) == UNS
    big = dict(vocab=128256, ps=128256, qs=128256)
    need = cs.cs_spec_verify_workspace_bytes(2, 128256)
    assert need > 0
    assert _verify(wb=need - 1, **big) == SMALL and _verify(ws=None, **big) == INV and _verify(ws=DEV + 8, **big) == INV
    for bad in ((0, 100), (-1, 100), (70000, 100), (1, 0), (1, (1 << 20) + 1)):
        assert cs.cs_spec_verify_workspace_bytes(*bad) == 0


def _commit(pool=None, l0=0, l1=2, batch=None, path=DEV, count=DEV):
    pool, batch = pool or _pool(), batch or _batch()
    return cs.lib().cs_kv_tree_commit(ctypes.byref(pool), l0, l1, ctypes.byref(batch), path, count, None)


def test_commit_refused():
    for kw in (dict(l0=-1), dict(l1=3), dict(l0=2, l1=1), dict(path=None), dict(count=None), dict(path=DEV + 2), dict(count=DEV + 1), dict(batch=_batch(blocks=0))):
        assert _commit(**kw) == INV, kw
    assert _commit(pool=_pool(ps=32)) == UNS
    assert _commit(l0=1, l1=1) == cs.CS_OK and _commit(batch=_batch((1,), (0,))) == cs.CS_OK


def test_far_positions_refused():
    """Positions, rounded up to a workgroup's keys, are 32-bit numbers."""
    far = lambda c: _batch((5, c), (1, 3), 2 ** 28)  # noqa: E731
    ask = lambda b: cs.lib().cs_paged_attention_tree_workspace_bytes(ctypes.byref(b), 4, 2, 64)  # noqa: E731
    last = 2 ** 31 - 1 - 4096 - 3
    for c in (last + 1, 2 ** 31 - 4, 2 ** 31 - 1):
        assert _append(_rope(), batch=far(c)) == UNS and _tree(batch=far(c)) == UNS and _commit(batch=far(c)) == UNS and ask(far(c)) == 0
    # the last one that is taken is planned for: it is cut, so a call without room for the pieces is refused
    assert 0 < ask(far(last)) < 1 << 30 and _tree(batch=far(last), wb=16) == SMALL


def test_threads_plan_for_themselves():
    import threading
    batches = [_batch((20000 + 100 * i, 7), (1 + i, 5), 4000) for i in range(12)]
    ask = lambda b: cs.lib().cs_paged_attention_tree_workspace_bytes(ctypes.byref(b), 8, 2, 128)  # noqa: E731
    want, wrong = [ask(b) for b in batches], []

    def work(seed):
        for i in np.random.default_rng(seed).integers(0, 12, 400):
            if ask(batches[i]) != want[i]:
                wrong.append(i)
    threads = [threading.Thread(target=work, args=(s,)) for s in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert len(set(want)) > 1 and not wrong


def test_binding_refuses_views_that_the_calls_would_read_past():
    inv, pos = torch.ones(32), torch.arange(7, dtype=torch.int32)
    q, k = torch.zeros(7, 4, 64, dtype=torch.bfloat16), torch.zeros(7, 2, 64, dtype=torch.bfloat16)
    for bad in (dict(inv_freq=torch.ones(31)), dict(inv_freq=inv.double()), dict(positions=pos.long()), dict(positions=pos.expand(3, 7)), dict(q_norm=torch.ones(64))):
        with pytest.raises((AssertionError, TypeError)):
            cs.Rope(**{**dict(inv_freq=inv, rotary_dim=64, positions=pos), **bad})
    rope = cs.Rope(inv, 64, pos)
    for qq, kk, qo, ko in ((q.transpose(0, 1).contiguous().transpose(0, 1), k, q, k), (q.float(), k, q, k), (q, k[:6], q, k), (q, k, q[:6], k), (q, k, q, k[..., ::2]),
                           (torch.zeros(8, 4, 64, dtype=torch.bfloat16), torch.zeros(8, 2, 64, dtype=torch.bfloat16), torch.zeros(8, 4, 64, dtype=torch.bfloat16), torch.zeros(8, 2, 64))):
        with pytest.raises(AssertionError):
            cs.cs_qk_rope(rope, qq, kk, qo, ko)


def test_struct_is_the_header_s():
    text = open(os.path.join(ROOT, "include", "conserve_kv.h")).read()
    body = re.sub(r"/\*.*?\*/", "", re.search(r"typedef struct \{([^}]*)\} cs_rope;", text).group(1), flags=re.S)
    names = re.findall(r"(\w+)(?:\[3\])?;", body)
    assert names == [n for n, _ in cs.cs_rope._fields_]
    assert ctypes.sizeof(cs.cs_rope) == 8 + 4 + 4 + 8 + 8 + 4 + 12 + 8 + 8 + 8


@pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"), reason="no hipcc")
def test_generated_code_around_the_copies_to_lds(tmp_path):
    """The tree kernels hold the same inline assembly as the prefill kernel: no SCC value lives across it, and none of it reads a matrix result
    that may not be there."""
    out = tmp_path / "cs_tree.s"
    subprocess.run([shutil.which("hipcc") or "/opt/rocm/bin/hipcc", "--offload-arch=gfx950", "-O3", "-std=c++17", "-I" + os.path.join(ROOT, "include"), "-Xclang", "-target-feature",
                    "-Xclang", "-packed-fp32-ops", "-S", "--cuda-device-only", "-o", str(out), os.path.join(ROOT, "paper_2410_01228_amd", "csrc", "cs_tree.hip")],
                   check=True, stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
    text = out.read_text()
    assert text.count("global_load_lds_dwordx4") > 50 and text.count("v_mfma_f32") > 100
    assert test_asm_hazards.scc_reads_after_asm(text) == []
    assert test_asm_hazards.matrix_results_read_in_asm(text) == []
    # and no kernel keeps what it works with in scratch memory
    assert set(re.findall(r"\.private_segment_fixed_size: *(\d+)", text)) == {"0"}


@pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"), reason="no hipcc")
def test_what_lds_is_read_by_sixteen_bytes_is_aligned_to_them(tmp_path):
    """Members of the kernels' LDS that they access as vectors of 16 bytes: their places, their rows and the blocks themselves."""
    csrc = os.path.join(ROOT, "paper_2410_01228_amd", "csrc")
    lines = ['#include "cs_tree_impl.h"', '#include "cs_rope.hip"', "using namespace cs;"]
    for d in (64, 128):
        kinds = [("TreeLds<%d, %d>" % (d, nc), ("q", "o"), ("o[0][0]",)) for nc in (1, 2)] + [("RingLds<%d, %d>" % (d, nc), ("ring",), ("ring[0]",)) for nc in (1, 2, 3)]
        for kind, members, rows in kinds + [("SlotLds<%d>" % d, ("k", "v"), ("k[0][0][0]", "v[0][0][0]"))]:
            lines.append("{ typedef %s T; static_assert(alignof(T) %% 16 == 0);" % kind)
            lines += ["static_assert(__builtin_offsetof(T, %s) %% 16 == 0);" % m for m in members]
            lines += ["static_assert(sizeof(((T*)nullptr)->%s) %% 16 == 0);" % r for r in rows] + ["}"]
    source = tmp_path / "places.hip"
    source.write_text("\n".join(lines[:3]) + "\nvoid places() {\n" + "\n".join(lines[3:]) + "\n}\n")
    run = subprocess.run([shutil.which("hipcc") or "/opt/rocm/bin/hipcc", "--offload-arch=gfx950", "-std=c++17", "-fsyntax-only", "--cuda-host-only", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                          str(source)], capture_output=True, text=True)
    assert run.returncode == 0, run.stderr


@pytest.mark.parametrize("f16", [False, True])
def test_binding_refuses_tensors_of_another_type(f16):
    """Rows of the other 16-bit type would be read as other bits, and outputs of one byte an element written past their end."""
    mine, other = (torch.float16, torch.bfloat16) if f16 else (torch.bfloat16, torch.float16)
    fn = lambda name: getattr(cs, name + ("_f16" if f16 else ""))  # noqa: E731
    rows = lambda h, t: torch.zeros(7, h, 64, dtype=t)  # noqa: E731
    pool = cs.Pool.empty(1, 4, 2, 64, device="cpu")
    batch = cs.Batch(torch.arange(4, dtype=torch.int32).view(2, 2), torch.tensor([3, 0]), torch.tensor([0, 2, 7]), device="cpu")
    inv, norm = torch.ones(32), torch.ones(64, dtype=mine)
    rope = cs.Rope(inv, 64, torch.arange(7, dtype=torch.int32), q_norm=norm, k_norm=norm)
    for bad in (other, torch.float32, torch.uint8, torch.int16):
        for i in range(4):
            args = [rows(h, bad if i == j else mine) for j, h in enumerate((4, 2, 4, 2))]
            with pytest.raises(AssertionError):
                fn("cs_qk_rope")(rope, *args)
            args = [rows(h, bad if i == j else mine) for j, h in enumerate((4, 2, 2, 4))]
            with pytest.raises(AssertionError):
                fn("cs_kv_append_rope")(pool, 0, batch, rope, *args)
        for i in range(2):
            q, out = (rows(4, bad if i == j else mine) for j in range(2))
            with pytest.raises(AssertionError):
                fn("cs_paged_attention_tree")(pool, 0, batch, q, out, 4, 0.1, None, None)
        for weights in ((norm.to(bad), norm), (norm, norm.to(bad)), (norm.to(bad), norm.to(bad)), (None, norm.to(bad))):
            with pytest.raises(AssertionError):
                fn("cs_qk_rope")(cs.Rope(inv, 64, torch.arange(7, dtype=torch.int32), q_norm=weights[0], k_norm=weights[1]), rows(4, mine), rows(2, mine), rows(4, mine), rows(2, mine))
    # the calls over 8 bits take either type's rows, and no shorter elements
    pool8 = cs.Pool8.empty(1, 4, 2, 64, device="cpu")
    for i in range(2):
        for bad in (torch.uint8, torch.float32):
            with pytest.raises(AssertionError):
                fn("cs_kv8_append")(pool8, 0, batch, *(rows(2, bad if i == j else mine) for j in range(2)))
            with pytest.raises(AssertionError):
                fn("cs_paged_attention_mixed_kv8")(pool8, 0, batch, *(rows(4, bad if i == j else mine) for j in range(2)), 4, 0.1, None)
