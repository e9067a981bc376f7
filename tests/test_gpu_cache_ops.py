"""Rotary append, attention of drafted trees, moving and reading back cache entries, against 64-bit references (GPU, through
the C ABI)."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2512_03416_amd as ts
from cache_ops_ref import (PAGE, SIZE, STEP, TORCH, Batch, check, pack_bits, places, random_tree, rotate, rotate_error, tree_reference,
                           tree_see)
from paper_2512_03416_amd import binding

pytestmark = pytest.mark.gpu

KINDS = [("f32", "f32"), ("bf16", "bf16"), ("bf16", "fp8")]
HEADS = [(4, 1, 64), (32, 8, 128), (10, 2, 128), (16, 1, 64), (3, 3, 128)]


def bits(t):
    return t.view(torch.uint8).cpu().numpy()


def mask_on_gpu(see_list, words=None):
    return torch.from_numpy(pack_bits(see_list, words).view(np.int64)).cuda()


# ---- rotary append -----------------------------------------------------------------------------------------------------

ROPES = [dict(rot_dim=128, base=10000.0), dict(rot_dim=64, base=5e5, layout="interleaved"),
         dict(rot_dim=22, base=1e4, scaling="linear", factor=4.0), dict(rot_dim=2, layout="interleaved", scaling="ntk", factor=2.0),
         dict(rot_dim=48, base=5e5, scaling="yarn", factor=16.0, original_length=8192),
         dict(rot_dim=64, base=5e5, scaling="wavelength", factor=8.0, original_length=8192),
         dict(rot_dim=6, table=[1.0, -0.5, 3.0], attn_scale=0.75)]


def rope_case(b, rope, q, k, v, strided, positions, in_place=False, offset=0):
    """One call on fresh caches, checked: outputs, every byte of the caches."""
    rot = rope["rot_dim"]
    if rot > b.D:
        rope = dict(rope, rot_dim=b.D)
        rot = b.D
    layout = rope.get("layout", "half")
    freq, scale = ts.rope_frequencies(**rope)
    ctx = ts.Context(b.desc())
    ctx.set_rope(**rope)
    kc, vc, ks, vs, table = b.on_gpu()
    if strided:                                            # slices of one projection's rows, from any element on
        pad = 3 if offset else 0
        row = (b.Hq + 2 * b.Hkv) * b.D + pad
        flat = torch.zeros(b.T * row + offset, dtype=TORCH[b.dtype]).cuda()
        rows = flat[offset:].view(b.T, row)
        q3, k3, v3 = (rows[:, at * b.D:(at + h) * b.D].view(b.T, h, b.D) for at, h in ((0, b.Hq), (b.Hq, b.Hkv), (b.Hq + b.Hkv, b.Hkv)))
        for dst, src in ((q3, q), (k3, k), (v3, v)):
            dst.copy_(src)
    else:
        q3, k3, v3 = (t.cuda() for t in (q, k, v))
    out = q3 if in_place else torch.full((b.T, b.Hq, b.D), float("nan"), dtype=TORCH[b.dtype], device="cuda")
    pos = b.pos if positions is None else positions
    ctx.rope_kv_append(q3, k3, v3, out, kc, vc, ks, vs, table, b.q_lens, b.ctx_lens,
                       positions=None if positions is None else torch.from_numpy(positions.astype(np.int32)).cuda())
    torch.cuda.synchronize()
    step, half = STEP[b.dtype], {"f32": 0.0, "bf16": 2.0 ** -134, "fp8": 2.0 ** -10}
    qd, kd = q.double().numpy(), k.double().numpy()
    want = rotate(qd, pos, freq, scale, rot, layout)
    check(out, want, np.abs(want) * step + rotate_error(qd, scale, rot, layout) * (1 + step) + half[b.dtype], "q_out")
    assert np.array_equal(bits(out[..., rot:].contiguous()), bits(q[..., rot:].contiguous()))
    want = rotate(kd, pos, freq, scale, rot, layout)
    err = rotate_error(kd, scale, rot, layout)
    at = places("k", b.table, b.seq, b.pos, b.Hkv, b.D, b.kind)
    got = b.numbers(0, kc.cpu().view(b.caches[0].dtype))
    if b.kind == "fp8":
        s = b.k_scale.double().numpy()[None, :, None]
        want, err = np.clip(want / s, -448, 448), err / s + np.abs(want / s) * 2.0 ** -24
    step = STEP[b.kind]
    check(got[at], want, np.abs(want) * step + err * (1 + step) + half[b.kind], "k cache")
    rest = np.ones(got.size, bool)
    rest[at] = False
    raw = lambda t: bits(t).view({4: np.uint32, 2: np.uint16, 1: np.uint8}[SIZE[b.kind]])  # noqa: E731
    assert np.array_equal(raw(kc)[rest], raw(b.caches[0])[rest]), "other k entries"
    # V as the plain append stores it, and nothing else
    kc2, vc2, *_ = b.on_gpu()
    ctx.kv_append(k.cuda(), v.cuda(), kc2, vc2, ks, vs, table, b.q_lens, b.ctx_lens)
    torch.cuda.synchronize()
    assert np.array_equal(raw(vc), raw(vc2)), "v cache"
    ctx.close()


BATCHES = [([1], [1]), ([1, 0, 1, 1], [17, 5, 16, 300]), ([3, 16, 1, 37, 15], [3, 16, 33, 90, 80]), ([200], [263])]


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("rope", range(len(ROPES)))
def test_rope_append(dtype, kind, heads, rope):
    for i, (ql, cl) in enumerate(BATCHES):
        b = Batch(heads, dtype, kind, ql, cl, seed=10 * rope + i)
        q, k, v = b.randn(b.T, b.Hq, b.D), b.randn(b.T, b.Hkv, b.D), b.randn(b.T, b.Hkv, b.D)
        rng = np.random.default_rng(i)
        positions = None if i % 2 else rng.integers(0, 1 << 20, b.T)
        rope_case(b, ROPES[rope], q, k, v, strided=(i + rope) % 2 == 0, positions=positions, in_place=(i + rope) % 4 == 1,
                  offset=(0, 8, 1, 0)[i])


@pytest.mark.parametrize("dtype,kind", KINDS)
def test_rope_append_far_positions(dtype, kind):
    """Positions up to the end of int32 and negative ones: the angle keeps its place within a turn."""
    b = Batch((4, 2, 64), dtype, kind, [6], [22], seed=4)
    pos = np.array([0, 1, 131071, 2 ** 24 + 1, 2 ** 31 - 1, -77])
    q, k, v = b.randn(b.T, 4, 64), b.randn(b.T, 2, 64), b.randn(b.T, 2, 64)
    # (the reference's angle in double precision is off by 2^-53 of 2^31: 2.4e-7, within the bound's slack at unit values)
    rope_case(b, dict(rot_dim=64, base=5e5), q, k, v, strided=False, positions=pos)


def test_rope_append_many_sequences():
    """More sequences than one launch takes, some of them without new tokens, the page table's rows beyond the first launch."""
    n = 600
    rng = np.random.default_rng(8)
    ql = rng.integers(0, 3, n)
    ql[255:260] = 0
    b = Batch((4, 1, 64), "bf16", "bf16", ql, ql + rng.integers(0, 40, n), seed=9)
    rope_case(b, ROPES[0], b.randn(b.T, 4, 64), b.randn(b.T, 1, 64), b.randn(b.T, 1, 64), strided=True, positions=None)


@pytest.mark.parametrize("dtype,kind", KINDS)
def test_rope_append_values_out_of_the_ordinary(dtype, kind):
    """Infinities and NaN stay with their pair; dims behind the rotated ones keep their bits; saturation; no q."""
    b = Batch((2, 1, 64), dtype, kind, [4], [4], seed=2)
    k, v = b.randn(b.T, 1, 64), b.randn(b.T, 1, 64)
    k[0, 0, 3], k[1, 0, 20], k[2, 0, 40] = float("nan"), float("inf"), float("inf")
    k[3] *= 1e6
    ctx = ts.Context(b.desc())
    ctx.set_rope(16)
    kc, vc, ks, vs, table = b.on_gpu()
    ctx.rope_kv_append(None, k.cuda(), v.cuda(), None, kc, vc, ks, vs, table, b.q_lens, b.ctx_lens)
    torch.cuda.synchronize()
    at = places("k", b.table, b.seq, b.pos, 1, 64, kind)
    got = b.numbers(0, kc.cpu().view(b.caches[0].dtype))[at][:, 0]
    nan = np.isnan(got)
    assert set(np.nonzero(nan[0])[0]) == {3, 11} and not nan[1:].any()
    if kind == "fp8":
        assert got[1, 20] == 448 and got[2, 40] == 448 and np.abs(got[3]).max() == 448
    else:
        assert np.isinf(got[1, 20]) and np.isinf(got[2, 40]) and np.isfinite(np.delete(got[1], 20)).all()
    ctx.close()


# ---- attention of drafted trees ----------------------------------------------------------------------------------------

def tree_run(b, q, see_list, sm_scale=0.0, caches=None, words=None, chain=False, ctx=None):
    own = ctx is None
    ctx = ctx or ts.Context(b.desc())
    kc, vc, ks, vs, table = b.on_gpu()
    if caches is not None:
        kc, vc = (c.view(torch.uint8).cuda() for c in caches)
    out = torch.full((b.T, b.Hq, b.D), float("nan"), dtype=TORCH[b.dtype], device="cuda")
    ctx.tree_attention(q.cuda(), kc, vc, ks, vs, table, None if chain else mask_on_gpu(see_list, words), b.q_lens, b.ctx_lens, sm_scale, out)
    torch.cuda.synchronize()
    if own:
        ctx.close()
    return out


TREES = [([1], [1]), ([1, 0, 2], [16, 40, 33]), ([13, 1, 64], [13, 200, 500]), ([5, 33], [1000, 47]), ([65, 130], [300, 131]),
         ([8], [2000]), ([17, 3, 16, 15, 1], [160, 19, 16, 47, 64])]


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("tree", range(len(TREES)))
def test_tree_attention(dtype, kind, heads, tree):
    ql, cl = TREES[tree]
    b = Batch(heads, dtype, kind, ql, cl, seed=100 + tree)
    rng = np.random.default_rng(tree)
    see = [tree_see(random_tree(rng, n, roots=1 + tree % 2)) for n in b.q_lens]
    q = b.randn(b.T, b.Hq, b.D)
    check(tree_run(b, q, see, words=3 if tree % 3 == 0 else None), *tree_reference(b, q, see))


@pytest.mark.parametrize("dtype,kind", KINDS)
def test_tree_attention_any_mask(dtype, kind):
    """Masks that are no trees: rows that see nothing, not themselves, later nodes; bits of nodes that do not exist; scale."""
    rng = np.random.default_rng(5)
    for ql, cl in (([70, 9, 40], [70, 9, 43]), ([9, 30], [1500, 46])):
        b = Batch((8, 2, 128), dtype, kind, ql, cl, seed=31)
        see = [rng.random((n, n)) < 0.3 for n in ql]
        see[0][:3] = False
        see[1][4] = False
        wide = [np.concatenate([m, np.ones((len(m), 7), bool)], 1) for m in see]      # (bits behind the last node)
        q = b.randn(b.T, b.Hq, b.D)
        got = tree_run(b, q, wide, sm_scale=0.3)
        check(got, *tree_reference(b, q, see, 0.3))
        if cl[0] == ql[0]:
            assert (got[:3] == 0).all()


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("n", [1, 16, 31, 100])
def test_tree_attention_chains(dtype, kind, n):
    """Without a mask, with the mask of a chain, and a causal chunk of the mixed pass."""
    b = Batch((32, 8, 128), dtype, kind, [n, 2 * n], [n + 333, 2 * n], seed=n)
    see = [np.tril(np.ones((m, m), bool)) for m in b.q_lens]
    q = b.randn(b.T, b.Hq, b.D)
    want, bound = tree_reference(b, q, see)
    one, two = tree_run(b, q, see, chain=True), tree_run(b, q, see)
    check(one, want, bound)
    assert np.array_equal(bits(one), bits(two))
    ctx = ts.Context(b.desc())
    kc, vc, ks, vs, table = b.on_gpu()
    out = torch.empty_like(one)
    ctx.mixed_paged_attention(q.cuda(), None, None, kc, vc, ks, vs, table, b.q_lens, b.ctx_lens, 0.0, out)
    torch.cuda.synchronize()
    check(out, want, 2 * bound)                            # (the weights of both are rounded, at other references)
    ctx.close()


@pytest.mark.parametrize("dtype,kind", KINDS)
def test_tree_attention_what_is_not_seen_has_no_influence(dtype, kind):
    """Infinities and NaN in entries behind the sequence, in unseen nodes (K and V), and in nodes that some rows see."""
    b = Batch((8, 2, 64), dtype, kind, [20, 6], [77, 1000], seed=12)
    rng = np.random.default_rng(12)
    see = [tree_see(random_tree(rng, n)) for n in b.q_lens]
    see[0][:, 7] = False                                   # nobody sees node 7; node 9's descendants see node 9
    q = b.randn(b.T, b.Hq, b.D)
    caches = [c.clone() for c in b.caches]
    nan = float("nan")
    for i in (0, 1):
        flat = caches[i] if kind != "fp8" else caches[i].view(torch.uint8)
        poison = nan if kind != "fp8" else 0x7f
        for s, pos in ((0, np.arange(77, 80)), (0, np.array([57 + 7])), (1, np.arange(1000, 1008))):
            at = places("kv"[i], b.table, np.full(len(pos), s), pos, b.Hkv, b.D, kind)
            flat[torch.from_numpy(at.reshape(-1))] = poison
    at = places("v", b.table, np.array([0]), np.array([57 + 9]), b.Hkv, b.D, kind).reshape(-1)
    flat = caches[1] if kind != "fp8" else caches[1].view(torch.uint8)
    flat[torch.from_numpy(at[::5])] = nan if kind != "fp8" else 0x7f
    if kind != "fp8":
        flat[torch.from_numpy(at[2::5])] = float("inf")
    want, bound = tree_reference(b, q, see, cache=caches)
    rows = np.isnan(want).any((1, 2))
    assert rows[:20].any() and not rows[:20].all() and not rows[20:].any()
    assert np.array_equal(rows[:20], see[0][:, 9])
    check(tree_run(b, q, see, caches=caches), want, bound)


def test_tree_attention_infinite_scores():
    """A row whose seen scores are all -inf is NaN, one that also sees another key is not, +inf gives NaN."""
    b = Batch((1, 1, 64), "f32", "f32", [4], [4], seed=3)
    see = [np.array([[1, 0, 0, 0], [1, 1, 0, 0], [0, 0, 1, 0], [0, 0, 1, 1]], bool)]
    q = torch.ones((4, 1, 64))
    k = b.caches[0].clone()
    for node, v in ((0, -float("inf")), (2, float("inf"))):
        k[torch.from_numpy(places("k", b.table, np.array([0]), np.array([node]), 1, 64, "f32").reshape(-1))[:1]] = v
    got = tree_run(b, q, see, caches=[k, b.caches[1]]).cpu()
    assert torch.isnan(got[0]).all() and torch.isnan(got[2]).all() and torch.isnan(got[3]).all()
    v1 = b.tokens(1, 0, 2)[1]
    check(got[1], v1, np.abs(v1) * 2.0 ** -22)


@pytest.mark.parametrize("dtype,kind", KINDS)
def test_tree_attention_large_scores(dtype, kind):
    """Scores of hundreds that grow along the keys: the reference maximum is raised again and again, in every wave and part."""
    b = Batch((4, 2, 128), dtype, kind, [5], [1501], seed=21)
    x = b.randn(1, 1, 128)
    at = places("k", b.table, np.zeros(1501, int), np.arange(1501), 2, 128, kind)
    k = b.numbers(0).copy()
    ramp = np.linspace(-4, 4, 1501)[:, None, None] * x.double().numpy() * (30 if kind == "fp8" else 1)
    k[at] = ramp
    b.caches[0] = torch.from_numpy(k).to(torch.float32).to(b.caches[0].dtype)
    q = x.repeat(5, 4, 1) * 2
    see = [tree_see(random_tree(np.random.default_rng(1), 5))]
    check(tree_run(b, q, see), *tree_reference(b, q, see))


@pytest.mark.parametrize("dtype,kind", KINDS)
def test_tree_attention_negative_scales(dtype, kind):
    b = Batch((4, 2, 64), dtype, kind, [7], [100], seed=23)
    if kind == "fp8":
        b.k_scale[0] *= -1
        b.v_scale[1] *= -1
    see = [tree_see(random_tree(np.random.default_rng(1), 7))]
    q = b.randn(b.T, 4, 64)
    check(tree_run(b, q, see), *tree_reference(b, q, see))


def test_tree_attention_many_sequences():
    """More trees than one launch takes, long ones among short ones (cut scans in both launches), some empty."""
    rng = np.random.default_rng(6)
    ql = rng.integers(0, 6, 300)
    cl = ql + rng.integers(0, 60, 300)
    cl[[3, 290]] = 2500
    b = Batch((4, 1, 64), "bf16", "bf16", ql, cl, seed=7)
    see = [tree_see(random_tree(rng, n)) if n else np.zeros((0, 0), bool) for n in ql]
    q = b.randn(b.T, 4, 64)
    check(tree_run(b, q, see), *tree_reference(b, q, see))


def test_tree_attention_is_repeatable_and_leaves_the_rest():
    """Run-to-run identical; rows behind the last sequence stay as they are."""
    b = Batch((32, 8, 128), "bf16", "bf16", [12, 30], [3000, 700], seed=8)
    see = [tree_see(random_tree(np.random.default_rng(2), n)) for n in b.q_lens]
    q = b.randn(b.T, b.Hq, b.D)
    ctx = ts.Context(b.desc())
    kc, vc, ks, vs, table = b.on_gpu()
    out = torch.full((b.T + 3, b.Hq, b.D), 7.0, dtype=torch.bfloat16, device="cuda")
    mask, first = mask_on_gpu(see), None
    for _ in range(4):
        ctx.tree_attention(q.cuda(), kc, vc, ks, vs, table, mask, b.q_lens, b.ctx_lens, 0.0, out)
        torch.cuda.synchronize()
        assert (out[b.T:] == 7.0).all()
        first = bits(out) if first is None else first
        assert np.array_equal(bits(out), first)
    ctx.close()


# ---- moving and reading back -------------------------------------------------------------------------------------------

def moved(b, which, pairs):
    """The cache (raw elements) after the pairs (sequence, src, dst), all read before any is written; the last of several with one
    destination counts."""
    raw = b.caches[which].view({4: torch.int32, 2: torch.int16, 1: torch.uint8}[SIZE[b.kind]]).numpy()
    new = raw.copy()
    for s, src, dst in pairs:
        if 0 <= src < b.ctx_lens[s] and 0 <= dst < b.ctx_lens[s]:
            f, t = (places("kv"[which], b.table, np.array([s]), np.array([p]), b.Hkv, b.D, b.kind) for p in (src, dst))
            new[t] = raw[f]
    return new


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("heads", [(4, 1, 64), (32, 8, 128), (3, 3, 128)])
def test_kv_move(dtype, kind, heads):
    """Paths, swaps, chains, one source for many, one destination of many, padding and positions out of range."""
    b = Batch(heads, dtype, kind, [0] * 6, [40, 100, 17, 200, 64, 1], seed=40)
    rng = np.random.default_rng(4)
    pairs = [(0, [20, 23, 29], [20, 21, 22]), (1, [5, 50, 99, 50], [50, 5, 98, 97]), (2, [-1, 16, 17, 3], [0, -1, 2, 17]),
             (3, list(rng.integers(-2, 205, 64)), list(rng.integers(-2, 205, 64))), (4, [], []), (5, [0], [0])]
    flat = [(s, f, t) for s, fs, ts_ in pairs for f, t in zip(fs, ts_)]
    ctx = ts.Context(b.desc())
    kc, vc, _, _, table = b.on_gpu()
    dev = lambda i: torch.tensor([p[i] for p in flat], dtype=torch.int32, device="cuda")  # noqa: E731
    ctx.kv_move(kc, vc, table, dev(1), dev(2), [len(p[1]) for p in pairs], b.ctx_lens)
    torch.cuda.synchronize()
    for which, t in ((0, kc), (1, vc)):
        assert np.array_equal(bits(t), moved(b, which, flat).view(np.uint8)), "kv"[which]
    ctx.close()


def test_kv_move_many_sequences():
    n = 700
    rng = np.random.default_rng(1)
    b = Batch((2, 1, 64), "bf16", "bf16", [0] * n, rng.integers(1, 50, n), seed=41)
    lens = rng.integers(0, 4, n)
    lens[200:600] = 0
    flat = [(s, int(rng.integers(0, b.ctx_lens[s])), int(rng.integers(0, b.ctx_lens[s]))) for s in range(n) for _ in range(lens[s])]
    ctx = ts.Context(b.desc())
    kc, vc, _, _, table = b.on_gpu()
    dev = lambda i: torch.tensor([p[i] for p in flat], dtype=torch.int32, device="cuda")  # noqa: E731
    ctx.kv_move(kc, vc, table, dev(1), dev(2), lens, b.ctx_lens)
    torch.cuda.synchronize()
    for which, t in ((0, kc), (1, vc)):
        assert np.array_equal(bits(t), moved(b, which, flat).view(np.uint8))
    ctx.close()


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("heads", HEADS)
def test_kv_read(dtype, kind, heads):
    """Rows from any position on; e4m3: value times scale in single precision, rounded to nearest even (NaN kept)."""
    starts, lens = np.array([0, 16, 7, 30, 0, 5]), np.array([1, 16, 20, 0, 300, 3])
    b = Batch(heads, dtype, kind, [0] * 6, starts + lens, seed=50)
    if kind == "fp8":
        for c in b.caches:
            c.view(torch.uint8)[::97] = 0x7f
    ctx = ts.Context(b.desc())
    kc, vc, ks, vs, table = b.on_gpu()
    T = int(lens.sum())
    for offset in (0, 1):                                  # (outputs on any element)
        outs = [torch.full((T * b.Hkv * b.D + offset + 5,), 7.0, dtype=TORCH[dtype], device="cuda") for _ in range(2)]
        o = [x[offset:offset + T * b.Hkv * b.D].view(T, b.Hkv, b.D) for x in outs]
        ctx.kv_read(kc, vc, ks, vs, table, starts, lens, *o)
        torch.cuda.synchronize()
        seq = np.repeat(np.arange(6), lens)
        pos = np.concatenate([np.arange(s, s + n) for s, n in zip(starts, lens)])
        for i, got in enumerate(o):
            at = torch.from_numpy(places("kv"[i], b.table, seq, pos, b.Hkv, b.D, kind))
            if kind == "fp8":
                want = (b.caches[i].float()[at] * (b.k_scale, b.v_scale)[i][None, :, None]).to(TORCH[dtype])
                assert torch.equal(torch.isnan(got.cpu()), torch.isnan(want))
                assert torch.equal(torch.nan_to_num(got.cpu()), torch.nan_to_num(want))
            else:
                assert torch.equal(got.cpu(), b.caches[i][at])
            assert (outs[i][:offset] == 7.0).all() and (outs[i][offset + T * b.Hkv * b.D:] == 7.0).all()
    # one of the two, from the first position on
    only = torch.zeros((T, b.Hkv, b.D), dtype=TORCH[dtype], device="cuda")
    ctx.kv_read(kc, vc, ks, vs, table, None, lens, None, only)
    ctx.kv_read(kc, vc, ks, vs, table, np.zeros(6, int), lens, o[0], o[1])
    torch.cuda.synchronize()
    assert np.array_equal(bits(only), bits(o[1].contiguous()))
    ctx.close()


def test_kv_read_many_sequences():
    rng = np.random.default_rng(2)
    n = 600
    lens, starts = rng.integers(0, 20, n), rng.integers(0, 30, n)
    b = Batch((2, 2, 64), "f32", "f32", [0] * n, starts + lens, seed=51)
    ctx = ts.Context(b.desc())
    kc, vc, ks, vs, table = b.on_gpu()
    o = [torch.empty((int(lens.sum()), 2, 64), device="cuda") for _ in range(2)]
    ctx.kv_read(kc, vc, ks, vs, table, starts, lens, *o)
    torch.cuda.synchronize()
    seq = np.repeat(np.arange(n), lens)
    pos = np.concatenate([np.arange(s, s + m) for s, m in zip(starts, lens)])
    for i in (0, 1):
        assert torch.equal(o[i].cpu(), b.caches[i][torch.from_numpy(places("kv"[i], b.table, seq, pos, 2, 64, "f32"))])
    ctx.close()


# ---- together, streams, graphs, refusals -------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,kind", KINDS)
def test_a_verified_step(dtype, kind):
    """As a decoder uses them: prompts appended with rotary positions, a drafted tree appended and attended, the accepted path
    moved together, the next token's pass -- and the cache then holds what appending the accepted tokens one after the other gives."""
    heads, rope = (8, 2, 128), dict(rot_dim=128, base=5e5)
    Hq, Hkv, D = heads
    rng = np.random.default_rng(0)
    prompts, nodes = np.array([50, 130, 7]), np.array([9, 20, 4])
    b = Batch(heads, dtype, kind, nodes, prompts + nodes, seed=60, extra_width=2)
    ctx = ts.Context(b.desc())
    ctx.set_rope(**rope)
    trees = [random_tree(rng, n) for n in nodes]
    masks, depths = ts.tree_masks(np.concatenate(trees), nodes)
    paths = []
    for t in trees:                                        # the path to the last node
        p = [len(t) - 1]
        while t[p[-1]] >= 0:
            p.append(int(t[p[-1]]))
        paths.append(p[::-1])
    pq, pk, pv = (b.randn(int(prompts.sum()), h, D).cuda() for h in (Hq, Hkv, Hkv))
    nq, nk, nv = (b.randn(int(nodes.sum()), h, D).cuda() for h in (Hq, Hkv, Hkv))
    kc, vc, ks, vs, table = b.on_gpu()
    ctx.rope_kv_append(pq, pk, pv, torch.empty_like(pq), kc, vc, ks, vs, table, prompts, prompts)
    pos = torch.from_numpy((np.repeat(prompts, nodes) + depths).astype(np.int32)).cuda()
    q = torch.empty_like(nq)
    ctx.rope_kv_append(nq, nk, nv, q, kc, vc, ks, vs, table, nodes, prompts + nodes, positions=pos)
    out = torch.empty_like(q)
    ctx.tree_attention(q, kc, vc, ks, vs, table, torch.from_numpy(masks.view(np.int64)).cuda(), nodes, prompts + nodes, 0.0, out)
    torch.cuda.synchronize()
    b.caches = [c.cpu().view(b.caches[0].dtype) for c in (kc, vc)]
    want, bound = tree_reference(b, q.cpu(), [tree_see(t) for t in trees])
    check(out, want, bound, "tree")
    lens = np.array([len(p) for p in paths])
    dev = lambda a: torch.from_numpy(np.concatenate(a).astype(np.int32)).cuda()  # noqa: E731
    ctx.kv_move(kc, vc, table, dev([n + np.array(p) for n, p in zip(prompts, paths)]), dev([n + np.arange(len(p)) for n, p in zip(prompts, paths)]),
                lens, prompts + nodes)
    # the accepted tokens one after the other, at their places
    at = np.concatenate([first + np.array(p) for first, p in zip(np.cumsum(nodes) - nodes, paths)])
    kc2, vc2, *_ = b.on_gpu()
    ctx.rope_kv_append(None, nk[at], nv[at], None, kc2, vc2, ks, vs, table, lens, prompts + lens)
    rows = [[torch.empty((int((prompts + lens).sum()), Hkv, D), dtype=TORCH[dtype], device="cuda") for _ in range(2)] for _ in range(2)]
    ctx.kv_read(kc, vc, ks, vs, table, None, prompts + lens, *rows[0])
    ctx.kv_read(kc2, vc2, ks, vs, table, None, prompts + lens, *rows[1])
    torch.cuda.synchronize()
    for x, y in zip(*rows):
        assert np.array_equal(bits(x), bits(y))
    # the pass over the path's last token, its row of the tree: the same keys
    last = np.cumsum(nodes) - 1
    one = torch.empty((3, Hq, D), dtype=TORCH[dtype], device="cuda")
    ctx.mixed_paged_attention(q[last].contiguous(), None, None, kc, vc, ks, vs, table, [1, 1, 1], prompts + lens, 0.0, one)
    torch.cuda.synchronize()
    check(one, want[last], 2 * bound[last] + 1e-6, "pass")
    ctx.close()


def _hip():
    with open("/proc/self/maps") as f:
        return ctypes.CDLL(next(l.split()[-1] for l in f if "libamdhip64.so" in l))


def test_captured_and_replayed():
    """The four calls in one graph: replayed between eager work with other inputs in the same buffers, against eager calls."""
    b = Batch((32, 8, 128), "bf16", "fp8", [12, 30, 1], [2000, 300, 40], seed=70)
    rng = np.random.default_rng(1)
    see = [tree_see(random_tree(rng, n)) for n in b.q_lens]
    ctx, other = ts.Context(b.desc()), ts.Context(b.desc())
    kc, vc, ks, vs, table = b.on_gpu()
    mask = mask_on_gpu(see)
    x = torch.empty((b.T, b.Hq + 2 * b.Hkv, b.D), dtype=torch.bfloat16, device="cuda")
    src = torch.tensor([1999, 1990, 299, 39], dtype=torch.int32, device="cuda")
    dst = torch.tensor([1988, 1989, 270, 39], dtype=torch.int32, device="cuda")
    moves, lens = [2, 1, 1], [100, 300, 7]
    new = lambda: (torch.empty((b.T, b.Hq, b.D), dtype=torch.bfloat16, device="cuda"), torch.empty((b.T, b.Hq, b.D), dtype=torch.bfloat16, device="cuda"),  # noqa: E731
                   *(torch.empty((sum(lens), b.Hkv, b.D), dtype=torch.bfloat16, device="cuda") for _ in range(2)))

    def calls(c, kc, vc, bufs, stream=None):
        q, out, ko, vo = bufs
        c.rope_kv_append(x[:, :b.Hq], x[:, b.Hq:b.Hq + b.Hkv], x[:, b.Hq + b.Hkv:], q, kc, vc, ks, vs, table, b.q_lens, b.ctx_lens, stream=stream)
        c.tree_attention(q, kc, vc, ks, vs, table, mask, b.q_lens, b.ctx_lens, 0.0, out, stream=stream)
        c.kv_move(kc, vc, table, src, dst, moves, b.ctx_lens, stream=stream)
        c.kv_read(kc, vc, ks, vs, table, None, lens, ko, vo, stream=stream)

    for c in (ctx, other):
        c.set_rope(128, base=5e5)
    x.normal_()
    stream, hip = torch.cuda.Stream(), _hip()
    bufs = new()
    calls(ctx, kc.clone(), vc.clone(), bufs)               # an eager call on another stream before the capture
    torch.cuda.synchronize()
    kc1, vc1 = kc.clone(), vc.clone()
    st, graph, execg = ctypes.c_void_p(stream.cuda_stream), ctypes.c_void_p(), ctypes.c_void_p()
    n0 = ctx.get_option("scratch_allocations")
    assert hip.hipStreamBeginCapture(st, 2) == 0
    calls(ctx, kc1, vc1, bufs, stream)
    assert hip.hipStreamEndCapture(st, ctypes.byref(graph)) == 0
    assert hip.hipGraphInstantiate(ctypes.byref(execg), graph, None, None, ctypes.c_size_t(0)) == 0
    ctx.set_rope(64, base=1e4)                             # (the graph keeps its rotation)
    kc2, vc2 = kc.clone(), vc.clone()
    for i in range(4):
        x.normal_()
        for t in bufs:
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        assert hip.hipGraphLaunch(execg, st) == 0
        torch.cuda.synchronize()
        want = new()
        calls(other, kc2, vc2, want)
        torch.cuda.synchronize()
        for g, w in zip((*bufs, kc1, vc1), (*want, kc2, vc2)):
            assert np.array_equal(bits(g), bits(w)), i
    assert ctx.get_option("scratch_allocations") == n0
    assert hip.hipGraphExecDestroy(execg) == 0 and hip.hipGraphDestroy(graph) == 0
    ctx.close()
    other.close()


def test_scratch_is_not_allocated_under_capture():
    b = Batch((32, 8, 128), "bf16", "bf16", [12], [4000], seed=71)
    see = [tree_see(random_tree(np.random.default_rng(1), 12))]
    ctx, hip = ts.Context(b.desc()), _hip()
    kc, vc, ks, vs, table = b.on_gpu()
    q, mask = b.randn(b.T, b.Hq, b.D).cuda(), mask_on_gpu(see)
    out = torch.zeros_like(q)
    call = lambda s: ctx.tree_attention(q, kc, vc, ks, vs, table, mask, b.q_lens, b.ctx_lens, 0.0, out, stream=s)  # noqa: E731
    stream, graph = torch.cuda.Stream(), ctypes.c_void_p()
    torch.cuda.synchronize()
    st = ctypes.c_void_p(stream.cuda_stream)
    assert hip.hipStreamBeginCapture(st, 2) == 0
    with pytest.raises(ts.TokenScaleError) as e:
        call(stream)
    assert hip.hipStreamEndCapture(st, ctypes.byref(graph)) == 0
    assert e.value.code == binding.TS_ERR_UNSUPPORTED and "ts_reserve_tree" in str(e.value)
    hip.hipGraphDestroy(graph)
    ctx.reserve_tree()
    n0 = ctx.get_option("scratch_allocations")
    call(None)
    ctx.reserve_tree()
    torch.cuda.synchronize()
    assert ctx.get_option("scratch_allocations") == n0
    check(out, *tree_reference(b, q.cpu(), see))
    ctx.close()


def test_calls_of_a_context_are_ordered_among_streams():
    """Append on one stream, attention, move and read on others, without an event of the caller's between them."""
    b = Batch((32, 8, 128), "bf16", "bf16", [40] * 16, [2000] * 16, seed=72)
    see = [tree_see(random_tree(np.random.default_rng(1), 40))] * 16
    x = b.randn(b.T, b.Hq + 2 * b.Hkv, b.D).cuda()
    mask, rows = mask_on_gpu(see), 16 * 40
    src = torch.full((16,), 1999, dtype=torch.int32, device="cuda")
    dst = torch.full((16,), 1960, dtype=torch.int32, device="cuda")

    def step(streams):
        ctx = ts.Context(b.desc())
        ctx.set_rope(128)
        ctx.reserve_tree()
        kc, vc, ks, vs, table = b.on_gpu()
        q, out = (torch.zeros((b.T, b.Hq, b.D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        ko, vo = (torch.zeros((rows, b.Hkv, b.D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        torch.cuda.synchronize()
        for i in range(12):
            s = [streams[(i + j) % len(streams)] for j in range(4)]
            ctx.rope_kv_append(x[:, :b.Hq], x[:, b.Hq:b.Hq + b.Hkv], x[:, b.Hq + b.Hkv:], q, kc, vc, ks, vs, table, b.q_lens, b.ctx_lens, stream=s[0])
            ctx.tree_attention(q, kc, vc, ks, vs, table, mask, b.q_lens, b.ctx_lens, 0.0, out, stream=s[1])
            ctx.kv_move(kc, vc, table, src, dst, [1] * 16, b.ctx_lens, stream=s[2])
            ctx.kv_read(kc, vc, ks, vs, table, [1960] * 16, [40] * 16, ko, vo, stream=s[3])
        torch.cuda.synchronize()
        ctx.close()
        return [bits(t) for t in (q, out, ko, vo)]

    one, many = step([torch.cuda.current_stream()]), step([torch.cuda.Stream() for _ in range(3)])
    for g, w in zip(many, one):
        assert np.array_equal(g, w)


def test_refusals():
    """What is refused has no effect on device memory."""
    b = Batch((8, 2, 64), "bf16", "bf16", [3, 2], [20, 40], seed=80)
    ctx = ts.Context(b.desc())
    kc, vc, ks, vs, table = b.on_gpu()
    q, k, v = (b.randn(b.T, h, 64).cuda() for h in (8, 2, 2))
    out = torch.full_like(q, 7.0)
    kc0, vc0 = kc.clone(), vc.clone()
    mask = torch.zeros((b.T, 1), dtype=torch.int64, device="cuda")
    i5 = torch.zeros(5, dtype=torch.int32, device="cuda")

    def refused(code, call, text=""):
        with pytest.raises(ts.TokenScaleError) as e:
            call()
        assert e.value.code == code and text in str(e.value), str(e.value)

    INV, UNS = binding.TS_ERR_INVALID_ARG, binding.TS_ERR_UNSUPPORTED
    append = lambda q=q, k=k, v=v, o=out, ql=b.q_lens, cl=b.ctx_lens, kc=kc: ctx.rope_kv_append(q, k, v, o, kc, vc, ks, vs, table, ql, cl)  # noqa: E731
    refused(INV, append, "ts_set_rope")
    for bad in (dict(rot_dim=66), dict(rot_dim=7), dict(rot_dim=128), dict(rot_dim=64, base=0.5)):
        refused(INV, lambda: ctx.set_rope(**bad))
    ctx.set_rope(64)
    refused(INV, lambda: append(q=None))
    refused(INV, lambda: append(o=None))
    refused(INV, lambda: append(k=None))
    refused(INV, lambda: append(ql=[3, -1]))
    with pytest.raises(ValueError):                        # (too few rows for these lengths: the binding's own check)
        append(ql=[21, 2])
    refused(INV, lambda: append(cl=[20, 16 * b.width + 1]))
    refused(INV, lambda: append(kc=None))
    tree = lambda q=q, m=mask, ql=b.q_lens, cl=b.ctx_lens, sm=0.0, o=out: ctx.tree_attention(q, kc, vc, ks, vs, table, m, ql, cl, sm, o)  # noqa: E731
    refused(INV, lambda: tree(q=None))
    refused(INV, lambda: tree(o=None))
    refused(INV, lambda: tree(sm=float("nan")))
    refused(INV, lambda: tree(cl=[2, 40]))
    move = lambda ml=(3, 2), cl=b.ctx_lens, s=i5, d=i5: ctx.kv_move(kc, vc, table, s, d, ml, cl)  # noqa: E731
    refused(INV, lambda: move(ml=(3, -1)))
    refused(INV, lambda: move(s=None))
    refused(INV, lambda: move(cl=[20, 16 * b.width + 1]))
    read = lambda st=(0, 0), ln=(3, 2), k=out, v=out: ctx.kv_read(kc, vc, ks, vs, table, st, ln, k, v)  # noqa: E731
    refused(INV, lambda: read(k=None, v=None))
    refused(INV, lambda: read(st=(-1, 0)))
    refused(INV, lambda: read(st=(0, 16 * b.width)))
    refused(INV, lambda: read(st=(2 ** 31 - 1, 0)))
    with pytest.raises(ValueError):                        # the binding's own
        append(q=q.float())
    with pytest.raises(ValueError):
        append(q=q[:4])
    with pytest.raises(ValueError):
        append(k=k.transpose(1, 2))
    with pytest.raises(ValueError):
        append(cl=[20])
    with pytest.raises(ValueError):
        tree(m=mask[:4])
    with pytest.raises(ValueError):
        tree(m=mask.cpu())
    with pytest.raises(ValueError):
        append(kc=kc[:-1])
    # in place over rows that are not packed; a stride below a row; misaligned queries
    x = torch.zeros((b.T, 12, 64), dtype=torch.bfloat16, device="cuda")
    lib, n = ts.load_library(), lambda a: np.asarray(a, np.int32).tobytes()  # noqa: E731
    raw = lambda q, qs, o, ks_=0: lib.ts_rope_kv_append(ctx._h, 0, q, qs, k.data_ptr(), ks_, v.data_ptr(), 0, o, kc.data_ptr(), vc.data_ptr(), 0, 0,  # noqa: E731
                                                        table.data_ptr(), 0, n(b.q_lens), n(b.ctx_lens), 2)
    assert raw(x.data_ptr(), 12 * 64, x.data_ptr()) == INV
    assert lib.ts_rope_kv_append(ctx._h, 0, q.data_ptr(), 0, k.data_ptr(), 0, v.data_ptr(), 0, out.data_ptr(), kc.data_ptr(), vc.data_ptr(), 0, 0,
                                 table.data_ptr(), 0, n([21, 2]), n(b.ctx_lens), 2) == INV
    assert raw(x.data_ptr(), 8 * 64 - 1, out.data_ptr()) == INV
    assert raw(x.data_ptr(), 0, out.data_ptr(), 2 * 64 - 1) == INV
    assert lib.ts_tree_attention(ctx._h, 0, q.data_ptr() + 2, kc.data_ptr(), vc.data_ptr(), 0, 0, table.data_ptr(), mask.data_ptr(), 1, n([3, 1]),
                                 n(b.ctx_lens), 2, 0.0, out.data_ptr()) == INV
    torch.cuda.synchronize()
    assert (out == 7.0).all() and torch.equal(kc, kc0) and torch.equal(vc, vc0)
    # empty batches do nothing
    none = torch.zeros((0, 8, 64), dtype=torch.bfloat16, device="cuda")
    ctx.rope_kv_append(none, none[:, :2], none[:, :2], none, kc, vc, ks, vs, table, [0, 0], b.ctx_lens)
    ctx.tree_attention(none, kc, vc, ks, vs, table, mask[:0], [], [], 0.0, none)
    ctx.kv_move(kc, vc, table, None, None, [0, 0], b.ctx_lens)
    ctx.kv_read(kc, vc, ks, vs, table, None, [0, 0], None, None)
    torch.cuda.synchronize()
    assert torch.equal(kc, kc0)
    ctx.close()


def test_refusals_of_too_many():
    w = 40
    desc = ts.Desc.make(2, 1, 64, "bf16", "bf16", 64, w)
    ctx = ts.Context(desc)
    kc, vc = (torch.zeros(ts.cache_bytes(desc), dtype=torch.uint8, device="cuda") for _ in range(2))
    table = torch.arange(w, dtype=torch.int32, device="cuda").view(1, w)
    q = torch.zeros((300, 2, 64), dtype=torch.bfloat16, device="cuda")
    out, mask = torch.full_like(q, 7.0), torch.zeros((300, 5), dtype=torch.int64, device="cuda")
    for n, words, code in ((257, 5, binding.TS_ERR_UNSUPPORTED), (65, 1, binding.TS_ERR_INVALID_ARG)):
        with pytest.raises(ts.TokenScaleError) as e:
            ctx.tree_attention(q, kc, vc, None, None, table, mask[:, :words].contiguous(), [n], [n], 0.0, out)
        assert e.value.code == code
    i = torch.zeros(65, dtype=torch.int32, device="cuda")
    with pytest.raises(ts.TokenScaleError) as e:
        ctx.kv_move(kc, vc, table, i, i, [65], [640])
    assert e.value.code == binding.TS_ERR_UNSUPPORTED
    torch.cuda.synchronize()
    assert (out == 7.0).all()
    ctx.close()


@pytest.mark.parametrize("bad", [-1, 10 ** 6])
def test_validated_page_table(bad):
    """Option validate_block_table: a bad page id is reported before anything is launched; good tables work as without it."""
    b = Batch((8, 2, 64), "bf16", "bf16", [3, 2], [20, 40], seed=81)
    ctx = ts.Context(b.desc())
    ctx.set_rope(64)
    ctx.set_option("validate_block_table", 1)
    kc, vc, ks, vs, table = b.on_gpu()
    q, k, v = (b.randn(b.T, h, 64).cuda() for h in (8, 2, 2))
    see = [np.tril(np.ones((n, n), bool)) for n in b.q_lens]
    mask, i5 = mask_on_gpu(see), torch.zeros(5, dtype=torch.int32, device="cuda")
    out, ko = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
    wrong = table.clone()
    wrong[1, 2] = bad
    calls = [lambda t: ctx.rope_kv_append(q, k, v, out, kc, vc, ks, vs, t, b.q_lens, b.ctx_lens),
             lambda t: ctx.tree_attention(q, kc, vc, ks, vs, t, mask, b.q_lens, b.ctx_lens, 0.0, out),
             lambda t: ctx.kv_move(kc, vc, t, i5, i5, [3, 2], b.ctx_lens),
             lambda t: ctx.kv_read(kc, vc, ks, vs, t, None, [3, 40][:1] + [35], None, torch.empty((38, 2, 64), dtype=torch.bfloat16, device="cuda"))]
    before = kc.clone()
    for call in calls:
        with pytest.raises(ts.TokenScaleError) as e:
            call(wrong)
        assert e.value.code == binding.TS_ERR_INVALID_ARG and "sequence 1, page 2" in str(e.value)
    torch.cuda.synchronize()
    assert (out == 7.0).all() and torch.equal(kc, before)
    for call in calls:
        call(table)
    torch.cuda.synchronize()
    b.caches = [c.cpu().view(torch.bfloat16) for c in (kc, vc)]
    ctx.close()


# ---- far pages, many rows, large trees, graphs that share the scratch, more refusals -------------------------------------

@pytest.mark.parametrize("dtype,kind", KINDS)
def test_pages_far_into_a_large_cache(dtype, kind):
    """Pages behind the first 2^32 elements: the same bits as in a small cache."""
    heads, base = (16, 8, 128), 262144 + 5
    b = Batch(heads, dtype, kind, [5, 40, 1], [70, 300, 33], seed=90)
    rng = np.random.default_rng(3)
    masks = mask_on_gpu([tree_see(random_tree(rng, n)) for n in b.q_lens])
    x = b.randn(b.T, 32, 128).cuda()
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    src, dst, lens = dev([69, 68, 299, 5]), dev([65, 66, 261, 32]), [70, 300, 33]

    def run(desc, kc, vc, table, ks, vs):
        ctx = ts.Context(desc)
        ctx.set_rope(64, layout="interleaved")
        q, out = (torch.zeros((b.T, 16, 128), dtype=TORCH[dtype], device="cuda") for _ in range(2))
        ko, vo = (torch.zeros((sum(lens), 8, 128), dtype=TORCH[dtype], device="cuda") for _ in range(2))
        ctx.rope_kv_append(x[:, :16], x[:, 16:24], x[:, 24:], q, kc, vc, ks, vs, table, b.q_lens, b.ctx_lens)
        ctx.tree_attention(q, kc, vc, ks, vs, table, masks, b.q_lens, b.ctx_lens, 0.0, out)
        ctx.kv_move(kc, vc, table, src, dst, [2, 1, 1], b.ctx_lens)
        ctx.kv_read(kc, vc, ks, vs, table, None, lens, ko, vo)
        torch.cuda.synchronize()
        ctx.close()
        return [bits(t) for t in (q, out, ko, vo)]

    kc, vc, ks, vs, table = b.on_gpu()
    page = kc.numel() // b.pool
    big = [torch.zeros((base + b.pool, page), dtype=torch.uint8, device="cuda") for _ in range(2)]
    for large, small in zip(big, (kc, vc)):
        large[base:] = small.view(b.pool, page)
    want = run(b.desc(), kc, vc, table, ks, vs)
    got = run(ts.Desc.make(16, 8, 128, dtype, kind, base + b.pool, b.width), big[0].view(-1), big[1].view(-1), table + base, ks, vs)
    for g, w in zip(got, want):
        assert np.array_equal(g, w)
    for large, small in zip(big, (kc, vc)):
        assert torch.equal(large[base:].reshape(-1), small) and not large[:base].view(torch.int64).any()


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("offset", [0, 1])
def test_rope_append_decode_rows(dtype, kind, offset):
    """Many single tokens, of which a workgroup takes several KV heads; in 16-byte pieces and element by element."""
    rng = np.random.default_rng(11)
    b = Batch((20, 5, 128), dtype, kind, np.ones(400, int), rng.integers(1, 60, 400), seed=91)
    rope_case(b, dict(rot_dim=96, base=1e6), b.randn(b.T, 20, 128), b.randn(b.T, 5, 128), b.randn(b.T, 5, 128), strided=True, positions=None, offset=offset)


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("shape", [([256], [256]), ([200, 3], [1800, 900]), ([64] * 12, [700] * 12), ([256] * 3, [300, 256, 257])])
def test_tree_attention_large_trees(dtype, kind, shape):
    """Trees of up to 256 nodes, with masks wider than needed, cut and whole, rows of a workgroup of every number."""
    b = Batch((8, 2, 64), dtype, kind, *shape, seed=92)
    rng = np.random.default_rng(12)
    see = [tree_see(random_tree(rng, n, roots=3)) for n in b.q_lens]
    see[0][[0, -1]] = False                                # (nothing but the prefix, if there is one)
    q = b.randn(b.T, b.Hq, b.D)
    got = tree_run(b, q, see, words=5)
    check(got, *tree_reference(b, q, see))
    if b.ctx_lens[0] == b.q_lens[0]:
        assert (got[0] == 0).all() and (got[b.q_lens[0] - 1] == 0).all()


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("offset", [0, 1])
def test_rope_append_rows_next_to_chunks(dtype, kind, offset):
    """Pages with one token and whole pages in one launch, which share their heads out differently; sequences behind the first launch's."""
    rng = np.random.default_rng(14)
    ql = np.ones(420, int)
    ql[[0, 130, 131, 400]] = 37, 22, 0, 50
    ql[300:340] = 0
    b = Batch((20, 5, 128), dtype, kind, ql, ql + rng.integers(0, 60, 420), seed=96)
    rope_case(b, dict(rot_dim=128, base=1e6), b.randn(b.T, 20, 128), b.randn(b.T, 5, 128), b.randn(b.T, 5, 128), strided=True, positions=None, offset=offset)


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("nodes", [8, 16])
def test_tree_attention_scans_of_every_length(dtype, kind, dim, nodes):
    """Prefixes of 0 to 312 tokens in one batch: scans of no step to ten before the steps with nodes.  Queries of four times the size, so
    that the reference maximum is raised on the way."""
    n = 40
    b = Batch((64, 8, dim), dtype, kind, np.full(n, nodes), nodes + 8 * np.arange(n), seed=95)
    rng = np.random.default_rng(13)
    see = [tree_see(random_tree(rng, nodes)) for _ in range(n)]
    q = b.randn(b.T, 64, dim) * 4
    check(tree_run(b, q, see), *tree_reference(b, q, see))


def test_two_graphs_of_one_context():
    """Two captured tree calls, whose scratch is the same, replayed in turn with an eager call between them."""
    batches = [Batch((32, 8, 128), "bf16", "bf16", ql, cl, seed=93 + i) for i, (ql, cl) in enumerate((([12], [4000]), ([30, 7], [2500, 900])))]
    width, pool = max(b.width for b in batches), max(b.pool for b in batches)
    ctx, hip, stream = ts.Context(ts.Desc.make(32, 8, 128, "bf16", "bf16", pool, width)), _hip(), torch.cuda.Stream()
    ctx.reserve_tree()
    st, runs = ctypes.c_void_p(stream.cuda_stream), []
    for b in batches:
        see = [tree_see(random_tree(np.random.default_rng(1), n)) for n in b.q_lens]
        kc, vc = (torch.zeros(pool * 8 * PAGE * 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        for c, x in zip((kc, vc), b.caches):
            c[:x.numel()] = x.cuda()
        table = np.full((len(b.q_lens), width), -1, np.int32)
        table[:, :b.width] = b.table
        q, mask, table = b.randn(b.T, 32, 128).cuda(), mask_on_gpu(see), torch.from_numpy(table).cuda()
        outs = [torch.zeros_like(q) for _ in range(2)]
        call = lambda out, s, b=b, q=q, kc=kc, vc=vc, table=table, mask=mask: ctx.tree_attention(  # noqa: E731
            q, kc, vc, None, None, table, mask, b.q_lens, b.ctx_lens, 0.0, out, stream=s)
        torch.cuda.synchronize()
        graph, execg = ctypes.c_void_p(), ctypes.c_void_p()
        assert hip.hipStreamBeginCapture(st, 2) == 0
        call(outs[0], stream)
        assert hip.hipStreamEndCapture(st, ctypes.byref(graph)) == 0
        assert hip.hipGraphInstantiate(ctypes.byref(execg), graph, None, None, ctypes.c_size_t(0)) == 0
        runs.append((call, outs, q, graph, execg))
    for i in range(3):
        for call, outs, q, graph, execg in runs:
            q.normal_()
            outs[0].fill_(float("nan"))
        torch.cuda.synchronize()
        for call, outs, q, graph, execg in runs:
            assert hip.hipGraphLaunch(execg, st) == 0
        torch.cuda.synchronize()
        for call, outs, q, graph, execg in runs:
            call(outs[1], None)
        torch.cuda.synchronize()
        for call, outs, q, graph, execg in runs:
            assert np.array_equal(bits(outs[0]), bits(outs[1])), i
    for call, outs, q, graph, execg in runs:
        assert hip.hipGraphExecDestroy(execg) == 0 and hip.hipGraphDestroy(graph) == 0
    ctx.close()


def test_refusals_of_addresses_and_rows():
    """Rows that overlap (an expanded tensor's stride of 0 is not that of packed rows); caches and masks off their alignment."""
    b = Batch((8, 2, 64), "bf16", "bf16", [3, 2], [20, 40], seed=94)
    ctx, lib = ts.Context(b.desc()), ts.load_library()
    ctx.set_rope(64)
    kc, vc, ks, vs, table = b.on_gpu()
    q, k, v = (b.randn(b.T, h, 64).cuda() for h in (8, 2, 2))
    out, mask, i5 = torch.full_like(q, 7.0), torch.zeros((b.T + 1, 1), dtype=torch.int64, device="cuda"), torch.zeros(5, dtype=torch.int32, device="cuda")
    before = [t.clone() for t in (kc, vc)]
    for i in range(3):
        rows = [q, k, v]
        rows[i] = rows[i][:1].expand(b.T, -1, -1)
        with pytest.raises(ValueError):
            ctx.rope_kv_append(*rows, out, kc, vc, ks, vs, table, b.q_lens, b.ctx_lens)
    lens = lambda *a: np.asarray(a, np.int32).tobytes()  # noqa: E731
    ql, cl, t = lens(*b.q_lens), lens(*b.ctx_lens), table.data_ptr()
    for dk, dv in ((8, 0), (0, 4)):
        kp, vp = kc.data_ptr() + dk, vc.data_ptr() + dv
        assert lib.ts_rope_kv_append(ctx._h, 0, q.data_ptr(), 0, k.data_ptr(), 0, v.data_ptr(), 0, out.data_ptr(), kp, vp, 0, 0, t, 0, ql, cl, 2) == binding.TS_ERR_INVALID_ARG
        assert lib.ts_tree_attention(ctx._h, 0, q.data_ptr(), kp, vp, 0, 0, t, mask.data_ptr(), 1, ql, cl, 2, 0.0, out.data_ptr()) == binding.TS_ERR_INVALID_ARG
        assert lib.ts_kv_move(ctx._h, 0, kp, vp, t, i5.data_ptr(), i5.data_ptr(), ql, cl, 2) == binding.TS_ERR_INVALID_ARG
        assert lib.ts_kv_read(ctx._h, 0, kp, vp, 0, 0, t, None, ql, 2, out.data_ptr(), None) == binding.TS_ERR_INVALID_ARG
    assert lib.ts_tree_attention(ctx._h, 0, q.data_ptr(), kc.data_ptr(), vc.data_ptr(), 0, 0, t, mask.data_ptr() + 4, 1, ql, cl, 2, 0.0, out.data_ptr()) == binding.TS_ERR_INVALID_ARG
    torch.cuda.synchronize()
    assert (out == 7.0).all() and torch.equal(kc, before[0]) and torch.equal(vc, before[1])
    ctx.close()


def test_refusal_of_key_numbers_beyond_int32():
    """Refused before anything is launched: a tree whose last round of keys has numbers beyond int32."""
    lib, lens = ts.load_library(), lambda *a: np.asarray(a, np.int32).tobytes()  # noqa: E731
    t = torch.zeros(64, dtype=torch.int64, device="cuda")
    p, ctx = t.data_ptr(), ts.Context(ts.Desc.make(2, 1, 64, "bf16", "bf16", 64, 1 << 27))
    assert lib.ts_tree_attention(ctx._h, 0, p, p, p, 0, 0, p, p, 1, lens(1), lens(2 ** 31 - 1), 1, 0.0, p) == binding.TS_ERR_UNSUPPORTED
    assert "too large" in ctx.last_error()
    ctx.close()
    torch.cuda.synchronize()
    assert not t.any()


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("heads", [(8, 2, 64), (64, 8, 128)])
@pytest.mark.parametrize("shape", [([5], [3005]), ([64] * 4, [700] * 4), ([16, 3, 30], [1800, 900, 40])])
def test_tree_attention_weights_add_up(dtype, kind, heads, shape):
    """V is the same for every key, so that the output is V whatever the weights: numerator and denominator take the same ones.  One key a
    page has a larger score, all others have one score, so that a row's weights are all rounded alike (a share of up to 2^-8 of 16-bit ones).
    Bound: the sums over n keys are off by n 2^-24 twice, with a dozen roundings besides 4.4e-4 at the most; V is a number of q's type, and
    the next one is 2^-8 of it away at the least, so that 16-bit outputs are V itself."""
    b = Batch(heads, dtype, kind, *shape, seed=97)
    if kind == "fp8":                                      # (powers of two: V times its scale is a bf16 number)
        b.k_scale, b.v_scale = torch.full((b.Hkv,), 2.0 ** -6), torch.full((b.Hkv,), 2.0 ** -5)
    unit = 64 if kind == "fp8" else 1
    sign = torch.randint(0, 2, (b.D,), generator=b.gen).double().numpy() * 2 - 1
    row = b.cache_of(torch.randn((b.Hkv, b.D), generator=b.gen)).double().numpy()
    caches = [b.numbers(0).copy(), b.numbers(1).copy()]
    for s, n in enumerate(b.ctx_lens):
        pos = np.arange(n)
        caches[0][places("k", b.table, np.full(n, s), pos, b.Hkv, b.D, kind)] = \
            np.where(pos % PAGE == 0, 1.0, 0.25)[:, None, None] * unit * sign
        caches[1][places("v", b.table, np.full(n, s), pos, b.Hkv, b.D, kind)] = row
    caches = [torch.from_numpy(c).to(torch.float32).to(b.caches[0].dtype) for c in caches]
    size = 0.02 + 0.4 * torch.rand((b.T, b.Hq, 1), generator=b.gen)
    q = (size.to(TORCH[dtype]).double() * torch.from_numpy(sign)).to(TORCH[dtype])
    rng = np.random.default_rng(15)
    see = [tree_see(random_tree(rng, n)) for n in b.q_lens]
    want = np.repeat(row * (2.0 ** -5 if kind == "fp8" else 1.0), b.Hq // b.Hkv, 0)[None].repeat(b.T, 0)
    bound = np.abs(want) * 2 * (int(b.ctx_lens.max()) + 12) * 2.0 ** -24 if dtype == "f32" else np.zeros_like(want)
    check(tree_run(b, q, see, caches=caches), want, bound)


@pytest.mark.parametrize("dtype,kind", KINDS)
def test_steps_without_tokens(dtype, kind):
    """No sequence brings a token, the buffers are there all the same (a serving loop's, of its largest batch): nothing is done, nothing is
    refused, through the binding and through the C entry points."""
    b = Batch((8, 2, 64), dtype, kind, [3, 2], [20, 40], seed=98)
    ctx, lib = ts.Context(b.desc()), ts.load_library()
    ctx.set_rope(64)
    kc, vc, ks, vs, table = b.on_gpu()
    q, k, v = (b.randn(b.T, h, 64).cuda() for h in (8, 2, 2))
    out, ko, vo = (torch.full((b.T, h, 64), 7.0, dtype=TORCH[dtype], device="cuda") for h in (8, 2, 2))
    before = [t.clone() for t in (kc, vc, q)]
    i5, mask = torch.zeros(5, dtype=torch.int32, device="cuda"), torch.zeros((b.T, 1), dtype=torch.int64, device="cuda")
    for lens in ([0, 0], []):
        cl, tab = b.ctx_lens[:len(lens)], table[:len(lens)]
        ctx.rope_kv_append(q, k, v, out, kc, vc, ks, vs, tab, lens, cl)
        ctx.rope_kv_append(q, k, v, q, kc, vc, ks, vs, tab, lens, cl, positions=i5)
        ctx.rope_kv_append(None, k, v, None, kc, vc, ks, vs, tab, lens, cl)
        ctx.tree_attention(q, kc, vc, ks, vs, tab, mask, lens, cl, 0.0, out)
        ctx.kv_move(kc, vc, tab, i5, i5, lens, cl)
        ctx.kv_read(kc, vc, ks, vs, tab, None, lens, ko, vo)
    zero, cl = np.zeros(2, np.int32).tobytes(), b.ctx_lens.tobytes()
    p = [t.data_ptr() if t is not None else 0 for t in (kc, vc, ks, vs, table)]
    assert lib.ts_rope_kv_append(ctx._h, 0, None, 0, None, 0, None, 0, out.data_ptr(), *p, 0, zero, cl, 2) == binding.TS_OK
    assert lib.ts_rope_kv_append(ctx._h, 0, q.data_ptr(), 0, k.data_ptr(), 0, v.data_ptr(), 0, out.data_ptr(), *p, 0, zero, cl, 2) == binding.TS_OK
    torch.cuda.synchronize()
    assert all((t == 7.0).all() for t in (out, ko, vo)) and all(torch.equal(x, y) for x, y in zip((kc, vc, q), before))
    ctx.close()


def test_read_checks_the_pages_that_it_reads():
    """Option validate_block_table: pages in front of the tokens that are read may be gone (-1), as may those behind them."""
    b = Batch((8, 2, 64), "bf16", "bf16", [0, 0], [200, 90], seed=99)
    ctx = ts.Context(b.desc())
    kc, vc, ks, vs, table = b.on_gpu()
    starts, lens = [70, 33], [50, 31]                      # pages 4 .. 7 and 2 .. 3
    rows = lambda: [torch.full((81, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]  # noqa: E731
    want, got, refused = rows(), rows(), rows()
    ctx.kv_read(kc, vc, ks, vs, table, starts, lens, *want)
    ctx.set_option("validate_block_table", 1)
    holes = torch.full_like(table, -1)
    for s, (first, behind) in enumerate(((4, 8), (2, 4))):
        holes[s, first:behind] = table[s, first:behind]
    ctx.kv_read(kc, vc, ks, vs, holes, starts, lens, *got)
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert torch.equal(g, w)
    for s, page, bad in ((0, 4, -1), (0, 7, b.pool), (1, 2, b.pool), (1, 3, -1)):
        wrong = holes.clone()
        wrong[s, page] = bad
        with pytest.raises(ts.TokenScaleError) as e:
            ctx.kv_read(kc, vc, ks, vs, wrong, starts, lens, *refused)
        assert e.value.code == binding.TS_ERR_INVALID_ARG and f"sequence {s}, page {page}" in str(e.value)
    torch.cuda.synchronize()
    assert all((t == 7.0).all() for t in refused)
    ctx.close()


@pytest.mark.parametrize("dtype,kind", KINDS)
def test_validated_calls_give_the_same(dtype, kind):
    """Option validate_block_table on good tables: outputs and caches as without it, over more sequences than one check takes."""
    n = 600
    rng = np.random.default_rng(16)
    ql = rng.integers(0, 4, n)
    b = Batch((8, 2, 64), dtype, kind, ql, ql + rng.integers(0, 60, n), seed=100)
    see = [tree_see(random_tree(rng, m)) if m else np.zeros((0, 0), bool) for m in ql]
    q, k, v = (b.randn(b.T, h, 64).cuda() for h in (8, 2, 2))
    mask = mask_on_gpu(see)
    moves = np.minimum(ql, 2)
    src, dst = (torch.from_numpy(rng.integers(0, np.repeat(b.ctx_lens, moves)).astype(np.int32)).cuda() for _ in range(2))
    starts = rng.integers(0, b.ctx_lens + 1)
    lens = b.ctx_lens - starts
    runs = []
    for validate in (0, 1):
        ctx = ts.Context(b.desc())
        ctx.set_rope(64)
        ctx.set_option("validate_block_table", validate)
        kc, vc, ks, vs, table = b.on_gpu()
        turned, out = (torch.full((b.T, 8, 64), 7.0, dtype=TORCH[dtype], device="cuda") for _ in range(2))
        rows = [torch.full((int(lens.sum()), 2, 64), 7.0, dtype=TORCH[dtype], device="cuda") for _ in range(2)]
        ctx.rope_kv_append(q, k, v, turned, kc, vc, ks, vs, table, b.q_lens, b.ctx_lens)
        ctx.tree_attention(turned, kc, vc, ks, vs, table, mask, b.q_lens, b.ctx_lens, 0.0, out)
        ctx.kv_move(kc, vc, table, src, dst, moves, b.ctx_lens)
        ctx.kv_read(kc, vc, ks, vs, table, starts, lens, *rows)
        torch.cuda.synchronize()
        runs.append([bits(t) for t in (turned, out, kc, vc, *rows)])
        ctx.close()
    for x, y in zip(*runs):
        assert np.array_equal(x, y)
    assert not np.array_equal(runs[1][2], bits(b.caches[0]))


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("empty", [(64, 192), (0, 64), (384, 768), (0, 384), (320, 900)])
def test_blocks_of_sequences_without_tokens(dtype, kind, empty):
    """Append and read where whole aligned blocks of 64 sequences, or the 384 of a launch, bring no token."""
    n = 900
    rng = np.random.default_rng(17)
    ql = rng.integers(1, 4, n)
    ql[empty[0]:empty[1]] = 0
    b = Batch((4, 1, 64), dtype, kind, ql, ql + rng.integers(0, 40, n), seed=101)
    rope_case(b, ROPES[1], b.randn(b.T, 4, 64), b.randn(b.T, 1, 64), b.randn(b.T, 1, 64), strided=True, positions=None)
    ctx = ts.Context(b.desc())
    kc, vc, ks, vs, table = b.on_gpu()
    rows = [torch.empty((b.T, 1, 64), dtype=TORCH[dtype], device="cuda") for _ in range(2)]
    ctx.kv_read(kc, vc, ks, vs, table, b.ctx_lens - b.q_lens, b.q_lens, *rows)
    torch.cuda.synchronize()
    for i, got in enumerate(rows):
        want = b.caches[i].float()[torch.from_numpy(places("kv"[i], b.table, b.seq, b.pos, 1, 64, kind))]
        if kind == "fp8":
            want = (want * (b.k_scale, b.v_scale)[i][None, :, None]).to(TORCH[dtype])
        assert torch.equal(got.cpu().float(), want.float())
    ctx.close()


@pytest.mark.parametrize("heads", [(4, 1, 64), (64, 8, 128)])
@pytest.mark.parametrize("nodes,prefix", [(4, 0), (4, 600), (60, 700)])
def test_tree_attention_infinite_scores_in_16_bits(heads, nodes, prefix):
    """Every key of the prefix and the first node have a score of -inf, the second node a finite one, the third one +inf: a row that sees the
    first node only is NaN, one that sees the second too has its V, one that sees the third is NaN."""
    b = Batch(heads, "bf16", "bf16", [nodes], [prefix + nodes], seed=102)
    k = b.caches[0].clone()
    at = places("k", b.table, np.zeros(prefix + 1, int), np.arange(prefix + 1), b.Hkv, b.D, b.kind)
    k[torch.from_numpy(at[:, :, 5].reshape(-1))] = -float("inf")
    k[torch.from_numpy(places("k", b.table, np.array([0]), np.array([prefix + 2]), b.Hkv, b.D, b.kind)[:, :, 5].reshape(-1))] = float("inf")
    see = np.zeros((nodes, nodes), bool)
    see[:, 0] = True
    see[1::3, 1] = True
    see[2::3, 1:3] = True
    got = tree_run(b, torch.ones((nodes, b.Hq, b.D)).to(torch.bfloat16), [see], caches=[k, b.caches[1]]).cpu()
    assert torch.isnan(got[0::3]).all() and torch.isnan(got[2::3]).all()
    v = torch.from_numpy(b.tokens(1, 0, prefix + 2)[-1]).repeat_interleave(b.Hq // b.Hkv, 0)
    assert (got[1::3].double() == v).all()                 # (a weight of one, whatever the reference: nothing is rounded)
