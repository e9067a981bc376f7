"""Host side of the rotary append and of the tree attention: frequencies, masks, refusals (no GPU)."""
import ctypes
import math
import os
import re
import subprocess
import sys

import numpy as np
import pytest

import paper_2512_03416_amd as ts
from cache_ops_ref import pack_bits, random_tree, tree_see
from paper_2512_03416_amd import binding, build


@pytest.mark.parametrize("rot", [2, 6, 64, 128])
@pytest.mark.parametrize("base", [10000.0, 5e5])
def test_frequencies_of_the_plain_scalings(rot, base):
    i = np.arange(rot // 2)
    f, m = ts.rope_frequencies(rot, base=base)
    np.testing.assert_allclose(f, base ** (-2 * i / rot), rtol=1e-14)
    assert m == 1.0
    f2, m2 = ts.rope_frequencies(rot, base=base, scaling="linear", factor=4)
    np.testing.assert_allclose(f2, f / 4, rtol=1e-14)
    assert m2 == 1.0
    f3, _ = ts.rope_frequencies(rot, base=base, scaling="ntk", factor=4)
    if rot > 2:                                            # the slowest pair is slowed by the factor, the fastest not at all
        assert f3[0] == 1.0 and math.isclose(f3[-1], f[-1] / 4, rel_tol=1e-12)
    else:
        assert f3[0] == 1.0
    f4, m4 = ts.rope_frequencies(rot, table=0.25 + i, attn_scale=1.5)
    assert np.array_equal(f4, 0.25 + i) and m4 == 1.5


def test_frequencies_of_the_ranged_scalings():
    rot, base, n, factor = 128, 5e5, 8192, 8.0
    plain, _ = ts.rope_frequencies(rot, base=base)
    turns = n * plain / (2 * math.pi)
    f, m = ts.rope_frequencies(rot, base=base, scaling="wavelength", factor=factor, original_length=n)
    assert m == 1.0
    np.testing.assert_allclose(f[turns > 4], plain[turns > 4], rtol=1e-14)
    np.testing.assert_allclose(f[turns < 1], plain[turns < 1] / factor, rtol=1e-14)
    mid = (turns > 1) & (turns < 4)
    assert mid.any() and np.all(f[mid] < plain[mid]) and np.all(f[mid] > plain[mid] / factor)
    f, m = ts.rope_frequencies(rot, base=base, scaling="yarn", factor=factor, original_length=n)
    assert math.isclose(m, 1 + 0.1 * math.log(factor), rel_tol=1e-14)
    lo, hi = np.nonzero(turns >= 32)[0][-1], np.nonzero(turns <= 1)[0][0]      # whole pairs on either side of the ramp
    np.testing.assert_allclose(f[:lo + 1], plain[:lo + 1], rtol=1e-14)
    np.testing.assert_allclose(f[hi:], plain[hi:] / factor, rtol=1e-14)
    ratio = f / plain
    assert np.all(np.diff(ratio) <= 1e-15)


@pytest.mark.parametrize("bad", [dict(rot_dim=3), dict(rot_dim=0), dict(rot_dim=130), dict(rot_dim=64, base=1.0),
                                 dict(rot_dim=64, base=float("inf")), dict(rot_dim=64, scaling="linear", factor=0.5),
                                 dict(rot_dim=64, scaling="linear", factor=float("nan")),
                                 dict(rot_dim=64, scaling="yarn", factor=2.0), dict(rot_dim=64, attn_scale=-1.0),
                                 dict(rot_dim=64, scaling="wavelength", factor=2.0, original_length=4096, low=4.0, high=4.0),
                                 dict(rot_dim=64, layout=2), dict(rot_dim=64, scaling=6), dict(rot_dim=64, scaling=5),
                                 dict(rot_dim=4, table=[1.0, float("inf")])])
def test_frequencies_refuse(bad):
    with pytest.raises(ts.TokenScaleError) as e:
        ts.rope_frequencies(**bad)
    assert e.value.code == binding.TS_ERR_INVALID_ARG


def test_rope_description_refuses_unknown_words():
    for bad in (dict(layout="halves"), dict(scaling="dynamic"), dict(table=[1.0])):
        with pytest.raises(ValueError):
            ts.RopeDesc.make(64, **bad)


def test_masks_and_depths():
    rng = np.random.default_rng(3)
    lens = [1, 0, 17, 64, 65, 200]
    trees = [random_tree(rng, n, roots=1 + (n > 20)) for n in lens]
    masks, depths = ts.tree_masks(np.concatenate(trees), lens)
    assert masks.shape == (sum(lens), 4) and masks.dtype == np.uint64
    assert np.array_equal(masks, pack_bits([tree_see(t) for t in trees], 4))
    assert np.array_equal(depths, np.concatenate([tree_see(t).sum(1) - 1 for t in trees]))
    empty, none = ts.tree_masks([], [])
    assert empty.shape == (0, 1) and none.shape == (0,)


@pytest.mark.parametrize("parents,lens,words", [([0], [1], 1), ([-1, 1], [2], 1), ([-2], [1], 1), ([-1, 5], [2], 1),
                                                ([-1] * 65, [65], 1)])
def test_masks_refuse(parents, lens, words):
    with pytest.raises(ts.TokenScaleError) as e:
        ts.tree_masks(parents, lens, words)
    assert e.value.code == binding.TS_ERR_INVALID_ARG


def test_masks_refuse_other_counts():
    with pytest.raises(ValueError):
        ts.tree_masks([-1, 0], [3])


def test_entry_points_refuse_a_missing_context():
    lib, null, one = ts.load_library(), ctypes.c_void_p(0), np.ones(1, np.int32).tobytes()
    assert lib.ts_set_rope(null, None) == binding.TS_ERR_INVALID_ARG
    assert lib.ts_reserve_tree(null) == binding.TS_ERR_INVALID_ARG
    assert lib.ts_rope_kv_append(null, *[null] * 2, 0, null, 0, null, 0, *[null] * 7, one, one, 1) == binding.TS_ERR_INVALID_ARG
    assert lib.ts_tree_attention(null, *[null] * 8, 1, one, one, 1, 0.0, null) == binding.TS_ERR_INVALID_ARG
    assert lib.ts_kv_move(null, *[null] * 6, one, one, 1) == binding.TS_ERR_INVALID_ARG
    assert lib.ts_kv_read(null, *[null] * 6, one, one, 1, null, null) == binding.TS_ERR_INVALID_ARG
    assert lib.ts_rope_frequencies(None, null, null) == binding.TS_ERR_INVALID_ARG


def test_kernels_keep_their_values_in_registers():
    """No kernel here spills: two workgroups of the tree attention share a CU at 256 vector registers a lane, and a spilled value next to
    copies in flight would wait for all of them.  No accumulator registers either: a value parked there while some lanes are masked
    off is lost to those lanes."""
    names = set()
    for src in ("ts_kernels_rope.hip", "ts_kernels_tree.hip"):
        r = subprocess.run([build.HIPCC] + build.FLAGS + ["-Rpass-analysis=kernel-resource-usage", "-x", "hip", "-c",
                                                          os.path.join(build.CSRC, src), "-o", os.devnull], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-2000:]
        name = None
        for line in r.stderr.splitlines():
            m = re.search(r"Function Name: (\S+)", line)
            if m:
                name = m.group(1)
                names.add(next((k for k in ("tree_merge_kernel", "tree_kernel", "rope_append_vec_kernel", "rope_append_kernel",
                                            "kv_read_vec_kernel", "kv_read_kernel", "kv_move_kernel") if k in name), ""))
            for what, most in (("VGPRs", 256), ("AGPRs", 0), ("VGPRs Spill", 0), (r"ScratchSize \[bytes/lane\]", 0)):
                m = re.search(r" " + what + r": (\d+)", line)
                if m and name:
                    assert int(m.group(1)) <= most, (name, line)
    assert len(names - {""}) == 7


def test_a_context_of_raw_pointers_needs_no_torch():
    """Device pointers and a stream handle as integers: nothing imports torch, which here cannot be imported (the library's calls are
    stood in for, there being no GPU)."""
    code = """
import ctypes, sys
sys.modules["torch"] = None
from paper_2512_03416_amd import binding
binding.load_library()
class Calls:
    made = []
    def __getattr__(self, name):
        if name == "ts_cache_bytes":
            return lambda d: 1 << 20
        return lambda *a: self.made.append((name, a)) or 0
binding._lib = Calls()
c = binding.Context(binding.Desc.make(8, 2, 64, "bf16", "bf16", 8, 4))
page = 1 << 20
c.set_rope(64)
c.kv_append(page, page, page, page, None, None, page, [3], [20], stream=0)
c.mixed_paged_attention(page, None, None, page, page, None, None, page, [3], [20], 0.0, page, stream=0)
c.tree_attention(page, page, page, None, None, page, None, [3], [20], 0.0, page, stream=0)
c.kv_move(page, page, page, page, page, [3], [20], stream=0)
c.kv_read(page, page, page, page, page, None, [3], page, page, stream=0)
print(" ".join(name for name, a in Calls.made))
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert r.returncode == 0, r.stderr[-2000:]
    assert r.stdout.split() == ["ts_create", "ts_set_rope", "ts_kv_append", "ts_mixed_paged_attention", "ts_tree_attention", "ts_kv_move", "ts_kv_read"]


def test_tensors_are_checked_whenever_torch_was_loaded():
    """A context made before torch is loaded checks tensors as any other."""
    code = """
import sys
from paper_2512_03416_amd import binding
binding.load_library()
class Calls:
    def __getattr__(self, name):
        return lambda *a: 1 << 20 if name == "ts_cache_bytes" else 0
binding._lib = Calls()
assert "torch" not in sys.modules
c = binding.Context(binding.Desc.make(8, 2, 64, "bf16", "bf16", 8, 4), device=-1)      # (-1: where CPU tensors are)
c.kv_move(1, 1, 1, 1, 1, [3], [20], stream=0)
assert "torch" not in sys.modules
import torch
i5, i8, f5 = torch.zeros(5, dtype=torch.int32), torch.zeros(8, dtype=torch.int64), torch.zeros(5)
c.kv_move(1, 1, 1, i5, i5, [3], [20], stream=0)
for bad in (i8, f5):
    try:
        c.kv_move(1, 1, 1, i5, bad, [3], [20], stream=0)
    except ValueError as e:
        assert "expected torch.int32" in str(e), e
    else:
        raise AssertionError(bad.dtype)
q = torch.zeros((3, 8, 64), dtype=torch.bfloat16)
c.tree_attention(q, 1, 1, None, None, 1, torch.zeros((3, 1), dtype=torch.int64), [3], [20], 0.0, q, stream=0)
for bad in ((q.float(), None), (q, i5.view(5, 1))):
    try:
        c.tree_attention(bad[0], 1, 1, None, None, 1, bad[1], [3], [20], 0.0, q, stream=0)
    except ValueError as e:
        assert "expected torch." in str(e), e
    else:
        raise AssertionError(bad)
print("ok")
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stderr[-2000:]
