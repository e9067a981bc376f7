"""Plain 64-bit references of the operators around the paged cache, and batches for their tests."""
import numpy as np
import torch

PAGE = 16
SIZE = {"f32": 4, "bf16": 2, "fp8": 1}
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
CACHE = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}
# Half a step of a type relative to the value.
STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp8": 2.0 ** -4}


def element(which, page, slot, head, dim, Hkv, D, kind):
    """Number of an element in a flat cache buffer (arrays broadcast)."""
    x = 16 // SIZE[kind]
    base = (page.astype(np.int64) * Hkv + head) * (PAGE * D)
    return base + (dim // x * (PAGE * x) + slot * x + dim % x if which == "k" else dim * PAGE + slot)


def places(which, table, seq, pos, Hkv, D, kind):
    """Element numbers of tokens: [token, head, dim]."""
    seq, pos = np.asarray(seq), np.asarray(pos)
    h, d = np.arange(Hkv)[None, :, None], np.arange(D)[None, None, :]
    return element(which, table[seq, pos // PAGE][:, None, None], (pos % PAGE)[:, None, None], h, d, Hkv, D, kind)


class Batch:
    """Sequences over a paged cache whose bytes are normal values, with a quarter of the pool unused; q_lens new tokens or
    nodes at the end of ctx_lens."""

    def __init__(self, heads, dtype, kind, q_lens, ctx_lens, seed=0, extra_width=1):
        self.Hq, self.Hkv, self.D = heads
        self.dtype, self.kind = dtype, kind
        self.q_lens, self.ctx_lens = np.asarray(q_lens, np.int32), np.asarray(ctx_lens, np.int32)
        rng = np.random.default_rng(seed)
        pages = -(-self.ctx_lens // PAGE)
        self.width = int(pages.max(initial=0)) + extra_width
        self.pool = int(pages.sum() * 1.25) + 3
        perm = rng.permutation(self.pool).astype(np.int32)
        self.table = np.full((len(pages), self.width), -1, np.int32)
        at = 0
        for s, n in enumerate(pages):
            self.table[s, :n] = perm[at:at + n]
            at += n
        self.gen = torch.Generator().manual_seed(seed)
        n = self.pool * self.Hkv * PAGE * self.D
        self.k_scale = self.v_scale = None
        if kind == "fp8":
            self.k_scale, self.v_scale = ((0.5 + torch.rand(self.Hkv, generator=self.gen)) / 64 for _ in range(2))
        self.caches = [self.cache_of(torch.randn(n, generator=self.gen)) for _ in range(2)]
        self.T = int(self.q_lens.sum())
        self.seq = np.repeat(np.arange(len(pages)), self.q_lens)
        self.place = np.arange(self.T) - np.repeat(np.cumsum(self.q_lens) - self.q_lens, self.q_lens)
        self.pos = (self.ctx_lens - self.q_lens)[self.seq] + self.place

    def cache_of(self, x):
        return (x * 40).clamp(-448, 448).to(torch.float8_e4m3fn) if self.kind == "fp8" else x.to(CACHE[self.kind])

    def randn(self, *shape):
        return torch.randn(shape, generator=self.gen).to(TORCH[self.dtype])

    def numbers(self, i, cache=None):
        """Cache i (0 K, 1 V) in 64 bits, e4m3 not yet times its scale."""
        return (self.caches[i] if cache is None else cache).double().numpy()

    def tokens(self, i, s, n, cache=None):
        """K or V of the first n tokens of sequence s in 64 bits, [n, head, dim]."""
        at = places("kv"[i], self.table, np.full(n, s), np.arange(n), self.Hkv, self.D, self.kind)
        x = self.numbers(i, cache)[at]
        if self.kind == "fp8":
            x = x * (self.k_scale, self.v_scale)[i].double().numpy()[None, :, None]
        return x

    def desc(self):
        import paper_2512_03416_amd as ts
        return ts.Desc.make(self.Hq, self.Hkv, self.D, self.dtype, self.kind, self.pool, self.width)

    def on_gpu(self):
        """(k cache, v cache, k scale, v scale, table) on the GPU."""
        up = lambda t: None if t is None else t.cuda()  # noqa: E731
        return (*(c.view(torch.uint8).cuda() for c in self.caches), up(self.k_scale), up(self.v_scale), torch.from_numpy(self.table).cuda())


def rotate(x, pos, freq, scale, rot, layout):
    """x [token, head, dim] in 64 bits, pairs turned by pos * freq."""
    y = x.copy()
    a = np.outer(pos.astype(np.float64), freq)[:, None, :]
    c, s = scale * np.cos(a), scale * np.sin(a)
    i = np.arange(rot // 2)
    p, q = (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)
    y[..., p] = x[..., p] * c - x[..., q] * s
    y[..., q] = x[..., q] * c + x[..., p] * s
    return y


def rotate_error(x, scale, rot, layout):
    """Bound of the single-precision arithmetic of `rotate` per element: the angle's rest of at most pi / 4 is off by 2^-24
    three times over (1.4e-7), a power series and the scale round three times more (1.8e-7), and the two products and their
    sum three times (1.8e-7): together below 6e-7 of |x| + |y|."""
    e = np.zeros_like(x)
    i = np.arange(rot // 2)
    p, q = (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)
    m = 6e-7 * scale * (np.abs(x[..., p]) + np.abs(x[..., q]))
    e[..., p], e[..., q] = m, m
    return e


def tree_see(parents):
    n = len(parents)
    see = np.eye(n, dtype=bool)
    for i, p in enumerate(parents):
        if p >= 0:
            see[i] |= see[p]
    return see


def random_tree(rng, n, roots=1):
    return np.array([-1 if i < roots else int(rng.integers(max(0, i - 6), i)) for i in range(n)], np.int32)


def pack_bits(see_list, words=None):
    words = words or max(1, -(-max((s.shape[1] for s in see_list), default=1) // 64))
    rows = []
    for see in see_list:
        m = np.zeros((see.shape[0], words), np.uint64)
        for j in range(see.shape[1]):
            m[:, j // 64] |= see[:, j].astype(np.uint64) << np.uint64(j % 64)
        rows.append(m)
    return np.concatenate(rows) if rows else np.zeros((0, words), np.uint64)


def tree_reference(b, q, see_list, sm_scale=None, cache=None):
    """(out, bound of the kernel's rounding) in 64 bits, [T, Hq, D].

    Bound, with A = sum of weights times |V|: the score of a key is a sum of D products in single precision and two more
    roundings, off by (D + 4) 2^-24 times its terms' absolute sum B (its range of log2 units adds 2^-22), which moves a weight
    by that share twice (numerator and sum); sums over n keys add n 2^-24 twice; the weights enter the second product rounded
    to q's type, and the output is rounded to it."""
    group = b.Hq // b.Hkv
    sm = sm_scale or b.D ** -0.5
    out, bound = np.zeros((b.T, b.Hq, b.D)), np.zeros((b.T, b.Hq, b.D))
    first = 0
    for s, n in enumerate(b.q_lens):
        if n == 0:
            continue
        ctx = int(b.ctx_lens[s])
        k, v = (b.tokens(i, s, ctx, None if cache is None else cache[i]) for i in (0, 1))
        see = np.concatenate([np.ones((n, ctx - n), bool), see_list[s][:n, :n]], 1)
        for h in range(b.Hq):
            kk, vv = k[:, h // group], v[:, h // group]
            qq = q[first:first + n, h].double().numpy()
            for i in range(n):
                keys = np.nonzero(see[i])[0]
                if len(keys) == 0:
                    continue
                with np.errstate(all="ignore"):
                    x = (kk[keys] * qq[i]).sum(1) * sm
                    w = np.exp(x - x.max())
                    w = w / w.sum()
                    out[first + i, h] = (w[:, None] * vv[keys]).sum(0)
                    a = (w[:, None] * np.abs(vv[keys])).sum(0)
                    terms = (np.abs(kk[keys] * qq[i])).sum(1).max() * sm
                    e = 2 * ((b.D + 4) * 2.0 ** -24 * terms + 2.0 ** -22 * (1 + 2 * terms / 32)) + 2 * (len(keys) + 8) * 2.0 ** -24
                    step = STEP[b.dtype] if b.dtype == "bf16" else 2.0 ** -24
                    bound[first + i, h] = a * (e + step) + np.abs(out[first + i, h]) * step + 1e-30
        first += n
    return out, bound


def check(got, want, bound, what=""):
    """Every element within its bound; NaN and infinities where the reference has them."""
    got = got.double().cpu().numpy() if isinstance(got, torch.Tensor) else got
    assert got.shape == want.shape, (got.shape, want.shape)
    same = (np.isnan(got) & np.isnan(want)) | (got == want)
    with np.errstate(invalid="ignore"):
        off = np.where(same, 0.0, np.abs(got - want) - bound)
    bad = ~(off <= 0)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size} elements off, e.g. at {np.argwhere(bad)[0]}: {got[bad][0]} for {want[bad][0]} (bound {np.broadcast_to(bound, got.shape)[bad][0]})"
