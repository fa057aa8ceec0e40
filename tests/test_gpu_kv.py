"""Paged keys and values on the GPU: rotary positions, appends, attention, accumulated weights, eviction, against plain forms in 64 bits.

Tolerances (eps = 2^-8 for bf16 with half steps eps/2 etc., torch.finfo):
* a result rounded once to its type is off by eps/2 of itself;
* a softmax weight is an operand of a product in the element type: off by eps/2 of itself (fp16: or 2^-25 below its normal range), independently, so the sum
  is off by at most eps/2 * sum_j p_j |v_j| (fp16: + 2^-25 sum_j |v_j|, the largest unnormalised weight being 1 or more);
* a score is a sum of head_dim exact products, added in fp32 in steps of 16 with truncation: head_dim / 16 + 4 roundings of at most 2^-23 of the sum of
  the products' magnitudes, 12 * 2^-23 < 2^-19; times the scale that is the relative error of the exponential, twice (weight and norm);
* exponential, logarithm, the product with the scale: 2^-22 each, and 2^-23 of the exponent's size.
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda", 0)
BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def fd():
    import __graft_entry__ as g
    g.build()
    import paper_2609_38198_b200 as fd
    assert torch.cuda.is_available()
    return fd


def randn(seed, *shape, dtype=FP32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype).to(DEV)


# ------------------------------------------------------------------------------------------------ plain forms in 64 bits
def rotate64(x, pos, freqs, layout, scale=1.0, inverse=False):
    r = 2 * freqs.numel()
    a = pos.double()[:, None] * freqs.double()
    c, s = scale * a.cos()[:, None], scale * a.sin()[:, None] * (-1 if inverse else 1)
    y = x.double().clone()
    i = torch.arange(r // 2, device=x.device)
    p, q = (i, i + r // 2) if layout == "half" else (2 * i, 2 * i + 1)
    u, v = x.double()[..., p], x.double()[..., q]
    y[..., p], y[..., q] = u * c - v * s, v * c + u * s
    return y


def rotary_tolerance(x, want, freqs, layout, scale, dtype):
    """Half a step of the result, and 2^-20 of the pair's length: the remainder of an angle is rounded to fp32 (2^-24 of half a turn, pi 2^-24 < 2^-22),
    sine and cosine are off by 2^-22 together, and three fp32 operations follow."""
    r = 2 * freqs.numel()
    i = torch.arange(r // 2, device=x.device)
    p, q = (i, i + r // 2) if layout == "half" else (2 * i, 2 * i + 1)
    size = torch.zeros(x.shape, dtype=torch.float64, device=x.device)
    n = torch.hypot(x.double()[..., p], x.double()[..., q]) * abs(scale)
    size[..., p], size[..., q] = n, n
    tiny = {FP16: 2.0 ** -25, BF16: 0.0, FP32: 0.0}[dtype]
    return torch.finfo(dtype).eps / 2 * want.abs() + 2.0 ** -20 * size + tiny


class Pool:
    """Sequences in shuffled pages; what no sequence owns, and the rows behind each, hold NaN."""

    def __init__(self, fd, seed, kv, new, heads, dim, page, dtype, layout="token", spare=3, cols=0, extra_q=0):
        self.kv, self.new, self.heads, self.dim, self.page, self.dtype = kv, new, heads, dim, page, dtype
        need = [-(-n // page) for n in kv]
        self.pages = sum(need) + spare
        order = torch.from_numpy(np.random.RandomState(seed).permutation(self.pages).astype(np.int32)).to(DEV)
        self.cols = max(need + [1, cols])
        self.table = torch.full((len(kv), self.cols), -1, dtype=torch.int32, device=DEV)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.free = order[at:]
        shape = (self.pages, page, heads, dim) if layout == "token" else (self.pages, heads, page, dim)
        self.k = torch.full(shape, math.nan, dtype=dtype, device=DEV)
        self.v = torch.full(shape, math.nan, dtype=dtype, device=DEV)
        if layout == "head":
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        for b, n in enumerate(kv):
            self.set_rows(b, 0, randn(seed + 17 * b, n, heads, dim, dtype=dtype), randn(seed + 17 * b + 5, n, heads, dim, dtype=dtype))
        self.kv_len = torch.tensor(kv, dtype=torch.int32, device=DEV)
        self.q_start = torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32, device=DEV)
        self.total = sum(new) + extra_q
        self.cache = fd.KVCache(self.k, self.v)
        self.batch = fd.KVBatch(self.table, self.kv_len, self.q_start, self.total, max(new + [0]), max(kv + [0]))

    def where(self, b, slots):
        return self.table[b, slots // self.page].long(), slots % self.page

    def set_rows(self, b, slot0, k, v):
        p, r = self.where(b, torch.arange(slot0, slot0 + k.shape[0], device=DEV))
        self.k[p, r], self.v[p, r] = k, v

    def rows(self, b, n=None):
        p, r = self.where(b, torch.arange(self.kv[b] if n is None else n, device=DEV))
        return self.k[p, r].double(), self.v[p, r].double()


def attend64(pool, q, scale, causal=True, window=0):
    """(out, lse, weights per sequence, tolerance of out, relative tolerance of a weight) in 64 bits."""
    Hq = q.shape[1]
    G = Hq // pool.heads
    out = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    tol = torch.zeros_like(out)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=DEV)
    weights, rel = [], 0.0
    half, tiny = torch.finfo(q.dtype).eps / 2, (2.0 ** -25 if q.dtype == FP16 else 0.0)
    t = 0
    for b, (n, m) in enumerate(zip(pool.kv, pool.new)):
        k, v = pool.rows(b)
        w = torch.zeros(pool.heads, n, dtype=torch.float64, device=DEV)
        at = torch.arange(m, device=DEV)[:, None] + n - m
        j = torch.arange(n, device=DEV)[None]
        see = (j <= at) & ((j > at - window) if window else True) if causal else (j >= 0).expand(m, n)
        for h in range(Hq):
            if not (n and m):
                continue
            x, kk, vv = q[t:t + m, h].double(), k[:, h // G], v[:, h // G]
            s = torch.where(see, x @ kk.T * scale, -math.inf)
            top = s.amax(1, keepdim=True)
            e = torch.where(see, torch.exp(s - torch.where(top == -math.inf, 0.0, top)), 0.0)
            l = e.sum(1, keepdim=True)
            p = torch.where(l == 0, 0.0, e / l)
            # a weight of 0 times what is not finite is left out: the definition sums over what a row sees
            out[t:t + m, h] = torch.where(see[..., None], p[..., None] * vv, 0.0).sum(1) if not torch.isfinite(vv).all() else p @ vv
            lse[t:t + m, h] = torch.where(l[:, 0] == 0, -math.inf, top[:, 0] + l[:, 0].log())
            w[h // G] += p.sum(0)
            kf, vf = torch.nan_to_num(kk.abs(), posinf=0.0), torch.nan_to_num(vv.abs(), posinf=0.0)
            sure = 2.0 ** -19 * scale * float((x.abs() @ kf.T).max()) + 2.0 ** -22 * (8 + float(torch.nan_to_num(s.abs(), posinf=0.0).max()))
            rel = max(rel, 2 * sure)
            tol[t:t + m, h] = (half + 2 * sure) * (torch.nan_to_num(p) @ vf) + tiny * (see.double() @ vf) + tiny + half * out[t:t + m, h].abs().nan_to_num(posinf=0.0)
        weights.append(w)
        t += m
    return out, lse, weights, tol, rel


def check_attend(fd, pool, q, scale=None, causal=True, window=0, weigh=True, **kw):
    scale = pool.dim ** -0.5 if scale is None else scale
    want, lse, weights, tol, rel = attend64(pool, q, scale, causal, window)
    live = sum(pool.new)
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device=DEV)
    got_lse = torch.full(q.shape[:2], 7.0, device=DEV)
    B, L = len(pool.kv), max(pool.kv + [0]) + 3
    w_in = torch.rand(B, pool.heads, L, device=DEV)
    w = w_in.clone()
    pool.cache.attend(pool.batch, q, scale=scale, causal=causal, window=window, out=out, lse=got_lse, weights=w if weigh else None, **kw)
    pool.cache.synchronize()
    assert (out[live:] == 7.0).all() and (got_lse[live:] == 7.0).all(), "rows behind the last sequence"
    err = (out[:live].double() - want[:live]).abs()
    fine = torch.isfinite(want[:live])
    assert torch.equal(torch.isfinite(out[:live]), fine)
    assert torch.equal(torch.isnan(out[:live]), torch.isnan(want[:live]))
    assert (err <= tol[:live])[fine].all(), f"worst {float((err / tol[:live].clamp(min=1e-300))[fine].max()):.3g} of the tolerance"
    empty = lse[:live] == -math.inf
    assert torch.equal(got_lse[:live] == -math.inf, empty)
    assert (out[:live][empty] == 0).all()
    sure = torch.isfinite(lse[:live])
    e = (got_lse[:live].double() - lse[:live]).abs()[sure]
    assert (e <= rel + 2.0 ** -21 * (1 + lse[:live][sure].abs())).all()
    if weigh:
        for b, n in enumerate(pool.kv):
            e = (w[b, :, :n].double() - w_in[b, :, :n].double() - weights[b]).abs()
            assert (e <= weights[b] * (rel + 2.0 ** -20 * (1 + 40)) + 2.0 ** -22 * (w_in[b, :, :n] + weights[b])).all(), float(e.max())
            assert torch.equal(w[b, :, n:], w_in[b, :, n:]), "weights behind a sequence"
    return out, got_lse, w


# ------------------------------------------------------------------------------------------------ rotary positions
@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("tokens,heads,dim,rot,first", [(1, 1, 2, 2, 0), (3, 5, 64, 64, 7), (17, 3, 128, 32, 1 << 30), (700, 2, 96, 96, 100000),
                                                        (5, 2, 80, 20, 3), (2500, 4, 64, 48, 2 ** 31 - 2501)])
def test_rotary(fd, dtype, layout, tokens, heads, dim, rot, first):
    x = randn(1, tokens, heads, dim, dtype=dtype)
    pos = (first + torch.arange(tokens, device=DEV)).to(torch.int32)
    freqs = fd.fd_rotary_frequencies(rot, scaling="ramp", factor=4.0, original_len=4096, device=DEV)
    for inverse, scale in ((False, 1.0), (True, 1.25)):
        y = fd.fd_rotary(x, pos, freqs, layout=layout, scale=scale, inverse=inverse)
        want = rotate64(x, pos, freqs, layout, scale, inverse)
        assert ((y.double() - want).abs() <= rotary_tolerance(x, want, freqs, layout, scale, dtype)).all()
        assert torch.equal(y[..., rot:], x[..., rot:])
    z = x.clone()
    assert fd.fd_rotary(z, pos, freqs, layout=layout, out=z) is z
    assert torch.equal(z, fd.fd_rotary(x, pos, freqs, layout=layout))


def test_rotary_gradient(fd):
    """<g, R x> = <R^T g, x>, and R^T g against differences of <g, R x> (R is linear: differences of any width are exact but for rounding)."""
    x, g = randn(2, 9, 3, 64), randn(3, 9, 3, 64)
    pos = torch.arange(40, 49, dtype=torch.int32, device=DEV)
    freqs = fd.fd_rotary_frequencies(32, device=DEV)
    for layout in ("half", "interleaved"):
        back = fd.fd_rotary(g, pos, freqs, layout=layout, scale=1.5, inverse=True).double()
        f = lambda u: float((g.double() * fd.fd_rotary(u, pos, freqs, layout=layout, scale=1.5).double()).sum())  # noqa: E731
        # each of the 1728 terms is off by 2^-20 of its size
        room = 2.0 ** -20 * 2 * 1.5 * float((g.abs().double() * x.abs().double()).sum() + g.abs().sum())
        assert abs(f(x) - float((back * x.double()).sum())) <= 2 * room
        for t, h, i in ((0, 0, 0), (3, 1, 17), (8, 2, 40), (5, 0, 31)):
            d = torch.zeros_like(x)
            d[t, h, i] = 1.0
            assert abs((f(x + d) - f(x - d)) / 2 - float(back[t, h, i])) <= 2 * room


def test_rotary_strides_and_refusals(fd):
    big = randn(4, 6, 4, 200, dtype=BF16)
    pos = torch.arange(6, dtype=torch.int32, device=DEV)
    freqs = fd.fd_rotary_frequencies(64, device=DEV)
    for off in (0, 8, 3):                                    # (3: not 16-byte aligned)
        x = big[:, ::2, off:off + 64]
        out = torch.zeros(2, 6, 64, dtype=BF16, device=DEV).transpose(0, 1)
        y = fd.fd_rotary(x, pos, freqs, out=out)
        assert y is out and torch.equal(out, fd.fd_rotary(x.contiguous(), pos, freqs))
    x = randn(5, 6, 2, 64, dtype=BF16)
    for bad in (dict(positions=pos.long()), dict(positions=pos[:5]), dict(freqs=freqs.float()), dict(freqs=torch.cat([freqs, freqs])), dict(layout="other"),
                dict(x=x.double()), dict(x=x[0]), dict(x=x.cpu()), dict(x=x.transpose(1, 2)), dict(scale=math.inf), dict(out=x[:, :1])):
        with pytest.raises(fd.FdError):
            fd.fd_rotary(**{"x": x, "positions": pos, "freqs": freqs, **bad})
    assert fd.fd_rotary(x[:0], pos[:0], freqs).shape == (0, 2, 64)


# ------------------------------------------------------------------------------------------------ append
@pytest.mark.parametrize("dtype,dim,page,layout,heads,group", [(BF16, 128, 16, "half", 8, 4), (FP16, 64, 24, "interleaved", 2, 7), (BF16, 64, 8, "half", 1, 1)])
@pytest.mark.parametrize("pool_layout", ["token", "head"])
def test_append(fd, dtype, dim, page, layout, heads, group, pool_layout):
    kv, new = [1, 40, 129, 17, 300], [1, 3, 129, 0, 5]
    p = Pool(fd, 11, kv, new, heads, dim, page, dtype, pool_layout, extra_q=2)
    before_k, before_v = p.k.clone(), p.v.clone()
    T = p.total
    k, v, q = (randn(s, T, h, dim, dtype=dtype) for s, h in ((1, heads), (2, heads), (3, heads * group)))
    pos = torch.arange(1000, 1000 + T, dtype=torch.int32, device=DEV)
    freqs = fd.fd_rotary_frequencies(dim // 2, device=DEV)
    qo = torch.full_like(q, 7.0)
    assert p.cache.append(p.batch, k, v, positions=pos, freqs=freqs, layout=layout, q=q, scale=1.1, q_out=qo) is qo
    p.cache.synchronize()
    want_q = rotate64(q, pos, freqs, layout, 1.1)
    assert ((qo.double() - want_q).abs() <= rotary_tolerance(q, want_q, freqs, layout, 1.1, dtype))[:-2].all()
    assert (qo[-2:] == 7.0).all(), "rows behind the last sequence"
    t = 0
    turned = fd.fd_rotary(k, pos, freqs, layout=layout, scale=1.1)
    for b, (n, m) in enumerate(zip(kv, new)):
        pg, r = p.where(b, torch.arange(n - m, n, device=DEV))
        assert torch.equal(p.k[pg, r], turned[t:t + m]) and torch.equal(p.v[pg, r], v[t:t + m])
        before_k[pg, r], before_v[pg, r] = turned[t:t + m], v[t:t + m]
        t += m
    same = lambda a, b: torch.equal(torch.nan_to_num(a.float(), nan=99.0), torch.nan_to_num(b.float(), nan=99.0))  # noqa: E731
    assert same(p.k, before_k) and same(p.v, before_v), "other rows of the pool"
    p.cache.append(p.batch, k, v)                            # without positions: as they are
    p.cache.synchronize()
    pg, r = p.where(2, torch.arange(129, device=DEV))
    assert torch.equal(p.k[pg, r], k[4:133]) and torch.equal(p.v[pg, r], v[4:133])


# ------------------------------------------------------------------------------------------------ attention
SHAPES = [  # kv, new, heads, group, dim, page, dtype
    ([1], [1], 1, 1, 64, 8, BF16),
    ([700], [1], 8, 4, 128, 16, BF16),
    ([128, 127, 129, 1, 256, 33], [1] * 6, 2, 8, 128, 16, FP16),
    ([300, 5, 64], [3, 5, 1], 2, 7, 64, 24, BF16),
    ([1000, 250, 513], [200, 250, 77], 2, 3, 128, 32, FP16),
    ([700, 300], [260, 300], 1, 16, 64, 160, BF16),
    ([400], [129], 1, 128, 64, 128, FP16),
    ([0, 20, 0, 9], [0, 0, 1, 20], 2, 2, 64, 8, BF16),       # nothing cached, nothing new, rows that see nothing
    ([5000], [1], 2, 5, 64, 64, FP16),                       # the cache in parts
    ([9000, 100], [2, 1], 1, 4, 128, 16, BF16),
]


@pytest.mark.parametrize("case", range(len(SHAPES)))
@pytest.mark.parametrize("mask", ["causal", "window 1", "window 100", "all"])
def test_attend(fd, case, mask):
    kv, new, heads, group, dim, page, dtype = SHAPES[case]
    p = Pool(fd, 31 + case, kv, new, heads, dim, page, dtype, extra_q=3)
    q = randn(5, p.total, heads * group, dim, dtype=dtype, scale=2.0)
    window = int(mask.split()[1]) if mask.startswith("window") else 0
    check_attend(fd, p, q, causal=mask != "all", window=window)


def test_attend_large_scores(fd):
    """Scores up to some hundreds: the running maximum is raised again and again, in rising and falling order."""
    for order in (1, -1):
        p = Pool(fd, 7, [1500], [140], 1, 64, 16, BF16)
        k, v = p.rows(0)
        k = k * torch.linspace(0.1, 6, 1500, device=DEV, dtype=torch.float64)[::1, None, None]
        p.set_rows(0, 0, (k if order == 1 else k.flip(0)).to(BF16), v.to(BF16))
        check_attend(fd, p, randn(8, 140, 4, 64, dtype=BF16, scale=8.0))


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("new,group", [(1, 4), (150, 2)])
def test_attend_values_that_are_not_finite(fd, bad, new, group):
    """What a row sees reaches it, what it does not see cannot: in keys and in values, in whole tiles and in the last."""
    n = 600
    for j in (0, n - new, n - 1, n - new // 2 - 1):
        p = Pool(fd, 3, [n], [new], 2, 64, 16, FP16)
        k, v = p.rows(0)
        v[j, 1, 5] = bad
        p.set_rows(0, 0, k.to(FP16), v.to(FP16))
        check_attend(fd, p, randn(9, new, 2 * group, 64, dtype=FP16))
        if math.isnan(bad) and new > 1:
            p = Pool(fd, 3, [n], [new], 2, 64, 16, FP16)
            k, v = p.rows(0)
            k[j, 0, 9] = bad
            p.set_rows(0, 0, k.to(FP16), v.to(FP16))
            out, lse = p.cache.attend(p.batch, randn(9, new, 2 * group, 64, dtype=FP16))
            hit = torch.arange(new, device=DEV) >= j - (n - new)
            assert torch.equal(torch.isnan(out[:, :group]).all(-1).all(-1), hit)
            assert torch.isfinite(out[~hit]).all() and torch.isfinite(out[:, group:]).all() and torch.isfinite(lse[~hit]).all()


def test_attend_pool_and_tensor_strides(fd):
    p = Pool(fd, 5, [300, 40], [20, 1], 4, 128, 16, BF16, "head")
    big = randn(6, 21, 10, 256, dtype=BF16)
    q = big[:, 1:9, 128:]
    out, _, _ = check_attend(fd, p, q)
    wide = torch.zeros(8, 21, 136, dtype=BF16, device=DEV)
    view = wide.transpose(0, 1)[..., :128]
    got, _ = p.cache.attend(p.batch, q, out=view)
    assert got is view and torch.equal(view, out) and (wide[..., 128:] == 0).all()


def test_attend_long_sums_of_one_sign(fd):
    """131072 tokens whose values are all positive: truncation in the tensor core's accumulator adds up to no more than a quarter step of fp16 (2^-12) on average.
    One CTA's accumulator would lose 8e-4."""
    n, m, heads, dim = 131072, 4096, 8, 64
    g = torch.Generator(device=DEV).manual_seed(1)
    k = (torch.randn(n // 64, 64, heads, dim, device=DEV, generator=g) * 0.5).half()
    v = (1 + torch.rand(dim, device=DEV, generator=g) + 0.1 * torch.rand(n // 64, 64, heads, dim, device=DEV, generator=g)).half()
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    cache = fd.KVCache(k, v)
    batch = fd.KVBatch(torch.arange(n // 64, dtype=torch.int32, device=DEV)[None], i32(n), i32(0, m), m, m, n)
    q = torch.randn(m, heads, dim, device=DEV, generator=g).half()
    out, lse = cache.attend(batch, q, causal=False)
    cache.synchronize()
    for h in (0, heads - 1):
        s = q[:64, h].double() @ k[:, :, h].reshape(n, dim).double().T / 8
        want = torch.softmax(s, -1) @ v[:, :, h].reshape(n, dim).double()
        assert abs(float((out[:64, h].double() / want - 1).mean())) <= 2.0 ** -12
        assert (lse[:64, h].double() - torch.logsumexp(s, -1)).abs().max() < 1e-5


def test_attend_far_offsets(fd):
    """A pool of more than 2^32 bytes and 2^31 elements a tensor: pages at its end."""
    pages, page, heads, dim = 70000, 32, 8, 128              # 2.3e9 elements
    k = torch.empty(pages, page, heads, dim, dtype=BF16, device=DEV)
    v = torch.empty(pages, page, heads, dim, dtype=BF16, device=DEV)
    table = torch.tensor([[69999, 5, 69990, 68000]], dtype=torch.int32, device=DEV)
    n = 120
    kk, vv = randn(1, n, heads, dim, dtype=BF16), randn(2, n, heads, dim, dtype=BF16)
    cache = fd.KVCache(k, v)
    start = lambda m: torch.tensor([0, m], dtype=torch.int32, device=DEV)  # noqa: E731
    length = torch.tensor([n], dtype=torch.int32, device=DEV)
    cache.append(fd.KVBatch(table, length, start(n), n, n, n), kk, vv)
    small = Pool(fd, 5, [n], [9], heads, dim, page, BF16)
    small.set_rows(0, 0, kk, vv)
    q = randn(3, 9, 16, dim, dtype=BF16)
    out, lse = cache.attend(fd.KVBatch(table, length, start(9), 9, 9, n), q)
    ref, ref_lse = small.cache.attend(small.batch, q)
    assert torch.equal(out, ref) and torch.equal(lse, ref_lse)
    w = torch.rand(1, heads, n, device=DEV)
    w2 = w.clone()
    b0 = fd.KVBatch(table, length, start(0), 0, 0, n)
    kept, new_len, w = cache.evict(b0, w, 50, first=1, recent=9)
    small.total = 0
    kept2, _, w2 = small.cache.evict(fd.KVBatch(small.table, small.kv_len, start(0), 0, 0, n), w2, 50, first=1, recent=9)
    assert torch.equal(kept, kept2) and torch.equal(w, w2)
    cache.synchronize()
    slots = torch.arange(50, device=DEV)
    assert torch.equal(k[table[0, slots // page].long(), slots % page], small.rows(0, 50)[0].to(BF16))


def test_attend_bad_pages_and_lengths(fd):
    """A page outside the pool is never followed, a length beyond the table is cut, and both are reported once."""
    for what in ("page", "negative", "length", "short", "minus"):
        p = Pool(fd, 5, [300, 300], [4, 4], 2, 64, 16, BF16)
        q = randn(6, 8, 4, 64, dtype=BF16)
        good, _ = p.cache.attend(p.batch, q)
        if what == "page":
            p.table[0, 3] = p.pages + 7
        if what == "negative":
            p.table[0, 18] = -5
        if what == "length":
            p.kv_len[0] = 1 << 29
        if what == "minus":
            p.kv_len[0] = -3
        if what == "short":
            p.batch.struct.max_len = 200
            p.kv_len[1] = 200
        out, _ = p.cache.attend(p.batch, q)
        with pytest.raises(fd.FdError) as e:
            p.cache.synchronize()
        assert e.value.status == fd.FD_ERR_INVALID
        if what != "short":
            assert torch.equal(out[4:], good[4:]), "the other sequence"
        p.cache.synchronize()                                # cleared
        if what in ("page", "negative"):
            p.cache.append(p.batch, randn(1, 8, 2, 64, dtype=BF16), randn(2, 8, 2, 64, dtype=BF16))
            if what == "negative":
                with pytest.raises(fd.FdError):
                    p.cache.synchronize()


@pytest.mark.parametrize("new", [1, 40])
def test_attend_loose_bounds(fd, new):
    """Bounds far above the lengths (a captured step is sized for the longest context), pages for them, and a window beyond every length."""
    p = Pool(fd, 5, [300, 1, 2000], [new, 1, new], 2, 64, 16, BF16, cols=20000)
    q = randn(6, p.total, 8, 64, dtype=BF16)
    tight, lse, w = check_attend(fd, p, q)
    loose = fd.KVBatch(p.table, p.kv_len, p.q_start, p.total, new, 300000)
    wl = torch.zeros(3, 2, 300000, device=DEV)
    out, lse2 = p.cache.attend(loose, q, weights=wl, window=2 ** 31 - 1)
    p.cache.synchronize()
    # (the cache may be cut elsewhere, so sums are taken in another order)
    assert ((out.double() - tight.double()).abs() <= 2.0 ** -7 * tight.double().abs() + 2.0 ** -9).all() and (lse2 - lse).abs().max() < 1e-5
    want = torch.zeros_like(wl[:, :, :2003])
    p.cache.attend(p.batch, q, weights=want)
    n = p.kv_len.long()[:, None, None]
    assert ((wl[:, :, :2003] - want).abs() <= 1e-5 * want + 1e-7).all() and (wl[torch.arange(300000, device=DEV).expand_as(wl) >= n] == 0).all()


def test_attend_more_new_tokens_than_promised(fd):
    """max_new chose the kernel for few rows; a sequence with more rows than it holds is left out and reported, the others are answered."""
    p = Pool(fd, 5, [300, 200], [1, 30], 2, 64, 16, BF16)
    q = randn(6, 31, 8, 64, dtype=BF16)
    good, _ = p.cache.attend(p.batch, q)
    out = torch.full_like(q, 7.0)
    w = torch.rand(2, 2, 300, device=DEV)
    w0 = w.clone()
    p.cache.attend(fd.KVBatch(p.table, p.kv_len, p.q_start, 31, 1, 300), q, out=out, weights=w)
    with pytest.raises(fd.FdError) as e:
        p.cache.synchronize()
    assert e.value.status == fd.FD_ERR_INVALID
    assert ((out[0].double() - good[0].double()).abs() <= 2.0 ** -7 * good[0].double().abs() + 2.0 ** -9).all()
    assert (out[1:] == 7.0).all() and torch.equal(w[1], w0[1])


@pytest.mark.parametrize("batch", [300, 2000])
def test_attend_many_sequences(fd, batch):
    """More sequences than a block has threads, a third of them without a new token, some empty."""
    rng = np.random.RandomState(batch)
    kv = [int(x) for x in rng.randint(0, 90, batch)]
    new = [int(x) for x in rng.randint(0, 3, batch)]
    p = Pool(fd, 9, kv, new, 1, 64, 8, FP16)
    check_attend(fd, p, randn(3, p.total, 4, 64, dtype=FP16))


def test_attend_refusals(fd):
    p = Pool(fd, 5, [30, 20], [2, 1], 2, 64, 16, BF16)
    q = randn(6, 3, 4, 64, dtype=BF16)
    w = torch.zeros(2, 2, 30, device=DEV)
    launches = fd.fd_launch_count()
    for bad in (dict(q=q.half()), dict(q=q[:2]), dict(q=q[..., :32]), dict(q=q[:, :3]), dict(q=q.cpu()), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan),
                dict(window=-1), dict(window=5, causal=False), dict(out=q), dict(out=q[:, :2]), dict(lse=torch.zeros(3, 3, device=DEV)),
                dict(weights=w[..., :20].contiguous()), dict(weights=w[:1]), dict(weights=w.double()), dict(weights=w, weights_out=torch.zeros(2, 2, 31, device=DEV)),
                dict(q=randn(6, 3, 4, 68, dtype=BF16)[..., 2:66]), dict(q=randn(6, 3, 4, 68, dtype=BF16)[..., :64])):
        with pytest.raises(fd.FdError):
            p.cache.attend(**{"batch": p.batch, "q": q, **bad})
    with pytest.raises(fd.FdError):
        p.cache.attend(p.batch, randn(6, 3, 2 * 129, 64, dtype=BF16))
    for bad in (dict(keep=0), dict(first=-1), dict(first=5, recent=6, keep=10), dict(recent=-1), dict(new_table=p.table[:, :0]), dict(new_table=p.table.long()),
                dict(kept=torch.zeros(2, 2, 9, dtype=torch.int32, device=DEV)), dict(weights=w[:, :1])):
        with pytest.raises(fd.FdError):
            p.cache.evict(**{"batch": p.batch, "weights": w, "keep": 10, **bad})
    with pytest.raises(fd.FdError):
        p.cache.append(p.batch, q, q)
    with pytest.raises(fd.FdError):
        fd.KVCache(p.k[..., :32], p.v[..., :32])
    with pytest.raises(fd.FdError):
        fd.KVCache(p.k.float(), p.v.float())
    assert fd.fd_launch_count() == launches
    short = fd.lib.fd_kv_attend                              # a workspace that is too small
    long = Pool(fd, 5, [5000], [1], 1, 64, 16, BF16)
    import ctypes
    from paper_2609_38198_b200 import binding
    qq, oo = randn(1, 1, 4, 64, dtype=BF16), torch.zeros(1, 4, 64, dtype=BF16, device=DEV)
    a = binding.fd_kv_attend_args(binding.fd_heads(qq.data_ptr(), 256, 64, 4), binding.fd_heads(oo.data_ptr(), 256, 64, 4), 0.125, 1, 0)
    assert fd.lib.fd_kv_attend_bytes(long.cache._h, ctypes.byref(long.batch.struct), 4, 0) > 0
    assert short(long.cache._h, ctypes.byref(long.batch.struct), ctypes.byref(a), None, 0, None, None, 0) == fd.FD_ERR_WORKSPACE


def test_attend_repeats_bits_and_other_streams(fd):
    p = Pool(fd, 5, [5000, 3000, 700], [1, 40, 1], 2, 128, 16, BF16)
    q = randn(6, 42, 8, 128, dtype=BF16)
    w = torch.rand(3, 2, 5000, device=DEV)
    ref = p.cache.attend(p.batch, q, weights=w, weights_out=torch.zeros_like(w))
    ref_w = torch.zeros_like(w)
    p.cache.attend(p.batch, q, weights=w, weights_out=ref_w)
    torch.cuda.synchronize()
    side = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for _ in range(4):
        for s in side:
            with torch.cuda.stream(s):
                wo = torch.zeros_like(w)
                got.append((*p.cache.attend(p.batch, q, weights=w, weights_out=wo), wo))
    torch.cuda.synchronize()
    for o, l, wo in got:
        assert torch.equal(o, ref[0]) and torch.equal(l, ref[1]) and torch.equal(wo[0], ref_w[0]) and torch.equal(wo[1, :, :3000], ref_w[1, :, :3000])


def test_steps_in_a_graph(fd):
    """One decoding step (append, attention with totals) captured, replayed with new lengths, positions and tokens; two graphs in turn."""
    kv, heads, group, dim, page = [140, 1000], 2, 4, 128, 16
    p = Pool(fd, 5, kv, [1, 1], heads, dim, page, BF16)
    ref = Pool(fd, 5, kv, [1, 1], heads, dim, page, BF16)
    freqs = fd.fd_rotary_frequencies(dim, device=DEV)
    st = {n: torch.zeros(2, h, dim, dtype=BF16, device=DEV) for n, h in (("q", heads * group), ("k", heads), ("v", heads))}
    pos = torch.zeros(2, dtype=torch.int32, device=DEV)
    w = torch.zeros(2, heads, 1000, device=DEV)
    w_ref = w.clone()

    def step(pool, weights):
        q = pool.cache.append(pool.batch, st["k"], st["v"], positions=pos, freqs=freqs, q=st["q"])
        return pool.cache.attend(pool.batch, q, weights=weights)

    p.kv_len.copy_(torch.tensor([101, 900], dtype=torch.int32))
    graphs = []
    for _ in range(2):
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            out = step(p, w)
        graphs.append((g, out))
    for i in range(6):
        for n, t in st.items():
            t.copy_(randn(100 * i + len(n), *t.shape, dtype=BF16))
        n = torch.tensor([102 + i, 901 + 9 * i], dtype=torch.int32, device=DEV)
        p.kv_len.copy_(n)
        ref.kv_len.copy_(n)
        pos.copy_(n - 1)
        g, out = graphs[i % 2]
        g.replay()
        want = step(ref, w_ref)
        torch.cuda.synchronize()
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1]) and torch.equal(w, w_ref)
    p.cache.synchronize()


# ------------------------------------------------------------------------------------------------ eviction
def evict_plain(w, n, keep, first, recent):
    """Kept slots of one head: the first, the recent, and the largest of the others (of equal ones the earlier)."""
    if n <= keep:
        return np.arange(n)
    lo, hi = first, n - recent
    x = np.where(np.isnan(w[lo:hi]), -np.inf, w[lo:hi].astype(np.float64))
    nan = np.isnan(w[lo:hi])
    order = sorted(range(hi - lo), key=lambda i: (-x[i], nan[i], i))[:keep - first - recent]
    return np.sort(np.concatenate([np.arange(lo), lo + np.array(order, dtype=np.int64), np.arange(hi, n)]).astype(np.int64))


@pytest.mark.parametrize("kind", ["random", "ties", "equal", "special"])
@pytest.mark.parametrize("keep,first,recent", [(100, 4, 20), (1, 0, 0), (1, 1, 0), (64, 32, 32), (777, 0, 500), (5000, 3, 9)])
@pytest.mark.parametrize("in_place", [False, True])
def test_evict(fd, kind, keep, first, recent, in_place):
    kv, heads, dim, page = [1, 100, 101, 1500, 0, 3001], 2, 64 if keep % 2 else 128, 24
    dtype = FP16 if in_place else BF16
    cols = -(-keep // page)
    p = Pool(fd, 13, kv, [0] * 6, heads, dim, page, dtype, spare=6 * cols + 2, cols=cols if in_place else 0)
    rng = np.random.RandomState(keep)
    w = rng.rand(6, heads, 3001).astype(np.float32)
    if kind == "ties":
        w = np.floor(w * 4).astype(np.float32)
    if kind == "equal":
        w[:] = 0.25
    if kind == "special":
        w = rng.choice(np.array([0.0, -0.0, 1e-40, -1.0, np.inf, -np.inf, np.nan, 3.4e38], dtype=np.float32), w.shape)
    wd = torch.from_numpy(w).to(DEV)
    old = [p.rows(b) for b in range(6)]
    table = p.table if in_place else p.free[:6 * cols].reshape(6, cols).contiguous()
    w_out = wd if in_place else torch.full_like(wd, 5.0)
    new_len = p.kv_len if in_place else None
    # pages that no sequence of the batch owns may be out of the pool behind a short sequence's last page
    kept, got_len, w_new = p.cache.evict(p.batch, wd, keep, first=first, recent=recent, new_table=table, new_len=new_len, weights_out=w_out)
    p.cache.synchronize()
    assert got_len.tolist() == [min(n, keep) for n in kv]
    for b, n in enumerate(kv):
        for h in range(heads):
            want = evict_plain(w[b, h, :n], n, keep, first, recent)
            m = len(want)
            assert kept[b, h].tolist() == want.tolist() + [-1] * (keep - m)
            slots = torch.arange(m, device=DEV)
            pg, r = table[b, slots // page].long(), slots % page
            src = torch.from_numpy(want).to(DEV)
            assert torch.equal(p.k[pg, r, h].double(), old[b][0][src, h]) and torch.equal(p.v[pg, r, h].double(), old[b][1][src, h])
            have = w_new[b, h].cpu().numpy()
            assert np.array_equal(have[:m], w[b, h, want], equal_nan=True) and (have[m:n] == 0).all()
            assert np.array_equal(have[n:], w[b, h, n:] if in_place else np.full(3001 - n, 5.0, np.float32), equal_nan=True)


@pytest.mark.parametrize("kind", ["random", "ties"])
def test_evict_long(fd, kind):
    """Beyond what a block keeps in shared memory (40960 tokens), and beyond 4096 (more threads)."""
    kv, keep = [45000, 5000, 41500], 3000
    p = Pool(fd, 17, kv, [0] * 3, 1, 64, 64, BF16)
    w = np.random.RandomState(4).rand(3, 1, 45000).astype(np.float32)
    if kind == "ties":
        w = np.floor(w * 3).astype(np.float32)
    wd = torch.from_numpy(w).to(DEV)
    old = [p.rows(b) for b in range(3)]
    kept, n, w_new = p.cache.evict(p.batch, wd, keep, first=7, recent=300)
    p.cache.synchronize()
    assert n.tolist() == [keep] * 3
    for b in range(3):
        want = evict_plain(w[b, 0, :kv[b]], kv[b], keep, 7, 300)
        assert kept[b, 0].tolist() == want.tolist()
        now = p.rows(b, keep)
        src = torch.from_numpy(want).to(DEV)
        assert torch.equal(now[0], old[b][0][src]) and torch.equal(now[1], old[b][1][src])
        assert np.array_equal(w_new[b, 0, :keep].cpu().numpy(), w[b, 0, want]) and (w_new[b, 0, keep:kv[b]] == 0).all()


def test_decode_with_eviction(fd):
    """A prompt, decoding steps that keep totals, evictions in place, and on: against the same in 64 bits on the rows that the kept slots say."""
    heads, group, dim, page, budget = 2, 4, 64, 16, 96
    p = Pool(fd, 21, [400], [1], heads, dim, page, BF16, spare=10)
    freqs = fd.fd_rotary_frequencies(dim, device=DEV)
    cols = p.cols
    w = torch.zeros(1, heads, 512, device=DEV)
    n, seen = 0, 0                                          # tokens in the cache, tokens in all
    history_k, history_v = [[] for _ in range(heads)], [[] for _ in range(heads)]
    for i, m in enumerate([90, 1, 1, 70, 1, 1, 1, 33, 1]):
        n += m
        assert n <= cols * page
        q, k, v = (randn(7 * i + s, m, h, dim, dtype=BF16) for s, h in ((1, heads * group), (2, heads), (3, heads)))
        pos = torch.arange(seen, seen + m, dtype=torch.int32, device=DEV)
        batch = fd.KVBatch(p.table, torch.tensor([n], dtype=torch.int32, device=DEV), torch.tensor([0, m], dtype=torch.int32, device=DEV), m, m, n)
        q = p.cache.append(batch, k, v, positions=pos, freqs=freqs, q=q)
        turned = fd.fd_rotary(k, pos, freqs)
        for h in range(heads):
            history_k[h] += list(turned[:, h].double())
            history_v[h] += list(v[:, h].double())
        p.kv, p.new = [n], [m]
        rows = [torch.stack(x, 0) for hh in (history_k, history_v) for x in hh]
        pk, pv = p.rows(0)
        for h in range(heads):
            assert torch.equal(pk[:, h], rows[h]) and torch.equal(pv[:, h], rows[heads + h])
        want, lse, weights, tol, rel = attend64(p, q, dim ** -0.5)
        before = w.clone()
        out, got_lse = p.cache.attend(batch, q, weights=w)
        assert ((out.double() - want).abs() <= tol).all()
        assert ((w[0, :, :n].double() - before[0, :, :n] - weights[0]).abs() <= weights[0] * (rel + 2.0 ** -15) + 2.0 ** -22 * (before[0, :, :n] + weights[0])).all()
        seen += m
        if n > budget:
            kept, new_len, _ = p.cache.evict(batch, w, budget, first=2, recent=30)
            assert new_len.tolist() == [budget]
            for h in range(heads):
                history_k[h] = [history_k[h][j] for j in kept[0, h].tolist()]
                history_v[h] = [history_v[h][j] for j in kept[0, h].tolist()]
            n = budget
    p.cache.synchronize()


def test_attend_against_the_kernel_product(fd):
    """softmax over 2 beta x.y is the row-normalised Gaussian product with exp(beta |y|^2) on the right: attention agrees with the framework's own product of
    the same points (relative Frobenius error 1e-5 there)."""
    n, m, dim, beta = 700, 130, 32, 4.0
    x = torch.zeros(n + m, 64, device=DEV)
    x[:, :dim] = torch.nn.functional.normalize(randn(1, n + m, dim), dim=1)
    x = x.to(BF16)
    v = randn(2, n, 64, dtype=BF16)
    p = Pool(fd, 5, [n], [m], 1, 64, 16, BF16)
    p.set_rows(0, 0, x[:n, None], v[:, None])
    q = x[n:, None].contiguous()
    out, _ = p.cache.attend(p.batch, q, scale=2 * beta, causal=False)
    points = x[:, :dim].float().contiguous()
    ctx = fd.Context(points[:n], b_max=64)
    right = torch.exp(beta * (points[:n] ** 2).sum(1))
    num = ctx.apply_general(beta, v.float().t().contiguous().t(), right=right, Xrow=points[n:])
    den = ctx.apply_general(beta, None, right=right, Xrow=points[n:])
    ctx.synchronize()
    want = num.double() / den.double()
    _, _, _, tol, _ = attend64(p, q, 2 * beta, causal=False)
    assert float((out[:, 0].double() - want).norm()) <= float(tol.norm()) + 2e-5 * float(want.norm())
    ctx.close()


# ------------------------------------------------------------------------------------------------ workspaces, bounds, aliases
def attend_raw(pool, q, out, lse, fill=0xFF, causal=True, window=0, w_in=None, w_out=None, scale=None):
    """The C entry point with a workspace whose every byte is `fill` (0xFF: NaN)."""
    import ctypes
    from paper_2609_38198_b200 import binding as b
    head = lambda t: b.fd_heads(t.data_ptr(), t.stride(0), t.stride(1), t.shape[1])  # noqa: E731
    ptr = lambda t: 0 if t is None else t.data_ptr()  # noqa: E731
    a = b.fd_kv_attend_args(head(q), head(out), pool.dim ** -0.5 if scale is None else scale, int(causal), window, ptr(lse), ptr(w_in), ptr(w_out),
                            0 if w_out is None else w_out.shape[2])
    ref = ctypes.byref(pool.batch.struct)
    size = b.lib.fd_kv_attend_bytes(pool.cache._h, ref, q.shape[1], 0 if w_out is None else 1)
    ws = torch.full((max(size, 16),), fill, dtype=torch.uint8, device=DEV)
    err = ctypes.create_string_buffer(256)
    st = b.lib.fd_kv_attend(pool.cache._h, ref, ctypes.byref(a), ws.data_ptr(), size, torch.cuda.current_stream().cuda_stream, err, 256)
    assert st == 0, err.value
    pool.cache.synchronize()
    return size


@pytest.mark.parametrize("dtype,dim", [(BF16, 128), (FP16, 64)])
@pytest.mark.parametrize("new,group", [(2, 1), (5, 3), (4, 4), (30, 2)])
@pytest.mark.parametrize("mask", ["causal", "window 65", "window 130", "window 600"])
def test_attend_workspace_of_any_content(fd, dtype, dim, new, group, mask):
    """Nothing of the workspace is used that the call has not written: parts of a cache that one of several new tokens does not see, at the end of the cache
    (causal) and at the front of a window."""
    window = int(mask.split()[1]) if mask.startswith("window") else 0
    for n in (65, 66, 67, 68, 705, 709, 4099):
        p = Pool(fd, n + new, [n], [min(new, n)], 2, dim, 16, dtype)
        q = randn(n, p.total, 2 * group, dim, dtype=dtype, scale=2.0)
        want, lse, weights, tol, rel = attend64(p, q, dim ** -0.5, True, window)
        for weigh in (False, True):
            out, got_lse = torch.zeros_like(q), torch.zeros(q.shape[:2], device=DEV)
            w = torch.zeros(1, 2, n, device=DEV) if weigh else None
            attend_raw(p, q, out, got_lse, window=window, w_out=w)
            assert ((out.double() - want).abs() <= tol).all(), (n, weigh)
            assert ((got_lse.double() - lse).abs() <= rel + 2.0 ** -21 * (1 + lse.abs())).all()
            if weigh:
                e = (w[0].double() - weights[0]).abs()
                assert (e <= weights[0] * (rel + 2.0 ** -20 * (1 + 40)) + 2.0 ** -22 * weights[0]).all()


@pytest.mark.parametrize("how", ["bound", "table", "negative"])
def test_append_beyond_the_bounds_writes_nothing(fd, how):
    """A sequence whose length is out of range is not written at all: cut to the bound, its new tokens would land on older ones."""
    p = Pool(fd, 5, [300, 40], [4, 4], 2, 64, 16, BF16)
    batch = p.batch
    if how == "bound":
        batch = fd.KVBatch(p.table, p.kv_len, p.q_start, 8, 4, 299)
    if how == "table":
        p.kv_len[0] = p.cols * 16 + 1
        batch = fd.KVBatch(p.table, p.kv_len, p.q_start, 8, 4, 1000)
    if how == "negative":
        p.kv_len[0] = -1
    before = p.k.clone(), p.v.clone()
    k, v, q = (randn(s, 8, h, 64, dtype=BF16) for s, h in ((1, 2), (2, 2), (3, 4)))
    pos = torch.arange(8, dtype=torch.int32, device=DEV)
    freqs = fd.fd_rotary_frequencies(64, device=DEV)
    qo = p.cache.append(batch, k, v, positions=pos, freqs=freqs, q=q)
    with pytest.raises(fd.FdError) as e:
        p.cache.synchronize()
    assert e.value.status == fd.FD_ERR_INVALID
    assert torch.equal(qo, fd.fd_rotary(q, pos, freqs))
    pg, r = p.where(1, torch.arange(36, 40, device=DEV))
    before[0][pg, r], before[1][pg, r] = fd.fd_rotary(k, pos, freqs)[4:], v[4:]
    for got, want in zip((p.k, p.v), before):
        assert torch.equal(got.view(torch.int16), want.view(torch.int16))


@pytest.mark.parametrize("new", [1, 2, 40])
def test_page_table_of_one_row_for_all(fd, new):
    """Sequences that continue one prompt read the same pages through an expanded table, up to lengths of their own."""
    p = Pool(fd, 5, [700], [new], 2, 64, 16, BF16)
    lengths = [700, 650, 300]
    kv_len = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    start = torch.arange(4, dtype=torch.int32, device=DEV) * new
    q = randn(6, 3 * new, 4, 64, dtype=BF16)
    w, w_ref = torch.zeros(3, 2, 700, device=DEV), torch.zeros(3, 2, 700, device=DEV)
    shared = fd.KVBatch(p.table.expand(3, -1), kv_len, start, 3 * new, new, 700)
    copied = fd.KVBatch(p.table.repeat(3, 1), kv_len, start, 3 * new, new, 700)
    out, lse = p.cache.attend(shared, q, weights=w)
    ref, ref_lse = p.cache.attend(copied, q, weights=w_ref)
    assert torch.equal(out, ref) and torch.equal(lse, ref_lse) and torch.equal(w, w_ref)
    p.cache.synchronize()
    launches = fd.fd_launch_count()
    with pytest.raises(fd.FdError):                          # in place, or to pages in common
        p.cache.evict(shared, w, 10)
    assert fd.fd_launch_count() == launches


@pytest.mark.parametrize("new", [1, 64])
@pytest.mark.parametrize("above", [10, 16, 17, 18])
@pytest.mark.parametrize("spread", [0.0, 0.5])
def test_attend_one_key_above_all(fd, new, above, spread):
    """One key whose score lies far above 32767 others and whose value is 0, in as many caches as keep the GPU busy without cutting one: in fp16 a weight keeps
    its 11 bits down to 2^-24 of the largest, and is off by 2^-35 of it below (fp16's normal range ends at 2^-14, its steps at 2^-24; the largest weight
    is held at 2^10 or more; with few rows at 2^12 or more)."""
    n, dim, heads, batch = 32768, 64, 8, 37
    g = torch.Generator(device=DEV).manual_seed(above)
    k = torch.zeros(n // 64, 64, heads, dim, dtype=FP16, device=DEV)
    v = (1 + torch.rand(n // 64, 64, heads, dim, device=DEV, generator=g)).half()
    if spread:
        k[..., 1] = spread * torch.randn(n // 64, 64, heads, device=DEV, generator=g).half()
    place = 70 if spread else n - 100
    k[place // 64, place % 64] = 0
    k[place // 64, place % 64, :, 0] = above
    v[place // 64, place % 64] = 0
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    cache = fd.KVCache(k, v)
    table = torch.arange(n // 64, dtype=torch.int32, device=DEV)[None].repeat(batch, 1)
    q = torch.zeros(batch * new, heads, dim, dtype=FP16, device=DEV)
    q[:, :, :2] = 8.0
    out, lse = cache.attend(fd.KVBatch(table, i32([n] * batch), i32([new * b for b in range(batch + 1)]), batch * new, new, n), q, causal=False)
    cache.synchronize()
    for h in (0, heads - 1):
        s = q[:1, h].double() @ k[:, :, h].reshape(n, dim).double().T / 8
        p = torch.softmax(s, -1)
        vv = v[:, :, h].reshape(n, dim).double()
        want = p @ vv
        # a rounded weight, the exponential, and 2^-12 for sums of one sign (see test_attend_long_sums_of_one_sign); the rounded result
        tol = (2.0 ** -11 + 2.0 ** -12 + 2.0 ** -19) * want + 2.0 ** (-37 if new == 1 else -35) * p.max() * vv.sum(0) + torch.finfo(FP16).eps / 2 * want + 2.0 ** -25
        err = (out[:, h].double() - want).abs()
        assert (err <= tol).all(), float((err / want).max())
        # the norm: 256 additions (of 32 tokens by each of four warps, or of 128) beside the one large weight, each off by half a step of it or less; the
        # exponentials, the logarithm and the largest score
        sure = 256 * 2.0 ** -24 + 2.0 ** -22 * (8 + above)
        assert (lse[:, h].double() - torch.logsumexp(s, -1)).abs().max() <= sure


def test_attend_more_new_tokens_than_promised_few(fd):
    """As above, with no more rows than the kernel for few rows holds: every row of the sequence is left out, whatever parts the caches are cut into."""
    for n in (60, 5000):
        p = Pool(fd, 5, [300, n], [1, 3], 2, 64, 16, BF16)
        q = randn(6, 4, 4, 64, dtype=BF16)
        good, _ = p.cache.attend(p.batch, q)
        out = torch.full_like(q, 7.0)
        w = torch.rand(2, 2, max(n, 300), device=DEV)
        w0 = w.clone()
        p.cache.attend(fd.KVBatch(p.table, p.kv_len, p.q_start, 4, 1, max(n, 300)), q, out=out, weights=w)
        with pytest.raises(fd.FdError) as e:
            p.cache.synchronize()
        assert e.value.status == fd.FD_ERR_INVALID
        assert ((out[0].double() - good[0].double()).abs() <= 2.0 ** -7 * good[0].double().abs() + 2.0 ** -9).all()
        assert (out[1:] == 7.0).all() and torch.equal(w[1], w0[1])


@pytest.mark.parametrize("new", [1, 3, 40])
def test_rows_before_the_first_sequence(fd, new):
    """A batch may be the tail of a larger one (decoding sequences behind prompts in the same tensors): rows before its first are left as they were."""
    p = Pool(fd, 5, [5000], [new], 1, 64, 16, BF16)
    p.q_start += 4
    batch = fd.KVBatch(p.table, p.kv_len, p.q_start, new + 4, new, 5000)
    q = randn(6, new + 4, 4, 64, dtype=BF16)
    k, v = randn(1, new + 4, 1, 64, dtype=BF16), randn(2, new + 4, 1, 64, dtype=BF16)
    pos = torch.arange(new + 4, dtype=torch.int32, device=DEV)
    freqs = fd.fd_rotary_frequencies(64, device=DEV)
    turned = fd.fd_rotary(q, pos, freqs)
    qo = q.clone()
    p.cache.append(batch, k, v, positions=pos, freqs=freqs, q=qo, q_out=qo)
    p.cache.synchronize()
    assert torch.equal(qo[4:], turned[4:]) and torch.equal(qo[:4], q[:4])
    out, lse = torch.full_like(q, 7.0), torch.full((new + 4, 4), 7.0, device=DEV)
    p.batch = batch
    attend_raw(p, qo, out, lse)
    assert (out[:4] == 7.0).all() and (lse[:4] == 7.0).all()
    ref, ref_lse = p.cache.attend(fd.KVBatch(p.table, p.kv_len, p.q_start - 4, new, new, 5000), qo[4:])
    assert ((out[4:].double() - ref.double()).abs() <= 2.0 ** -7 * ref.double().abs() + 2.0 ** -9).all() and (lse[4:] - ref_lse).abs().max() < 1e-5


@pytest.mark.parametrize("new,group", [(1, 1), (1, 4), (2, 3), (5, 3), (16, 1)])
def test_attend_workspace_holds_the_rows_there_are(fd, new, group):
    """Scores of few rows take 4 bytes a row and token of the bound, for the rows that max_new allows."""
    import ctypes
    p = Pool(fd, 5, [300, 1700], [new, min(new, 2)], 2, 64, 16, FP16)
    q = randn(6, p.total, 2 * group, 64, dtype=FP16)
    ref = ctypes.byref(p.batch.struct)
    with_w, without = (fd.lib.fd_kv_attend_bytes(p.cache._h, ref, 2 * group, w) for w in (1, 0))
    assert with_w - without == 4 * 2 * 2 * new * group * 1728            # (1700 rounded up to a multiple of 64)
    want, _, weights, tol, rel = attend64(p, q, 0.125)
    out, lse, w = torch.zeros_like(q), torch.zeros(q.shape[:2], device=DEV), torch.zeros(2, 2, 1700, device=DEV)
    attend_raw(p, q, out, lse, w_out=w)
    assert ((out.double() - want).abs() <= tol).all()
    for b, n in enumerate(p.kv):
        e = (w[b, :, :n].double() - weights[b]).abs()
        assert (e <= weights[b] * (rel + 2.0 ** -20 * (1 + 40)) + 2.0 ** -22 * weights[b]).all()


def test_tensors_that_need_a_gradient_are_refused(fd):
    """The operators build no graph, so a gradient would be lost in silence."""
    p = Pool(fd, 5, [30], [2], 2, 64, 16, BF16)
    q, k, v = (randn(s, 2, h, 64, dtype=BF16).requires_grad_() for s, h in ((1, 4), (2, 2), (3, 2)))
    w = torch.zeros(1, 2, 30, device=DEV).requires_grad_()
    pos = torch.arange(2, dtype=torch.int32, device=DEV)
    freqs = fd.fd_rotary_frequencies(64, device=DEV)
    for call in (lambda: fd.fd_rotary(q, pos, freqs), lambda: p.cache.attend(p.batch, q), lambda: fd.KVCache(p.k.clone().requires_grad_(), p.v),
                 lambda: p.cache.evict(p.batch, w, 10), lambda: p.cache.append(p.batch, k, v.detach()),
                 lambda: p.cache.append(p.batch, k.detach(), v), lambda: p.cache.append(p.batch, k.detach(), v.detach(), positions=pos, freqs=freqs, q=q)):
        launches = fd.fd_launch_count()
        with pytest.raises(fd.FdError):
            call()
        assert fd.fd_launch_count() == launches
        with torch.no_grad():
            call()
    p.cache.synchronize()


def test_overlapping_rows_are_refused(fd):
    """Results whose rows overlap each other, which would depend on the order of writing."""
    p = Pool(fd, 5, [30, 20], [2, 1], 2, 64, 16, BF16)
    q, k = randn(1, 3, 4, 64, dtype=BF16), randn(2, 3, 2, 64, dtype=BF16)
    pos = torch.arange(3, dtype=torch.int32, device=DEV)
    freqs = fd.fd_rotary_frequencies(64, device=DEV)
    flat = torch.zeros(4096, dtype=BF16, device=DEV)
    for strides in ((64, 64), (192, 64), (64, 128), (72, 64), (128, 64)):
        bad = torch.as_strided(flat, (3, 4, 64), (*strides, 1))
        with pytest.raises(fd.FdError):
            fd.fd_rotary(q, pos, freqs, out=bad)
        with pytest.raises(fd.FdError):
            p.cache.append(p.batch, k, k, positions=pos, freqs=freqs, q=q, q_out=bad)
        with pytest.raises(fd.FdError):
            p.cache.attend(p.batch, q, out=bad)
    assert (flat == 0).all()
    ref, _ = p.cache.attend(p.batch, q)
    for strides in ((256, 64), (64, 192), (264, 64), (72, 216)):         # token by token, head by head, with gaps
        good = torch.as_strided(flat, (3, 4, 64), (*strides, 1))
        assert torch.equal(p.cache.attend(p.batch, q, out=good)[0], ref)
    p.cache.synchronize()


def test_totals_and_lengths_that_overlap_are_refused(fd):
    """weights_out may be weights and new_len may be kv_len; the one may not lie partly over the other."""
    p = Pool(fd, 5, [30, 20], [2, 1], 2, 64, 16, BF16)
    q = randn(1, 3, 4, 64, dtype=BF16)
    totals = torch.zeros(400, device=DEV)
    a, b = totals[:120].view(2, 2, 30), totals[8:128].view(2, 2, 30)
    lengths = torch.tensor([30, 20, 0], dtype=torch.int32, device=DEV)
    for x, y in ((a, b), (b, a)):
        with pytest.raises(fd.FdError):
            p.cache.attend(p.batch, q, weights=x, weights_out=y)
        with pytest.raises(fd.FdError):
            p.cache.evict(p.batch, x, 10, weights_out=y)
    with pytest.raises(fd.FdError):
        p.cache.evict(fd.KVBatch(p.table, lengths[:2], p.q_start, 3, 2, 30), a, 10, new_len=lengths[1:])
    assert (totals == 0).all() and lengths.tolist() == [30, 20, 0]
    p.cache.attend(p.batch, q, weights=a, weights_out=totals[120:240].view(2, 2, 30))
    p.cache.attend(p.batch, q, weights=a, weights_out=a)
    assert torch.equal(totals[:120], totals[120:240]) and float(totals.sum()) > 0
    p.cache.synchronize()


def test_attend_bytes_of_wrong_bounds(fd):
    """0, as for every wrong argument: no workspace is taken for a call that will be refused."""
    import ctypes
    p = Pool(fd, 5, [300], [2], 2, 64, 16, FP16)
    assert fd.lib.fd_kv_attend_bytes(p.cache._h, ctypes.byref(p.batch.struct), 4, 1) > 0
    q, w = randn(6, 2, 4, 64, dtype=FP16), torch.zeros(1, 2, 300, device=DEV)
    for name, value in (("max_len", -1), ("max_len", 2 ** 31 - 1), ("max_new", 3), ("max_new", -1), ("max_new", 0), ("batch", 70000)):
        batch = fd.KVBatch(p.table, p.kv_len, p.q_start, 2, 2, 300)
        setattr(batch.struct, name, value)
        assert fd.lib.fd_kv_attend_bytes(p.cache._h, ctypes.byref(batch.struct), 4, 1) == 0, name
        with pytest.raises(fd.FdError):
            p.cache.attend(batch, q, weights=w)
    batch = fd.KVBatch(p.table, p.kv_len, p.q_start, 2, 2, 300)
    size = fd.lib.fd_kv_attend_bytes(p.cache._h, ctypes.byref(batch.struct), 4, 1)
    batch.struct.table_dev = batch.struct.kv_len_dev = batch.struct.q_start_dev = None           # sizes are asked for before there are any arrays
    assert fd.lib.fd_kv_attend_bytes(p.cache._h, ctypes.byref(batch.struct), 4, 1) == size
    for total_q, max_new, max_len in ((2 ** 32 + 2, 2, 300), (2, 2 ** 32 + 2, 300), (2, 2, 2 ** 32 + 300), (-1, 0, 300)):
        with pytest.raises(fd.FdError):
            fd.KVBatch(p.table, p.kv_len, p.q_start, total_q, max_new, max_len)


def test_attend_smallest_scales(fd):
    """A scale that is no normal fp32 number is refused (0 times the -inf of a hidden score is NaN); the smallest normal ones give means."""
    p = Pool(fd, 5, [300, 300], [1, 40], 1, 64, 16, BF16)
    q = randn(6, 41, 1, 64, dtype=BF16)
    for scale in (1e-300, 1e-46, 1e-39):
        with pytest.raises(fd.FdError):
            p.cache.attend(p.batch, q, scale=scale)
    check_attend(fd, p, q, scale=1e-37)


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("new", [1, 40])
def test_attend_concentrated_rows_are_not_scaled(fd, dtype, new):
    """Two equal weights far above 32766 others: the result is the mean of two neighbouring numbers, a tie that goes to the even one.  Anything that multiplies the
    result by more than 1 makes it the odd one."""
    n, dim = 32768, 64
    k = torch.zeros(n // 64, 64, 1, dim, dtype=dtype, device=DEV)
    v = torch.zeros(n // 64, 64, 1, dim, dtype=dtype, device=DEV)
    k[3, 5, 0, 0] = k[400, 7, 0, 0] = 16.0
    v[3, 5] = 1.0
    v[400, 7] = 1.0 + torch.finfo(dtype).eps
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    cache = fd.KVCache(k, v)
    batch = fd.KVBatch(torch.arange(n // 64, dtype=torch.int32, device=DEV)[None], i32(n), i32(0, new), new, new, n)
    q = torch.zeros(new, 1, dim, dtype=dtype, device=DEV)
    q[..., 0] = 128.0                                        # in powers of two, all exact: scores of 256 and 0
    out, _ = cache.attend(batch, q, scale=math.log(2.0) / 8, causal=False)
    cache.synchronize()
    assert (out == 1.0).all()


@pytest.mark.parametrize("dtype", [FP16, BF16])
def test_attend_long_sums_of_one_sign_few_rows(fd, dtype):
    """As test_attend_long_sums_of_one_sign for one new token: 296 caches of 2^20 tokens (37 sequences read the same pages), so that a warp goes through 262144."""
    n, batch, heads, dim = 1 << 20, 37, 8, 64
    g = torch.Generator(device=DEV).manual_seed(1)
    k = (torch.randn(n // 64, 64, heads, dim, device=DEV, generator=g) * 0.5).to(dtype)
    v = (1 + torch.rand(dim, device=DEV, generator=g) + 0.1 * torch.rand(n // 64, 64, heads, dim, device=DEV, generator=g)).to(dtype)
    table = torch.arange(n // 64, dtype=torch.int32, device=DEV)[None].repeat(batch, 1)
    cache = fd.KVCache(k, v)
    kv_len = torch.full((batch,), n, dtype=torch.int32, device=DEV)
    q = torch.randn(batch, heads, dim, device=DEV, generator=g).to(dtype)
    out, lse = cache.attend(fd.KVBatch(table, kv_len, torch.arange(batch + 1, dtype=torch.int32, device=DEV), batch, 1, n), q)
    cache.synchronize()
    for h in (0, heads - 1):
        s = q[:, h].double() @ k[:, :, h].reshape(n, dim).double().T / 8
        want = torch.softmax(s, -1) @ v[:, :, h].reshape(n, dim).double()
        # (a mean over 37 x 64 results, whose own roundings average out)
        assert abs(float((out[:, h].double() / want - 1).mean())) <= 2.0 ** -12, float((out[:, h].double() / want - 1).mean())
        # 1024 additions of much the same size, each off by half a step of what is there or less; the exponentials, the logarithm and the largest score
        assert (lse[:, h].double() - torch.logsumexp(s, -1)).abs().max() <= 512 * 2.0 ** -24 + 2.0 ** -22 * (8 + 16)


@pytest.mark.parametrize("rising", [True, False])
def test_attend_few_rows_over_long_caches(fd, rising):
    """Caches that fill a warp's accumulators several times (296 of 300032 tokens, the pages shared), with scores that rise or fall along the cache, two new tokens
    and two query heads a cached head."""
    n, batch, heads, dim, new, group = 300032, 37, 8, 128, 2, 2
    g = torch.Generator(device=DEV).manual_seed(2)
    size = torch.linspace(0.1, 2.0, n, device=DEV)
    k = torch.randn(n, heads, dim, device=DEV, generator=g) * (size if rising else size.flip(0))[:, None, None]
    k = k.to(BF16).view(n // 64, 64, heads, dim)
    v = torch.randn(n // 64, 64, heads, dim, device=DEV, generator=g).to(BF16)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    cache = fd.KVCache(k, v)
    table = torch.arange(n // 64, dtype=torch.int32, device=DEV)[None].expand(batch, -1)
    q = torch.randn(batch * new, heads * group, dim, device=DEV, generator=g).to(BF16)
    w = torch.zeros(batch, heads, n, device=DEV)
    out, lse = cache.attend(fd.KVBatch(table, i32([n] * batch), i32([new * b for b in range(batch + 1)]), batch * new, new, n), q, weights=w)
    cache.synchronize()
    for b, h in ((0, 0), (17, 5), (36, 7)):
        x = q[new * b:new * (b + 1), group * h:group * (h + 1)].double()                         # [new, group, dim]
        kk, vv = k[:, :, h].reshape(n, dim).double(), v[:, :, h].reshape(n, dim).double()
        s = torch.einsum("igd,jd->igj", x, kk) * dim ** -0.5
        s[0, :, n - 1] = -math.inf
        p = torch.softmax(s, -1)
        want, size_ = p @ vv, p @ vv.abs()
        top = float(s[s > -math.inf].abs().max())
        sure = 2.0 ** -19 * dim ** -0.5 * float((x.abs() @ kk.abs().T).max()) + 2.0 ** -22 * (8 + top)
        got = out[new * b:new * (b + 1), group * h:group * (h + 1)].double()
        # (2^-12 of the sum of magnitudes for the truncation of 32768 tokens)
        tol = (2.0 ** -8 + 2 * sure + 2.0 ** -12) * size_ + 2.0 ** -8 * want.abs()
        assert ((got - want).abs() <= tol).all(), float(((got - want).abs() / tol).max())
        e = lse[new * b:new * (b + 1), group * h:group * (h + 1)].double() - torch.logsumexp(s, -1)
        assert e.abs().max() <= 2 * sure + 512 * 2.0 ** -24
        total = p.sum((0, 1))
        assert ((w[b, h].double() - total).abs() <= total * (2 * sure + 512 * 2.0 ** -24 + 2.0 ** -20 * (1 + 40)) + 2.0 ** -140).all()


def test_calls_from_several_threads(fd):
    """One cache, its calls from four threads on streams of their own: every result, and every launch counted."""
    import threading
    p = Pool(fd, 5, [300], [1], 2, 64, 16, BF16)
    q = randn(6, 1, 4, 64, dtype=BF16)
    ref, ref_lse = p.cache.attend(p.batch, q)
    pos, freqs = torch.zeros(1, dtype=torch.int32, device=DEV), fd.fd_rotary_frequencies(64, device=DEV)
    before = fd.fd_launch_count()
    p.cache.attend(p.batch, q)
    each = fd.fd_launch_count() - before + 1                # (and one for the rotation)
    torch.cuda.synchronize()
    wrong, calls, threads = [], 500, 4

    def work():
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(calls):
                fd.fd_rotary(q, pos, freqs)
                out, lse = p.cache.attend(p.batch, q)
            if not (torch.equal(out, ref) and torch.equal(lse, ref_lse)):
                wrong.append(1)

    before = fd.fd_launch_count()
    all_ = [threading.Thread(target=work) for _ in range(threads)]
    for t in all_:
        t.start()
    for t in all_:
        t.join()
    torch.cuda.synchronize()
    assert not wrong and fd.fd_launch_count() - before == threads * calls * each
    p.cache.synchronize()


def test_evict_keeps_no_more_than_lengths_reach(fd):
    """keep beyond 2^30, the longest length, is refused: loops over `keep` slots in 32 bits would run over."""
    import ctypes
    from paper_2609_38198_b200 import binding as b
    p = Pool(fd, 5, [30], [0], 2, 64, 16, BF16)
    w = torch.zeros(1, 2, 30, device=DEV)
    for keep in ((1 << 30) + 1, 2 ** 31 - 1):
        x = b.fd_kv_evict_args(w.data_ptr(), w.data_ptr(), 30, p.table.data_ptr(), p.cols, p.cols, keep, 0, 0, w.data_ptr(), p.kv_len.data_ptr())
        launches = fd.fd_launch_count()
        assert b.lib.fd_kv_evict(p.cache._h, ctypes.byref(p.batch.struct), ctypes.byref(x), None, None, 0) == fd.FD_ERR_UNSUPPORTED
        assert fd.fd_launch_count() == launches


def test_misaligned_arrays_are_refused(fd):
    """Arrays that do not lie on a multiple of their element, through the C entry points: refused before anything is launched."""
    import ctypes
    from paper_2609_38198_b200 import binding as b
    p = Pool(fd, 5, [30], [2], 2, 64, 16, BF16)
    w = torch.zeros(1, 2, 30, device=DEV)
    t = torch.zeros(2, 2, 64, dtype=BF16, device=DEV)
    o = torch.zeros(2, 2, 64, dtype=BF16, device=DEV)
    h, ho = b.fd_heads(t.data_ptr(), 128, 64, 2), b.fd_heads(o.data_ptr(), 128, 64, 2)
    pos, freqs = torch.zeros(4, dtype=torch.int32, device=DEV), torch.zeros(40, dtype=torch.float64, device=DEV)
    null = b.fd_heads(None, 0, 0, 0)
    launches = fd.fd_launch_count()

    def refused(entry, args, *more):
        err = ctypes.create_string_buffer(256)
        assert entry(p.cache._h, ctypes.byref(p.batch.struct), ctypes.byref(args), *more, None, err, 256) == fd.FD_ERR_INVALID and b"misaligned" in err.value

    for dp, df in ((2, 0), (0, 4)):
        refused(b.lib.fd_kv_append, b.fd_kv_append_args(h, h, null, null, pos.data_ptr() + dp, freqs.data_ptr() + df, 1.0, 64, 0))
    for dl, di, do in ((2, 0, 0), (0, 1, 0), (0, 0, 2)):
        refused(b.lib.fd_kv_attend, b.fd_kv_attend_args(h, ho, 1.0, 1, 0, w.data_ptr() + dl, w.data_ptr() + di, w.data_ptr() + do, 30), None, 0)
    for i in range(5):
        d = [2 * (j == i) for j in range(5)]
        refused(b.lib.fd_kv_evict, b.fd_kv_evict_args(w.data_ptr() + d[0], w.data_ptr() + d[1], 30, p.table.data_ptr() + d[2], p.cols, p.cols, 10, 0, 0,
                                                      w.data_ptr() + d[3], p.kv_len.data_ptr() + d[4]))
    for name in ("table_dev", "kv_len_dev", "q_start_dev"):
        whole = getattr(p.batch.struct, name)
        setattr(p.batch.struct, name, whole + 2)
        refused(b.lib.fd_kv_append, b.fd_kv_append_args(h, h, null, null, None, None, 1.0, 0, 0))
        setattr(p.batch.struct, name, whole)
    assert fd.fd_launch_count() == launches


@pytest.mark.parametrize("how", ["bound", "table", "negative"])
@pytest.mark.parametrize("over", [False, True])
def test_evict_beyond_the_bounds_loses_nothing(fd, how, over):
    """A sequence whose length is out of range is left alone and reported: cut to the bound, its newest tokens would be gone."""
    p = Pool(fd, 5, [300, 290], [0, 0], 2, 64, 16, BF16)
    w = torch.rand(2, 2, 400, device=DEV)
    bound = 400
    if how == "bound":
        bound = 299
    if how == "table":
        p.kv_len[0] = p.cols * 16 + 1
    if how == "negative":
        p.kv_len[0] = -1
    batch = fd.KVBatch(p.table, p.kv_len, p.q_start, 0, 0, bound)
    wrong = int(p.kv_len[0])
    old = [p.rows(b) for b in range(2)]
    w0 = w.clone()
    kept, new_len, _ = p.cache.evict(batch, w, 100, first=2, recent=30, new_len=p.kv_len if over else None)
    with pytest.raises(fd.FdError) as e:
        p.cache.synchronize()
    assert e.value.status == fd.FD_ERR_INVALID
    assert new_len.tolist() == [wrong, 100] and (kept[0] == -1).all() and torch.equal(w[0], w0[0])
    now = p.rows(0)
    assert torch.equal(now[0], old[0][0]) and torch.equal(now[1], old[0][1])
    for h in range(2):                                       # the other sequence, as ever
        want = torch.from_numpy(evict_plain(w0[1, h, :290].cpu().numpy(), 290, 100, 2, 30)).to(DEV)
        assert torch.equal(kept[1, h].long(), want)
        pg, r = p.where(1, torch.arange(100, device=DEV))
        assert torch.equal(p.k[pg, r, h].double(), old[1][0][want, h]) and torch.equal(w[1, h, :100], w0[1, h, want])


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("new", [1, 40])
def test_attend_scores_of_millions(fd, dtype, new):
    """Scores up to 2^28 (in powers of two), where the steps of fp32 are 16: one key far above the others, whose value the result is, whatever the largest score is
    rounded to.  A weight is then at most 2^16 smaller than its place in the type says (2^10 or more), so it keeps its bits."""
    for size in [300.0, 1000.0, 1500.0, 2000.0, 2500.0, 2900.0, *torch.linspace(3500, 4800, 14).tolist()]:
        p = Pool(fd, int(size), [3000], [new], 1, 64, 16, dtype)
        k, v = p.rows(0)
        k[500], k[2900] = size / 2, size
        p.set_rows(0, 0, k.to(dtype), v.to(dtype))
        q = torch.full((new, 2, 64), size, dtype=dtype, device=DEV)
        out, lse = p.cache.attend(p.batch, q, causal=False)
        p.cache.synchronize()
        want, half = v[2900], torch.finfo(dtype).eps / 2
        assert ((out.double() - want).abs() <= (2 * half + 2.0 ** -19) * want.abs()).all(), size      # the weight and the result, rounded
        top = float(64 * torch.tensor(size, dtype=dtype).double() ** 2 / 8)
        assert (lse.double() - top).abs().max() <= 2.0 ** -21 * top
