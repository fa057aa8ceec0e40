"""Paged keys and values, rotary positions: what the host decides alone -- frequencies, and the refusals of every entry point
before anything is launched."""
import ctypes
import math

import numpy as np
import pytest


@pytest.fixture(scope="module")
def fd():
    import __graft_entry__ as g
    g.build()
    import paper_2609_38198_b200 as fd
    return fd


@pytest.mark.parametrize("rot", [2, 16, 64, 128])
@pytest.mark.parametrize("scaling", ["none", "linear", "base", "ramp"])
def test_rotary_frequencies(fd, rot, scaling):
    if scaling == "base" and rot == 2:
        with pytest.raises(fd.FdError):
            fd.fd_rotary_frequencies(rot, scaling=scaling, factor=4.0)
        return
    got = fd.fd_rotary_frequencies(rot, 10000.0, scaling, factor=4.0, original_len=2048, lo=1.0, hi=32.0).numpy()
    i = np.arange(rot // 2)
    f = 10000.0 ** (-2.0 * i / rot)
    if scaling == "linear":
        f = f / 4
    if scaling == "base":
        f = (10000.0 * 4.0 ** (rot / (rot - 2.0))) ** (-2.0 * i / rot)
    if scaling == "ramp":
        turns = 2048 * f / (2 * math.pi)
        keep = np.clip((turns - 1) / 31, 0, 1)
        f = f / 4 * (1 - keep) + f * keep
        assert got[0] == f[0]                     # the fastest coordinate is not stretched
    # pow is off by an ulp or two, its base by one more times the exponent's size
    assert np.max(np.abs(got / f - 1)) < 1e-14


@pytest.mark.parametrize("kw", [dict(rot_dim=0), dict(rot_dim=3), dict(base=0.0), dict(base=float("nan")), dict(scaling="linear", factor=0.0),
                                dict(scaling="ramp", factor=2.0), dict(scaling="ramp", factor=2.0, original_len=10.0, lo=2.0, hi=2.0), dict(scaling="other")])
def test_rotary_frequencies_refuses(fd, kw):
    with pytest.raises(fd.FdError):
        fd.fd_rotary_frequencies(**{"rot_dim": 8, **kw})


def _desc(fd, **kw):
    from paper_2609_38198_b200 import binding
    base = dict(k_dev=4096, v_dev=8192, k_page_stride=16 * 2 * 64, k_token_stride=128, k_head_stride=64, v_page_stride=16 * 2 * 64,
                v_token_stride=128, v_head_stride=64, num_pages=4, page_size=16, heads=2, head_dim=64, dtype=fd.FD_BF16, status_dev=256)
    return binding.fd_kv_desc(**{**base, **kw})


@pytest.mark.parametrize("kw,status", [
    (dict(k_dev=None), 1), (dict(status_dev=None), 1), (dict(status_dev=258), 1), (dict(dtype=2), 6), (dict(dtype=7), 6), (dict(head_dim=96), 6),
    (dict(page_size=4), 6), (dict(page_size=20), 6), (dict(page_size=0), 6), (dict(num_pages=0), 1), (dict(heads=0), 1), (dict(k_dev=4098), 1),
    (dict(k_token_stride=60), 1), (dict(v_head_stride=68), 1), (dict(v_page_stride=0), 1), (dict(k_head_stride=-64), 1)])
def test_cache_refuses(fd, kw, status):
    h, err = ctypes.c_void_p(), ctypes.create_string_buffer(256)
    assert fd.lib.fd_kv_create(ctypes.byref(h), ctypes.byref(_desc(fd, **kw)), err, 256) == status
    assert not h.value and err.value
    assert fd.lib.fd_kv_create(ctypes.byref(h), ctypes.byref(_desc(fd, **kw)), None, 0) == status       # a message is optional
    assert fd.fd_launch_count() == 0


def test_null_handles(fd):
    from paper_2609_38198_b200 import binding
    b = binding.fd_kv_batch()
    assert fd.lib.fd_kv_create(None, None, None, 0) == fd.FD_ERR_INVALID
    assert fd.lib.fd_kv_append(None, ctypes.byref(b), None, None, None, 0) == fd.FD_ERR_INVALID
    assert fd.lib.fd_kv_attend(None, ctypes.byref(b), None, None, 0, None, None, 0) == fd.FD_ERR_INVALID
    assert fd.lib.fd_kv_evict(None, ctypes.byref(b), None, None, None, 0) == fd.FD_ERR_INVALID
    assert fd.lib.fd_kv_attend_bytes(None, ctypes.byref(b), 8, 0) == 0
    assert fd.lib.fd_kv_synchronize(None, None) == fd.FD_ERR_INVALID
    fd.lib.fd_kv_destroy(None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=3), 1), (dict(tokens=-1), 1), (dict(rot=0), 1), (dict(rot=66), 1), (dict(rot=31), 1), (dict(layout=2), 1), (dict(head_dim=63), 6),
    (dict(head_dim=2048), 6), (dict(scale=float("inf")), 1), (dict(scale=float("nan")), 1), (dict(positions=None), 1), (dict(freqs=None), 1),
    (dict(out=4096 + 64), 1), (dict(x=4097), 1), (dict(out_heads=3), 1), (dict(head_stride=32), 1), (dict(token_stride=-128), 1)])
def test_rotary_refuses(fd, kw, status):
    from paper_2609_38198_b200 import binding
    a = dict(x=4096, out=1 << 20, dtype=0, tokens=5, head_dim=64, rot=64, layout=0, scale=1.0, positions=256, freqs=512, heads=2, out_heads=2,
             head_stride=64, token_stride=128)
    a.update(kw)
    x = binding.fd_heads(a["x"], a["token_stride"], a["head_stride"], a["heads"])
    y = binding.fd_heads(a["out"], 128, 64, a["out_heads"])
    err = ctypes.create_string_buffer(256)
    st = fd.lib.fd_rotary(ctypes.byref(x), ctypes.byref(y), a["dtype"], a["tokens"], a["head_dim"], a["positions"], a["freqs"], a["rot"], a["layout"],
                          a["scale"], 0, None, err, 256)
    assert st == status and err.value
    assert fd.fd_launch_count() == 0


def test_packed_arguments(fd):
    """The formats that the binding packs in one step are the structures of the header, field by field."""
    from paper_2609_38198_b200 import binding as b
    values = iter(range(1, 100))
    for fmt, st in ((b._HEADS, b.fd_heads), (b._APPEND, b.fd_kv_append_args), (b._ATTEND, b.fd_kv_attend_args), (b._EVICT, b.fd_kv_evict_args)):
        assert fmt.size == ctypes.sizeof(st)

        def fields(t):
            return [x for n, f in t._fields_ for x in (fields(f) if issubclass(f, ctypes.Structure) else [n])]

        def read(o):
            return [x for n, f in o._fields_ for x in (read(getattr(o, n)) if issubclass(f, ctypes.Structure) else [getattr(o, n)])]

        want = [next(values) for _ in fields(st)]
        assert read(st.from_buffer_copy(fmt.pack(*want))) == want


def test_page_table_strides(fd):
    """Rows of a page table in any distance; an expanded one (every sequence reads the same pages) has stride 0, and its next row is not behind the first."""
    import torch
    from paper_2609_38198_b200 import binding as b
    t = torch.arange(24, dtype=torch.int32).view(4, 6)
    for x in (t, t[:, :3], t[::2], t[:1].expand(5, 6), t[:1, :2].expand(3, 2), t[:, 1:2], t.t()[:, :1], torch.as_strided(t, (4, 6), (2, 1)), t[:1], t[:, :0]):
        stride, cols = b._table(x, "table")
        assert cols == x.shape[1]
        for r in range(x.shape[0]):
            for c in range(cols):
                assert x.storage_offset() + r * stride + c < t.numel() and int(x[r, c]) == x.storage_offset() + r * stride + c
    for x in (t.t(), t[:, ::2]):
        with pytest.raises(fd.FdError):
            b._table(x, "table")


@pytest.mark.parametrize("tokens,heads", [(1, 3), (2, 1), (2, 2), (3, 4), (7, 3)])
def test_results_whose_rows_overlap_are_refused(fd, tokens, heads):
    """Against every pair of rows.  Every call is refused before anything is launched: x lies over the first row of the result."""
    from paper_2609_38198_b200 import binding
    dim = 8
    x = binding.fd_heads((1 << 16) + 4, heads * dim, dim, heads)
    for ts in (8, 9, 16, 20, 24, 28, 32, 40, 64):
        for hs in (8, 10, 12, 16, 20, 24, 56, 60):
            at = sorted(t * ts + h * hs for t in range(tokens) for h in range(heads))
            apart = all(b - a >= dim for a, b in zip(at, at[1:]))
            err = ctypes.create_string_buffer(256)
            st = fd.lib.fd_rotary(ctypes.byref(x), ctypes.byref(binding.fd_heads(1 << 16, ts, hs, heads)), fd.FD_FP32, tokens, dim, 256, 512, 8, 0, 1.0, 0,
                                  None, err, 256)
            assert st == fd.FD_ERR_INVALID and err.value == (b"out overlaps x without being x" if apart else b"out: rows overlap"), (ts, hs)
    assert fd.fd_launch_count() == 0


@pytest.mark.parametrize("kw", [dict(positions=258), dict(freqs=516)])
def test_rotary_refuses_misaligned_arrays(fd, kw):
    test_rotary_refuses(fd, kw, fd.FD_ERR_INVALID)
