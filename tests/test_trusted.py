"""The trusted half (4-bit products, the 4-bit cache and its pages): refusals on the CPU, numerics against 64 bits on the GPU."""
import ctypes
import itertools

import numpy as np
import pytest

from paper_2606_17421_b200 import bifrost as bf
from tests import trusted_ref as ref

gpu = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ refusals, without a device

@pytest.fixture
def stand_in():
    """A context that no call gets to use: arguments are looked at first, then the device, which there need not be."""
    from paper_2606_17421_b200 import build
    build.build()
    return ctypes.create_string_buffer(4096)


def matrix(**kw):
    d = dict(codes=4096, scales=4096, offsets=None, row_bytes=48, group_stride=8, d_out=10, d_in=90, group=32)
    return bf.bf_q4_matrix(**{**d, **kw})


def rows(**kw):
    return bf.bf_rows(**{**dict(data=4096, row_stride=128, head_stride=64, type=bf.BF_BF16), **kw})


def cache(**kw):
    d = dict(pool=4096, tables=4096, lengths=4096, refs=4096, n_layers=2, n_pages=8, n_kv_heads=2, head_dim=64, group=32, page_tokens=32,
             n_seqs=3, max_pages=4)
    return bf.bf_kv4_cache(**{**d, **kw})


def refused(code, call, *args):
    with pytest.raises(bf.BifrostError) as ei:
        call(*args)
    assert ei.value.code == code, ei.value


BAD_MATRIX = [(dict(codes=None), -1), (dict(codes=4104), -1), (dict(scales=None), -1), (dict(scales=4100), -1), (dict(offsets=4098), -1), (dict(d_out=0), -1),
              (dict(d_in=0), -1), (dict(group=16), -3), (dict(group=0), -3), (dict(group=48), -3), (dict(row_bytes=40), -3), (dict(row_bytes=32), -3),
              (dict(group_stride=4), -3), (dict(d_in=500, row_bytes=256), -3), (dict(d_out=2 ** 31), -3), (dict(d_in=2 ** 32 - 1, row_bytes=2 ** 31, group_stride=2 ** 27), -3)]


@pytest.mark.parametrize("change,code", BAD_MATRIX, ids=str)
def test_linear_refuses_matrices(stand_in, change, code):
    refused(code, bf.bf_q4_linear, stand_in, matrix(**change), rows(), 1, rows())


def test_linear_refuses_rows_and_counts(stand_in):
    for bad in (dict(data=None), dict(type=3), dict(type=-1), dict(data=4097), dict(data=4098, type=bf.BF_F32)):
        refused(bf.BF_ERR_INVALID_ARG, bf.bf_q4_linear, stand_in, matrix(), rows(**bad), 1, rows())
        refused(bf.BF_ERR_INVALID_ARG, bf.bf_q4_linear, stand_in, matrix(), rows(), 1, rows(**bad))
    refused(bf.BF_ERR_INVALID_ARG, bf.bf_q4_linear, stand_in, matrix(), rows(), 0, rows())
    refused(bf.BF_ERR_INVALID_ARG, bf.bf_q4_linear, None, matrix(), rows(), 1, rows())
    refused(bf.BF_ERR_INVALID_ARG, bf.bf_q4_linear, stand_in, None, rows(), 1, rows())
    refused(bf.BF_ERR_INVALID_ARG, bf.bf_q4_linear, stand_in, matrix(), None, 1, rows())
    refused(bf.BF_ERR_SHAPE, bf.bf_q4_linear, stand_in, matrix(), rows(), 2 ** 31, rows())


BAD_CACHE = [(dict(pool=None), -1), (dict(pool=4104), -1), (dict(tables=None), -1), (dict(tables=4098), -1), (dict(lengths=None), -1), (dict(refs=None), -1),
             (dict(n_layers=0), -1), (dict(n_pages=0), -1), (dict(n_kv_heads=0), -1), (dict(n_seqs=0), -1), (dict(max_pages=0), -1), (dict(head_dim=96), -3),
             (dict(head_dim=256), -3), (dict(group=16), -3), (dict(group=128), -3), (dict(page_tokens=24), -3), (dict(page_tokens=0), -3), (dict(page_tokens=512), -3),
             (dict(max_pages=2 ** 27), -3), (dict(n_pages=2 ** 31), -3), (dict(n_kv_heads=5000), -3), (dict(n_layers=2 ** 17), -3), (dict(n_pages=2 ** 30, n_kv_heads=1000), -3)]


@pytest.mark.parametrize("change,code", BAD_CACHE, ids=str)
def test_every_call_refuses_bad_caches(stand_in, change, code):
    c, r = cache(**change), rows()
    refused(code, bf.bf_kv4_grow, stand_in, c, None, None, 1)
    refused(code, bf.bf_kv4_append, stand_in, c, 0, None, None, 1, 1, r, r)
    refused(code, bf.bf_kv4_read, stand_in, c, 0, None, None, None, 1, 1, r, r)
    refused(code, bf.bf_kv4_attention, stand_in, c, 0, None, None, 1, 1, 1, r, 2, r, 1.0, 0, None)
    refused(code, bf.bf_kv4_fork, stand_in, c, 4096, 8192, 1)
    refused(code, bf.bf_kv4_free, stand_in, c, 4096, 1)
    refused(code, bf.bf_kv4_compact, stand_in, c, None, None, None)


def test_cache_calls_refuse_arguments(stand_in):
    c, r = cache(), rows()
    inv, shape, large = bf.BF_ERR_INVALID_ARG, bf.BF_ERR_SHAPE, bf.BF_ERR_TOO_LARGE
    att = lambda *a: bf.bf_kv4_attention(stand_in, *a)          # noqa: E731
    for n, most in ((0, 1), (1, 0)):
        refused(inv, bf.bf_kv4_append, stand_in, c, 0, None, None, n, most, r, r)
        refused(inv, bf.bf_kv4_read, stand_in, c, 0, None, None, None, n, most, r, r)
        refused(inv, att, c, 0, None, None, n, most, 1, r, 2, r, 1.0, 0, None)
    refused(shape, bf.bf_kv4_append, stand_in, c, 2, None, None, 1, 1, r, r)                    # no such layer
    refused(shape, bf.bf_kv4_append, stand_in, c, 0, None, None, 4, 1, r, r)                    # more than there are, unnamed
    refused(shape, bf.bf_kv4_grow, stand_in, c, None, None, 4)
    refused(inv, bf.bf_kv4_grow, stand_in, c, None, None, 0)
    refused(large, bf.bf_kv4_append, stand_in, c, 0, 4096, 4096, 2 ** 20, 2 ** 20, r, r)
    refused(inv, bf.bf_kv4_append, stand_in, c, 0, None, None, 1, 1, rows(type=5), r)
    refused(inv, att, c, 0, None, None, 1, 1, 1, rows(type=bf.BF_F32), 2, rows(type=bf.BF_F32), 1.0, 0, None)
    refused(inv, att, c, 0, None, None, 1, 1, 1, rows(type=bf.BF_F16), 2, r, 1.0, 0, None)      # out has another type
    refused(inv, att, c, 0, None, None, 1, 1, 0, r, 2, r, 1.0, 0, None)
    refused(inv, att, c, 0, None, None, 1, 1, 1, r, 2, r, float("nan"), 0, None)
    refused(inv, att, c, 0, None, None, 1, 1, 1, r, 2, r, float("inf"), 0, None)
    refused(shape, att, c, 0, None, None, 1, 1, 1, r, 3, r, 1.0, 0, None)
    refused(shape, att, c, 0, None, None, 1, 1, 1, r, 0, r, 1.0, 0, None)
    refused(inv, bf.bf_kv4_fork, stand_in, c, None, 4096, 1)
    refused(inv, bf.bf_kv4_fork, stand_in, c, 4096, 4096, 0)
    refused(inv, bf.bf_kv4_free, stand_in, c, None, 1)
    refused(inv, bf.bf_kv4_free, stand_in, c, 4096, 0)
    refused(large, bf.bf_kv4_fork, stand_in, c, 4096, 4096, 70000)
    # (the stand-in has no workspace)
    refused(large, bf.bf_kv4_compact, stand_in, c, None, None, None)
    refused(large, bf.bf_kv4_grow, stand_in, c, None, None, 1)
    assert bf.load().bf_trusted_create(None, 0, None) == inv
    out = ctypes.c_void_p()
    assert bf.load().bf_trusted_create(ctypes.byref(out), 1000, None) == inv and not out.value
    refused(inv, bf.bf_trusted_status, None)
    bf.bf_trusted_destroy(None)


def test_block_bytes():
    assert bf.bf_kv4_block_bytes(128, 64, 64) == 4 * (128 * 16 + 2 * 128)
    assert bf.bf_kv4_block_bytes(64, 64, 16) == 64 * 16 + 128
    for D, G, T in ((128, 32, 8), (64, 128, 16), (80, 16, 16), (128, 0, 16), (128, 32, 272)):
        assert bf.bf_kv4_block_bytes(D, G, T) == 0


def test_descriptors_refuse_tensors():
    torch = pytest.importorskip("torch")
    x = torch.zeros(4, 3, 64)
    assert bf.bf_rows.of(x[:, :2]).row_stride == 192 and bf.bf_rows.of(x[0]).head_stride == 0
    for bad in (x.int(), x.transpose(1, 2), x[0, 0]):
        with pytest.raises(ValueError):
            bf.bf_rows.of(bad)
    codes, scales = torch.zeros(4, 16, dtype=torch.uint8), torch.zeros(4, 8, dtype=torch.float16)
    assert bf.bf_q4_matrix.of(codes, scales, None, 32, 32).row_bytes == 16
    for c, s, o in ((codes.int(), scales, None), (codes, scales.float(), None), (codes[:3], scales, None), (codes, scales, scales[:, :4]), (codes.t(), scales, None)):
        with pytest.raises(ValueError):
            bf.bf_q4_matrix.of(c, s, o, 32, 32)
    with pytest.raises(bf.BifrostError):
        bf.bf_kv4_cache.of(torch.zeros(1, 2, 2, 100, dtype=torch.uint8), torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32),
                           torch.zeros(2, dtype=torch.int32), 64, 32, 16)


def test_reference_layout_fills_every_nibble_once():
    for D, G in ((64, 32), (64, 64), (128, 32), (128, 64), (128, 128)):
        kn, kp, vn, vp = ref.places(D, G)
        nib = np.concatenate([kn.ravel(), vn.ravel()])
        half = np.concatenate([kp.ravel(), kp.ravel() + 1, vp.ravel(), vp.ravel() + 4])
        used = np.concatenate([nib, *(4 * half + i for i in range(4))])
        assert len(used) == len(set(used.tolist())) == 2 * (16 * D + 128 * (D // G)) and used.max() == len(used) - 1


# ------------------------------------------------------------------------------------------------ on the device

class Side:
    """A context on a stream of its own, and torch's type names."""

    def __init__(self):
        import torch
        self.torch = torch
        torch.cuda.set_device(0)
        self.stream = torch.cuda.Stream()
        torch.cuda.set_stream(self.stream)
        self.t = bf.bf_trusted_create(0, self.stream.cuda_stream)
        self.types = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}

    def dev(self, a):
        return self.torch.from_numpy(np.ascontiguousarray(a)).cuda()

    def ints(self, a):
        return None if a is None else self.dev(np.asarray(a, np.int32))

    def host(self, x):
        self.torch.cuda.synchronize()
        return x.double().cpu().numpy() if x.is_floating_point() else x.cpu().numpy()


@pytest.fixture(scope="module")
def one_side():
    s = Side()
    yield s
    bf.bf_trusted_destroy(s.t)


@pytest.fixture
def side(one_side):
    one_side.torch.cuda.set_stream(one_side.stream)          # (a runner that a test made has set its own)
    return one_side


HALF_STEP = {"fp32": 2.0 ** -24, "fp16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"fp32": 2.0 ** -149, "fp16": 2.0 ** -25, "bf16": 2.0 ** -134}


def draw_matrix(rng, d_out, d_in, group, offsets):
    groups, bytes_ = -(-d_in // group), -(-d_in // 32) * 16
    packed = rng.integers(0, 256, (d_out, bytes_), dtype=np.uint8)                   # codes behind d_in are anything too
    scales = rng.uniform(0.001, 0.01, (d_out, -(-groups // 8) * 8)).astype(np.float16)
    offs = (rng.standard_normal(scales.shape) * 0.02).astype(np.float16) if offsets else None
    for a in (scales, offs):
        if a is not None:
            a[:, groups:] = np.nan                                                   # behind the last group: not used
    code = np.stack([packed & 15, packed >> 4], -1).reshape(d_out, -1)[:, :d_in].astype(np.float64)
    g = np.arange(d_in) // group
    W = scales[:, g].astype(np.float64) * (code - 8) + (offs[:, g].astype(np.float64) if offsets else 0)
    # what a sum in 32 bits meets on its way: codes up to 15, taken back by eight times the sum of x
    top = scales[:, g].astype(np.float64) * 23 + (np.abs(offs[:, g].astype(np.float64)) if offsets else 0)
    return packed, scales, offs, W, top


def linear_tolerance(x, y, top, ytype):
    """Half a step of y's type; 2^-22 of the largest magnitude met for each of the d_in/16 additions of 16 products and a few
    more a group; x taken to 2^-22 of itself or 2^-24 of the largest of its row."""
    K = x.shape[1]
    mag = np.abs(x) @ top.T
    big = np.abs(x).max(1, keepdims=True) * top.sum(1)[None]
    return HALF_STEP[ytype] * np.abs(y) + 2.0 ** -22 * (K / 16 + K / 32 + 24) * mag + 2.0 ** -24 * big + TINY[ytype]


LINEAR = [(1, 64, 16, 32), (1, 64, 17, 64), (1, 1, 1, 32), (1, 33, 5, 128), (2, 200, 129, 64), (3, 768, 300, 128), (7, 1000, 77, 32), (8, 1024, 64, 128), (9, 96, 2500, 32),
          (16, 2048, 130, 64), (17, 511, 33, 128), (31, 640, 50, 32), (33, 1500, 100, 64), (64, 256, 1000, 128), (65, 320, 47, 64), (130, 160, 40, 32), (1, 14336, 40, 128),
          (5, 9000, 20, 64), (40, 5000, 24, 128),
          # rows enough for blocks of 128: odd last tiles, one stage and several, columns behind the last
          (9, 256, 18944, 128), (16, 300, 19001, 64), (13, 600, 19072, 32), (32, 1100, 18945, 128), (25, 64, 20000, 32), (20, 513, 19000, 64), (64, 700, 2500, 128),
          (41, 1500, 2305, 64), (100, 257, 2400, 128), (60, 320, 19000, 32)]


@gpu
@pytest.mark.parametrize("n,d_in,d_out,group", LINEAR)
def test_linear_against_64_bits(side, n, d_in, d_out, group):
    torch = side.torch
    for i, (xt, yt, offsets) in enumerate(itertools.product(("bf16", "fp16", "fp32"), ("bf16", "fp16", "fp32"), (False, True))):
        rng = np.random.default_rng([n, d_in, d_out, i])
        packed, scales, offs, W, top = draw_matrix(rng, d_out, d_in, group, offsets)
        x = torch.from_numpy(rng.standard_normal((n, d_in)) * rng.choice([1, 1, 1, 8], d_in)).to(side.types[xt]).cuda()
        y = torch.full((n + 1, d_out), 5.0, dtype=side.types[yt], device="cuda")
        codes, sc, of = side.dev(packed), side.dev(scales), None if offs is None else side.dev(offs)
        M = bf.bf_q4_matrix.of(codes, sc, of, d_in, group)
        bf.bf_q4_linear(side.t, M, bf.bf_rows.of(x), n, bf.bf_rows.of(y))
        got, xd = side.host(y), side.host(x)
        want = xd @ W.T
        off = np.abs(got[:n] - want) - linear_tolerance(xd, want, top, yt)
        assert (off <= 0).all(), (xt, yt, offsets, off.max())
        assert (got[n:] == 5).all()
    bf.bf_trusted_status(side.t)


@gpu
@pytest.mark.parametrize("n", [1, 5, 20])
def test_linear_strided_and_unaligned_rows(side, n):
    torch, rng = side.torch, np.random.default_rng(n)
    for xt, yt in (("bf16", "fp32"), ("fp32", "fp16"), ("fp16", "bf16")):
        packed, scales, _, W, top = draw_matrix(rng, 70, 333, 64, False)
        codes, sc = side.dev(packed), side.dev(scales)
        big = torch.randn((n, 3, 401), device="cuda").to(side.types[xt])
        x = big[:, 1, 7:340]                                                        # odd stride, odd start
        out = torch.full((n, 201), 5.0, device="cuda").to(side.types[yt])
        y = out[:, 3:73]
        bf.bf_q4_linear(side.t, bf.bf_q4_matrix.of(codes, sc, None, 333, 64), bf.bf_rows.of(x), n, bf.bf_rows.of(y))
        xd, got = side.host(x), side.host(y)
        want = xd @ W.T
        assert (np.abs(got - want) <= linear_tolerance(xd, want, top, yt)).all()
        assert (side.host(out[:, :3]) == 5).all() and (side.host(out[:, 73:]) == 5).all()


@gpu
def test_linear_extreme_values(side):
    """Rows of zeros, of tiny and of huge values beside ordinary ones; a NaN or an infinity stays in its row."""
    torch, rng = side.torch, np.random.default_rng(3)
    packed, scales, offs, W, top = draw_matrix(rng, 48, 300, 32, True)
    codes, sc, of = side.dev(packed), side.dev(scales), side.dev(offs)
    M = bf.bf_q4_matrix.of(codes, sc, of, 300, 32)
    x = torch.randn((6, 300), device="cuda")
    x[0] = 0
    x[1] *= 1e-30
    x[2] *= 1e30
    x[3, ::7] *= 1e5
    for xt in ("fp32", "bf16"):
        xx = x.to(side.types[xt])
        xx[4, 100] = float("nan")
        xx[5, 299] = float("inf")
        y = torch.empty((6, 48), device="cuda")
        bf.bf_q4_linear(side.t, M, bf.bf_rows.of(xx), 6, bf.bf_rows.of(y))
        xd, got = side.host(xx[:4]), side.host(y)
        want = xd @ W.T
        assert (np.abs(got[:4] - want) <= linear_tolerance(xd, want, top, "fp32")).all()
        assert (got[0] == 0).all() and not np.isfinite(got[4]).any() and not np.isfinite(got[5]).any()
    h = torch.full((2, 300), 2.0 ** -24, device="cuda").half()                      # the smallest of the type
    h[1] = 65504.0
    y = torch.empty((2, 48), device="cuda")
    bf.bf_q4_linear(side.t, M, bf.bf_rows.of(h), 2, bf.bf_rows.of(y))
    xd, got = side.host(h), side.host(y)
    want = xd @ W.T
    assert (np.abs(got - want) <= linear_tolerance(xd, want, top, "fp32")).all()


# ---- the cache

class DeviceCache:
    def __init__(self, side, c):
        self.side, self.c = side, c
        self.pool = side.dev(c.pool.reshape(c.layers, c.pages, c.heads, -1))
        self.tables, self.lengths, self.refs = side.dev(c.tables), side.dev(c.lengths), side.dev(c.refs)
        self.desc = bf.bf_kv4_cache.of(self.pool, self.tables, self.lengths, self.refs, c.D, c.G, c.T)

    def same(self, pool=True):
        h, c = self.side.host, self.c
        assert np.array_equal(h(self.lengths), c.lengths)
        assert np.array_equal(h(self.refs), c.refs)
        assert np.array_equal(h(self.tables), c.tables)
        if pool:
            assert np.array_equal(h(self.pool).reshape(c.pool.shape), c.pool)


def status_of(side):
    try:
        bf.bf_trusted_status(side.t)
    except bf.BifrostError as e:
        return e.code
    return 0


def fill(side, c, lens, seed=0, type="fp32"):
    """A host cache with sequences of these lengths in all layers, its device twin, and nothing else in common with the kernels."""
    rng = np.random.default_rng(seed)
    order = rng.permutation(c.pages)
    at = 0
    for i, n in enumerate(lens):
        need = -(-n // c.T)
        c.tables[i, :need] = order[at:at + need]
        c.refs[order[at:at + need]] = 1
        at += need
        c.lengths[i] = n
        for layer in range(c.layers):
            for t in range(n):
                c.put(layer, i, t, rng.standard_normal((c.heads, c.D)) * 1.5, rng.standard_normal((c.heads, c.D)))
    return DeviceCache(side, c)


@gpu
@pytest.mark.parametrize("D,G", [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)])
@pytest.mark.parametrize("type", ["bf16", "fp16", "fp32"])
def test_append_bytes_and_read(side, D, G, type):
    """Chunks of every raggedness, then single tokens: every byte of the pool is what the definition says, borders of codes
    included; then read back, whole and in part."""
    torch, T = side.torch, 32
    c = ref.Cache(2, 14, 3, D, G, T, 4, 4, seed=D + G)
    d = DeviceCache(side, c)
    rng = np.random.default_rng(7)
    for step, (seqs, counts) in enumerate([([2, 0, 3], [1, 40, 17]), ([0, 2, 3], [5, 15, 1]), ([1, 0, 2, 3], [64, 19, 16, 30]), ([3, 2], [1, 1])]):
        bf.bf_kv4_grow(side.t, d.desc, side.ints(seqs), cs := side.ints(counts), len(seqs))
        assert not c.grow(seqs, counts)
        starts = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        for layer in range(2):
            qkv = rng.standard_normal((int(starts[-1]) + 2, 7, D)) * rng.choice([0.01, 1, 30], (1, 7, 1))
            qkv[0, :, :G] = np.arange(G) % 31 / 2                                    # many quotients exactly on a border
            qkv[-3, :, -G:] = 3.25                                                   # a group of one value
            qkv = torch.from_numpy(qkv).to(side.types[type]).cuda()
            k, v = qkv[:, 1:4], qkv[:, 4:]
            single = step == 3
            bf.bf_kv4_append(side.t, d.desc, layer, sq := side.ints(seqs), None if single else (st := side.ints(starts)), len(seqs), max(counts), bf.bf_rows.of(k), bf.bf_rows.of(v))
            kh, vh = side.host(k), side.host(v)
            for i, a in enumerate(seqs):
                for j in range(counts[i]):
                    c.put(layer, a, int(c.lengths[a]) - counts[i] + j, kh[starts[i] + j], vh[starts[i] + j])
            d.same()
    assert status_of(side) == 0
    for layer, first, counts in ((0, None, [3, 64, 1, 0]), (1, [60, 0, 31, 16], [4, 33, 2, 17])):
        starts = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        k = torch.full((int(starts[-1]) + 1, 3, D), 9.0, device="cuda").to(side.types[type])
        v = torch.full_like(k, 9.0)
        st, fi = side.ints(starts), side.ints(first)
        bf.bf_kv4_read(side.t, d.desc, layer, None, st, fi, 4, 64, bf.bf_rows.of(k), bf.bf_rows.of(v))
        for x, held in zip((k, v), (0, 1)):
            x = side.host(x)
            assert (x[starts[-1]:] == 9).all()
            for i in range(4):
                n = int(c.lengths[i])
                f = first[i] if first else n - counts[i]
                want = c.get(layer, i, n)[held][f:f + counts[i]]
                assert (np.abs(x[starts[i]:starts[i + 1]] - want) <= HALF_STEP[type] * np.abs(want) + 2.0 ** -24 * np.abs(want) + TINY[type]).all()
    assert status_of(side) == 0


@gpu
def test_append_special_values(side):
    torch = side.torch
    c = ref.Cache(1, 4, 2, 64, 32, 16, 2, 2)
    d = DeviceCache(side, c)
    c.grow([0], [6])
    bf.bf_kv4_grow(side.t, d.desc, side.ints([0]), n := side.ints([6]), 1)
    x = np.random.default_rng(0).standard_normal((6, 2, 64)).astype(np.float32)
    x[0, 0, 3] = np.nan
    x[1, 0, :3] = [np.inf, -np.inf, 70000.0]
    x[2] = 0
    x[3] = 1e-9                                          # a scale that fp16 does not hold
    x[3, :, 5] = -1e-9
    x[4, 1] = 61440.0 * (-1.0) ** np.arange(64)
    x[5] = 2.0 ** -14 * np.arange(64)
    xs = side.dev(x)
    st = side.ints([0, 6])
    bf.bf_kv4_append(side.t, d.desc, 0, None, st, 1, 6, bf.bf_rows.of(xs), bf.bf_rows.of(xs))
    for t in range(6):
        c.put(0, 0, t, x[t].astype(np.float64), x[t].astype(np.float64))
    got = side.host(d.pool).reshape(c.pool.shape)
    # (which NaN a group has is not part of the definition)
    gh, ch = (np.where(np.isnan(p.view(np.float16)), np.float16(np.nan), p.view(np.float16)).view(np.uint16) for p in (got.copy(), c.pool.copy()))
    assert np.array_equal(gh, ch)
    out = torch.zeros((6, 2, 64), device="cuda")
    bf.bf_kv4_read(side.t, d.desc, 0, None, st, None, 1, 6, bf.bf_rows.of(out), bf.bf_rows.of(torch.empty_like(out)))
    o = side.host(out)
    assert np.isnan(o[0, 0, :32]).all() and np.isfinite(o[0, 0, 32:]).all() and np.isfinite(o[1:]).all() and (o[2] == 0).all()
    assert status_of(side) == 0


@gpu
def test_append_and_read_leave_bad_calls_alone(side):
    torch = side.torch
    c = ref.Cache(1, 6, 1, 64, 64, 16, 3, 2)
    c.grow([0, 1, 2], [20, 16, 1])
    x = torch.randn((64, 1, 64), device="cuda")
    for seqs, starts, code in (([0, 5], [0, 1, 2], bf.BF_ERR_RANGE), ([-1], [0, 1], bf.BF_ERR_RANGE), ([0], [0, 9], bf.BF_ERR_RANGE), ([2], [0, 2], bf.BF_ERR_RANGE),
                               ([0], [3, 1], bf.BF_ERR_RANGE), ([0], [-2, 0], bf.BF_ERR_RANGE), ([1], [2, 2], 0)):
        d = DeviceCache(side, c)
        sq, st = side.ints(seqs), side.ints(starts)
        only = [a for a, n in zip(seqs, np.diff(starts)) if 0 <= a < 3 and 0 < n <= 8 and n <= c.lengths[a]] if starts[0] >= 0 else []
        before = side.host(d.pool).copy()
        bf.bf_kv4_append(side.t, d.desc, 0, sq, st, len(seqs), 8, bf.bf_rows.of(x), bf.bf_rows.of(x))
        assert status_of(side) == code
        if not only:
            assert np.array_equal(before, side.host(d.pool))
        y = torch.full_like(x, 4.0)
        bf.bf_kv4_read(side.t, d.desc, 0, sq, st, None, len(seqs), 8, bf.bf_rows.of(y), bf.bf_rows.of(torch.empty_like(y)))
        assert status_of(side) == code
        if not only:
            assert (side.host(y) == 4).all()
    # a sequence named twice is written once, as its first entry says; a page out of range and a length out of range are not followed
    d = DeviceCache(side, c)
    sq, st = side.ints([0, 0]), side.ints([0, 2, 4])
    bf.bf_kv4_append(side.t, d.desc, 0, sq, st, 2, 2, bf.bf_rows.of(x), bf.bf_rows.of(x))
    assert status_of(side) == bf.BF_ERR_RANGE
    e = DeviceCache(side, c)
    st1 = side.ints([0, 2])
    bf.bf_kv4_append(side.t, e.desc, 0, None, st1, 1, 2, bf.bf_rows.of(x), bf.bf_rows.of(x))
    assert np.array_equal(side.host(d.pool), side.host(e.pool)) and status_of(side) == 0
    for page in (-1, 6, 2 ** 31 - 1):
        d = DeviceCache(side, c)
        d.tables[0, 1] = page
        before = side.host(d.pool).copy()
        bf.bf_kv4_append(side.t, d.desc, 0, None, st1, 1, 2, bf.bf_rows.of(x), bf.bf_rows.of(x))
        assert status_of(side) == bf.BF_ERR_RANGE and np.array_equal(before, side.host(d.pool))
    for length in (-1, 33, 2 ** 31 - 1):
        d = DeviceCache(side, c)
        d.lengths[0] = length
        before = side.host(d.pool).copy()
        bf.bf_kv4_append(side.t, d.desc, 0, None, st1, 1, 2, bf.bf_rows.of(x), bf.bf_rows.of(x))
        assert status_of(side) == bf.BF_ERR_RANGE and np.array_equal(before, side.host(d.pool))


def check_attention(side, d, layer, seqs, counts, q, heads, window, type, max_q=None, max_len=None, scale=None, starts_given=True):
    torch, c = side.torch, d.c
    starts = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    scale = c.D ** -0.5 if scale is None else scale
    pad = torch.full((int(starts[-1]) + 3, heads + 1, c.D), 5.0, device="cuda").to(side.types[type])
    out = pad[:, :heads]                                                            # rows and heads behind the last stay as they were
    lse = torch.full((int(starts[-1]) + 1, heads), 5.0, device="cuda")
    st, sq = side.ints(starts) if starts_given else None, side.ints(seqs)
    bf.bf_kv4_attention(side.t, d.desc, layer, sq, st, len(counts), max_q or max(counts), max_len or max(1, int(c.lengths.max())), bf.bf_rows.of(q), heads,
                        bf.bf_rows.of(out), scale, window, lse)
    got, gl, qd = side.host(pad), side.host(lse), side.host(q)
    assert (got[starts[-1]:] == 5).all() and (got[:, heads] == 5).all() and (gl[starts[-1]:] == 5).all()
    for i, n in enumerate(counts):
        a = seqs[i] if seqs is not None else i
        want, wl, tol, tl = ref.attention(c, layer, a, qd[starts[i]:starts[i + 1]], scale, window)
        g = got[starts[i]:starts[i + 1], :heads]
        assert (np.abs(g - want) <= tol + HALF_STEP[type] * (np.abs(want) + tol) + TINY[type]).all(), (i, n, np.abs(g - want).max(), tol.max())
        l = gl[starts[i]:starts[i + 1]]
        assert np.array_equal(np.isneginf(l), np.isneginf(wl))
        seen = ~np.isneginf(wl)
        assert (np.abs(l[seen] - wl[seen]) <= tl[seen]).all()
    return got


@gpu
@pytest.mark.parametrize("D,G", [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (3, 3), (4, 2), (7, 1), (16, 2), (9, 1), (40, 2), (66, 2)])
def test_attention_against_64_bits(side, D, G, heads, kv_heads):
    torch = side.torch
    type = "bf16" if (D + G + heads) % 64 < 32 else "fp16"
    c = ref.Cache(2, 40, kv_heads, D, G, 32, 6, 8, seed=heads)
    lens = [1, 0, 33, 16, 100, 207]
    d = fill(side, c, lens, seed=heads)
    g = torch.Generator(device="cuda").manual_seed(heads)
    for counts, window in (([1] * 6, 0), ([1] * 6, 20), ([1, 0, 5, 16, 17, 3], 0), ([3, 2, 33, 20, 1, 9], 18), ([1, 1, 1, 1, 70, 1], 0), ([1] * 6, 1)):
        qkv = torch.randn((sum(counts), heads + 3, D), generator=g, device="cuda").to(side.types[type])
        check_attention(side, d, 1, None, counts, qkv[:, 2:2 + heads], heads, window, type, starts_given=counts != [1] * 6)
    assert status_of(side) == 0


@gpu
@pytest.mark.parametrize("T", [16, 48, 256])
def test_attention_pages_lists_and_hints(side, T):
    """Other pages, sequences named in any order and twice, bounds that are not tight, a hint of the length that is wrong."""
    torch = side.torch
    c = ref.Cache(1, 80, 2, 128, 64, T, 5, 20, seed=T)
    d = fill(side, c, [300, 5, 257, 0, 1], seed=T)
    q = torch.randn((40, 4, 128), device="cuda").half()
    one = check_attention(side, d, 0, [2, 0, 2, 4], [3, 1, 3, 1], torch.cat([q[:3], q[3:4], q[:3], q[4:5]]), 4, 0, "fp16", max_q=9, max_len=1)
    assert np.array_equal(one[:3], one[4:7])
    check_attention(side, d, 0, [1, 0, 3], [1, 1, 1], q[:3], 4, 0, "fp16", max_len=100000, starts_given=False)
    check_attention(side, d, 0, [0], [1], q[:1], 4, 7, "fp16", max_len=3)
    assert status_of(side) == 0


@gpu
def test_attention_more_rows_than_tokens_and_large_windows(side):
    """Rows far before the first token see nothing, those behind it all there is, whatever the window's size."""
    torch = side.torch
    c = ref.Cache(1, 12, 2, 64, 32, 16, 3, 4)
    d = fill(side, c, [20, 1, 0])
    q = torch.randn((90, 4, 64), device="cuda").half()
    for window in (0, 1, 7, 2 ** 31 - 1, 2 ** 31, 2 ** 32 - 1):
        check_attention(side, d, 0, None, [45, 30, 15], q, 4, window, "fp16", max_len=20)
    assert status_of(side) == 0


@gpu
def test_attention_extreme_scores(side):
    """Scores far apart, all alike, far below zero, and a growing row of them; a NaN in q stays in its row."""
    torch = side.torch
    c = ref.Cache(1, 40, 1, 64, 32, 16, 2, 40)
    rng = np.random.default_rng(5)
    c.grow([0], [600])
    for t in range(600):
        c.put(0, 0, t, np.full((1, 64), t / 8.0 - 40), rng.standard_normal((1, 64)) * (50 if t % 3 else 0.01))
    d = DeviceCache(side, c)
    q = torch.zeros((6, 2, 64), device="cuda")
    q[0] = 0.02
    q[1] = -0.02
    q[2] = 5
    q[3] = -5
    q[4] = 0
    q[5, 0] = 1e-6
    q[5, 1] = 300
    for type in ("fp16", "bf16"):
        for j in range(6):
            check_attention(side, d, 0, [0], [1], q[j:j + 1].to(side.types[type]), 2, 0, type)
        check_attention(side, d, 0, [0], [6], q.to(side.types[type]), 2, 0, type)
    q[1, 0, 3], q[2, 1, 5] = float("nan"), float("inf")
    out = torch.zeros((6, 2, 64), device="cuda").half()
    st = side.ints([0, 6])
    bf.bf_kv4_attention(side.t, d.desc, 0, None, st, 1, 6, 600, qq := bf.bf_rows.of(qh := q.half()), 2, bf.bf_rows.of(out), 0.125, 0, None)
    o = side.host(out)
    assert np.isnan(o[1, 0]).all() and not np.isfinite(o[2, 1]).any()
    keep = np.ones((6, 2), bool)
    keep[1, 0] = keep[2, 1] = False
    assert np.isfinite(o[keep]).all()
    assert status_of(side) == 0


@gpu
def test_attention_leaves_bad_entries_alone(side):
    torch = side.torch
    c = ref.Cache(1, 8, 1, 64, 64, 16, 3, 3)
    d0 = fill(side, c, [40, 20, 1])
    q = torch.randn((6, 2, 64), device="cuda").half()
    for seqs, starts, max_q in (([3], [0, 1], 1), ([-1], [0, 1], 1), ([0], [0, 3], 2), ([0], [2, 1], 2), ([0], [-1, 0], 1)):
        out = torch.full((6, 2, 64), 3.0, device="cuda").half()
        sq, st = side.ints(seqs), side.ints(starts)
        bf.bf_kv4_attention(side.t, d0.desc, 0, sq, st, 1, max_q, 40, bf.bf_rows.of(q), 2, bf.bf_rows.of(out), 0.1, 0, None)
        assert status_of(side) == bf.BF_ERR_RANGE and (side.host(out) == 3).all()
    for length in (-3, 49, 2 ** 31 - 1):
        d = DeviceCache(side, c)
        d.lengths[0] = length
        out = torch.full((6, 2, 64), 3.0, device="cuda").half()
        bf.bf_kv4_attention(side.t, d.desc, 0, None, None, 1, 1, 40, bf.bf_rows.of(q), 2, bf.bf_rows.of(out), 0.1, 0, None)
        assert status_of(side) == bf.BF_ERR_RANGE and (side.host(out) == 3).all()
    # pages out of range are passed over: what is left is attended to
    d = DeviceCache(side, c)
    d.tables[0, 1] = 8
    out = torch.zeros((1, 2, 64), device="cuda").half()
    bf.bf_kv4_attention(side.t, d.desc, 0, None, None, 1, 1, 40, bf.bf_rows.of(q[:1]), 2, bf.bf_rows.of(out), 0.1, 0, None)
    assert status_of(side) == bf.BF_ERR_RANGE
    k, v = (x[np.r_[0:16, 32:40], 0] for x in c.get(0, 0, 40))
    s = 0.1 * side.host(q[0]) @ k.T
    p = np.exp(s - s.max(1, keepdims=True))
    want = p / p.sum(1, keepdims=True) @ v
    assert np.abs(side.host(out)[0] - want).max() <= 2.0 ** -9 * np.abs(v).max()


# ---- pages

@gpu
@pytest.mark.parametrize("T,heads,layers", [(16, 1, 1), (32, 3, 2), (64, 8, 3)])
def test_pages_through_a_life(side, T, heads, layers):
    """Growing, forking, freeing and compacting at random, a page short now and then: tables, counts and bytes as the plain
    lists have them."""
    rng = np.random.default_rng(T)
    c = ref.Cache(layers, 37, heads, 64, 32, T, 12, 6, seed=T)
    c.pool[:] = rng.integers(0, 256, c.pool.shape)
    d = DeviceCache(side, c)
    codes = {"range": bf.BF_ERR_RANGE, "oom": bf.BF_ERR_OOM}
    met = set()
    for step in range(300):
        what = rng.choice(["grow", "grow", "fork", "free", "compact"])
        n = int(rng.integers(1, 7))
        bad = set()
        if what == "grow":
            seqs, counts = rng.permutation(12)[:n].tolist(), rng.integers(0, 2 * T, n).tolist()
            bad = c.grow(seqs, counts)
            bf.bf_kv4_grow(side.t, d.desc, a := side.ints(seqs), b := side.ints(counts), n)
        elif what == "fork":
            src, dst = rng.integers(0, 6, n).tolist(), (6 + rng.permutation(6)[:n]).tolist()
            bad = c.fork(src, dst)
            bf.bf_kv4_fork(side.t, d.desc, a := side.ints(src), b := side.ints(dst), n)
        elif what == "free":
            seqs = rng.permutation(12)[:n].tolist()
            c.free(seqs)
            bf.bf_kv4_free(side.t, d.desc, a := side.ints(seqs), n)
        else:
            live = side.ints([-7])
            bf.bf_kv4_compact(side.t, d.desc, None, None, live)
            assert side.host(live)[0] == c.compact()
        met |= {what, *bad}
        assert status_of(side) == (codes["range"] if "range" in bad else codes["oom"] if bad else 0), (step, what)
        d.same()
    assert {"oom", "fork", "free", "compact", "grow"} <= met


@gpu
def test_pages_refuse_in_the_kernel(side):
    c = ref.Cache(1, 6, 1, 64, 64, 16, 5, 3)
    c.grow([0, 1], [20, 16])
    R = bf.BF_ERR_RANGE

    def run(call, *lists):
        d = DeviceCache(side, c)
        keep = [side.ints(x) for x in lists]
        call(side.t, d.desc, *keep, len(lists[0]))
        return d, status_of(side)

    for seqs, counts in (([7], [1]), ([-1], [1]), ([0, 0], [1, 1]), ([0], [-1]), ([0], [29]), ([2], [49]), ([1], [2 ** 31 - 1])):
        d, code = run(bf.bf_kv4_grow, seqs, counts)
        assert code == R
        if seqs == [0, 0]:
            assert side.host(d.lengths)[0] == 21                                     # the first entry counts
        else:
            d.same()
    for src, dst in (([7], [2]), ([0], [9]), ([0], [-1]), ([0], [1]), ([0], [0])):
        d, code = run(bf.bf_kv4_fork, src, dst)
        assert code == R
        d.same()
    d, code = run(bf.bf_kv4_fork, [0, 2], [2, 3])                                     # a branch of what becomes a branch in the same call
    assert code == R and list(side.host(d.lengths)) == [20, 16, 20, 0, 0]
    d, code = run(bf.bf_kv4_fork, [0, 1], [2, 2])
    assert code == R and side.host(d.lengths)[2] == 20 and list(side.host(d.refs)[:3]) == [2, 1, 1]
    d, code = run(bf.bf_kv4_free, [9])
    assert code == R
    d.same()
    d, code = run(bf.bf_kv4_free, [0, 0, 0])                                          # freed once
    assert code == 0 and list(side.host(d.refs)) == [0, 0, 1, 0, 0, 0] and list(side.host(d.lengths)) == [0, 16, 0, 0, 0]
    d = DeviceCache(side, c)
    d.refs[0] = 0                                                                    # a count that is wrong already does not go below zero
    bf.bf_kv4_free(side.t, d.desc, a := side.ints([0]), 1)
    assert status_of(side) == R and side.host(d.refs)[0] == 0
    d = DeviceCache(side, c)
    d.tables[0, 0], d.tables[1, 0] = 5, 77                                           # a free page, and none
    bf.bf_kv4_compact(side.t, d.desc, None, None, None)
    assert status_of(side) == R and side.host(d.tables)[0, 0] == -1 and side.host(d.tables)[1, 0] == -1


@gpu
def test_compact_into_other_arrays(side):
    torch, rng = side.torch, np.random.default_rng(2)
    c = ref.Cache(3, 3000, 2, 64, 64, 16, 40, 60)
    c.pool[:] = rng.integers(0, 256, c.pool.shape)
    c.grow(list(range(40)), rng.integers(1, 900, 40).tolist())
    c.free(list(range(0, 40, 3)))
    d = DeviceCache(side, c)
    before = [side.host(x).copy() for x in (d.tables, d.refs)]
    tables, refs, live = torch.full_like(d.tables, 9), torch.full_like(d.refs, 9), side.ints([0])
    for _ in range(2):                                                               # the arrays of the cache stay, so it can be done again
        bf.bf_kv4_compact(side.t, d.desc, tables, refs, live)
    assert all(np.array_equal(side.host(x), y) for x, y in zip((d.tables, d.refs), before))
    n = c.compact()
    assert side.host(live)[0] == n and np.array_equal(side.host(tables), c.tables) and np.array_equal(side.host(refs), c.refs)
    assert np.array_equal(side.host(d.pool).reshape(c.pool.shape), c.pool) and status_of(side) == 0


# ---- together

@gpu
@pytest.mark.parametrize("D,G,T,type", [(64, 64, 16, "bf16"), (128, 32, 64, "fp16")])
def test_a_decode_from_prompt_to_end(side, D, G, T, type):
    """Prompts in, a few tokens each, a fork, more tokens, an end, a compaction, more tokens: every step's attention is right."""
    torch, H, Hk, L = side.torch, 4, 2, 2
    c = ref.Cache(L, 30, Hk, D, G, T, 6, 8)
    d = DeviceCache(side, c)
    gen = torch.Generator(device="cuda").manual_seed(1)

    def step(seqs, counts):
        starts = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        sq, cs, st = side.ints(seqs), side.ints(counts), side.ints(starts)
        bf.bf_kv4_grow(side.t, d.desc, sq, cs, len(seqs))
        assert not c.grow(seqs, counts)
        for layer in range(L):
            qkv = torch.randn((sum(counts), H + 2 * Hk, D), generator=gen, device="cuda").to(side.types[type])
            q, k, v = qkv.split([H, Hk, Hk], 1)
            bf.bf_kv4_append(side.t, d.desc, layer, sq, st, len(seqs), max(counts), bf.bf_rows.of(k), bf.bf_rows.of(v))
            kh, vh = side.host(k), side.host(v)
            for i, a in enumerate(seqs):
                for j in range(counts[i]):
                    c.put(layer, a, int(c.lengths[a]) - counts[i] + j, kh[starts[i] + j], vh[starts[i] + j])
            check_attention(side, d, layer, seqs, counts, q, H, 0, type)

    step([0, 1, 2], [30, 7, 16])
    for _ in range(3):
        step([0, 1, 2], [1, 1, 1])
    bf.bf_kv4_fork(side.t, d.desc, a := side.ints([0, 2, 0]), b := side.ints([3, 4, 5]), 3)
    c.fork([0, 2, 0], [3, 4, 5])
    step([5, 0, 3, 4, 2], [1, 2, 1, 3, 1])                                           # parents and branches go their ways
    bf.bf_kv4_free(side.t, d.desc, e := side.ints([1, 0]), 2)
    c.free([1, 0])
    bf.bf_kv4_compact(side.t, d.desc)
    c.compact()
    step([2, 3, 4, 5], [1, 1, 1, 1])
    d.same()
    assert status_of(side) == 0


@gpu
def test_captured_step_replays_on_new_lengths(side):
    """A captured step (pages, append, attention, projection) replayed: every replay is a token further, as eager steps are."""
    torch, H, Hk, D = side.torch, 8, 2, 64
    rng = np.random.default_rng(9)
    packed, scales, _, _, _ = draw_matrix(rng, 100, H * D, 64, False)
    codes, sc = side.dev(packed), side.dev(scales)
    M = bf.bf_q4_matrix.of(codes, sc, None, H * D, 64)
    qkv = torch.zeros((2, H + 2 * Hk, D), dtype=torch.bfloat16, device="cuda")
    q, k, v = qkv.split([H, Hk, Hk], 1)
    steps = [torch.randn(qkv.shape, device="cuda").bfloat16() for _ in range(40)]

    def twin():
        d = DeviceCache(side, ref.Cache(1, 12, Hk, D, 32, 16, 2, 6))
        return d, torch.zeros((2, H, D), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 100), device="cuda")

    def step(t, d, out, y):
        bf.bf_kv4_grow(t, d.desc, None, None, 2)
        bf.bf_kv4_append(t, d.desc, 0, None, None, 2, 1, bf.bf_rows.of(k), bf.bf_rows.of(v))
        bf.bf_kv4_attention(t, d.desc, 0, None, None, 2, 1, 96, bf.bf_rows.of(q), H, bf.bf_rows.of(out), 0.125, 0, None)
        bf.bf_q4_linear(t, M, bf.bf_rows.of(out.view(2, -1)), 2, bf.bf_rows.of(y))

    eager, want = twin(), []
    for x in steps:
        qkv.copy_(x)
        step(side.t, *eager)
        want.append((side.host(eager[1]).copy(), side.host(eager[2]).copy()))
    d, out, y = twin()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        # the context's own stream joins the capture by an event
        capturing = torch.cuda.current_stream()
        side.stream.wait_stream(capturing)
        with torch.cuda.stream(side.stream):
            step(side.t, d, out, y)
            refused(bf.BF_ERR_INVALID_ARG, bf.bf_trusted_status, side.t)
        capturing.wait_stream(side.stream)
    for x, (a, b) in zip(steps, want):
        qkv.copy_(x)
        graph.replay()
        assert np.array_equal(side.host(out), a) and np.array_equal(side.host(y), b)
    assert status_of(side) == 0
    assert np.array_equal(side.host(d.pool), side.host(eager[0].pool)) and side.host(d.lengths).tolist() == [40, 40]


@gpu
def test_two_contexts_on_two_streams(side):
    """Calls of two contexts at the same time do not meet in a workspace."""
    torch = side.torch
    c = ref.Cache(1, 300, 1, 64, 64, 16, 2, 150)
    d = fill(side, c, [2000, 1500])
    other = torch.cuda.Stream()
    t2 = bf.bf_trusted_create(1 << 20, other.cuda_stream)
    qs = [torch.randn((2, 8, 64), device="cuda").half() for _ in range(2)]
    torch.cuda.synchronize()

    def call(t, q, out):
        bf.bf_kv4_attention(t, d.desc, 0, None, None, 2, 1, 2000, bf.bf_rows.of(q), 8, bf.bf_rows.of(out), 0.125, 0, None)

    want = [torch.empty_like(q) for q in qs]
    for q, o in zip(qs, want):
        call(side.t, q, o)
    torch.cuda.synchronize()
    outs = [[torch.zeros_like(q) for _ in range(50)] for q in qs]
    torch.cuda.synchronize()
    for i in range(50):
        call(side.t, qs[0], outs[0][i])
        call(t2, qs[1], outs[1][i])
    torch.cuda.synchronize()
    for got, w in zip(outs, want):
        assert all(torch.equal(o, w) for o in got)
    bf.bf_trusted_destroy(t2)


# ---- the encrypted product from the same 4-bit matrix, and the runner

@gpu
@pytest.mark.parametrize("offsets", [False, True])
def test_encrypted_product_from_4_bits_is_that_of_the_matrix_it_stands_for(offsets):
    """Residues of cached and on-the-fly products from 4 bits equal those from the fp32 matrix, bit for bit; refusals."""
    import torch
    from paper_2606_17421_b200 import workloads as wl
    rng = np.random.default_rng(4)
    d_out, d_in = 70, 100
    packed, scales, offs, _, _ = draw_matrix(rng, d_out, d_in, 32, offsets)
    code = np.stack([packed & 15, packed >> 4], -1).reshape(d_out, -1)[:, :d_in].astype(np.float32)
    g = np.arange(d_in) // 32
    # one rounding to fp32: products of an 11-bit scale and a 4-bit code are exact, so an fp64 sum rounds once too
    W = (scales[:, g].astype(np.float64) * (code - 8) + (offs[:, g].astype(np.float64) if offsets else 0)).astype(np.float32)
    ps = wl.PARAM_SETS["n12"]
    N, primes, r = ps["N"], list(ps["primes"]), len(ps["primes"])
    ctx = bf.bf_ctx_create(N, primes + [ps["special"]], r, ps["scale"], bf.bf_plan(64, 1, 8, 8), torch.cuda.current_stream().cuda_stream)
    try:
        steps = [k for k in range(1, 8)] + [8 * j for j in range(1, 8)]
        gen = torch.Generator(device="cuda").manual_seed(0)

        def residues(*lead, moduli):
            return torch.stack([torch.randint(0, q, (*lead, N), generator=gen, device="cuda") for q in moduli], -2)

        keys = residues(len(steps), r, 2, moduli=primes + [ps["special"]])
        bf.bf_load_eval_keys(ctx, steps, len(steps), keys)
        ct = residues(2, 2, moduli=primes)
        codes, sc, of, w32 = (None if a is None else torch.from_numpy(a).cuda() for a in (packed, scales, offs, W))
        M = bf.bf_q4_matrix.of(codes, sc, of, d_in, 32)
        want, got = torch.empty((2, 2, r, N), dtype=torch.int64, device="cuda"), torch.zeros((2, 2, r, N), dtype=torch.int64, device="cuda")
        bf.bf_linear(ctx, ct, 2, None, w32, d_out, d_in, want, 2)
        bf.bf_linear_q4(ctx, ct, 2, M, got, 2)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and bool((want != 0).any())
        for split in ((0, 0), (8, 8)):
            h = bf.bf_encode_weights_q4(ctx, M, *split)
            got.zero_()
            bf.bf_linear(ctx, ct, 2, h, None, d_out, d_in, got, 2)
            torch.cuda.synchronize()
            assert torch.equal(got, want)
            bf.bf_weights_free(ctx, h)
        refused(bf.BF_ERR_SHAPE, bf.bf_linear_q4, ctx, ct, 1, M, got, 2)
        refused(bf.BF_ERR_INVALID_ARG, bf.bf_linear_q4, ctx, None, 2, M, got, 2)
        refused(bf.BF_ERR_SHAPE, bf.bf_encode_weights_q4, ctx, M, 4, 4)
        refused(bf.BF_ERR_INVALID_ARG, bf.bf_encode_weights_q4, ctx, matrix(codes=None))
        refused(bf.BF_ERR_SHAPE, bf.bf_encode_weights_q4, ctx, matrix(group=16))
        bf.bf_set_cache_budget(ctx, 1000)
        refused(bf.BF_ERR_OOM, bf.bf_encode_weights_q4, ctx, M)
    finally:
        bf.bf_ctx_destroy(ctx)


@gpu
def test_runner_with_its_trusted_half():
    """A step of the runner: the encrypted products as without the trusted half, attention and logits as direct calls give them, and a
    cache that starts over when it is full."""
    import torch
    from paper_2606_17421_b200.runner import TrustedHalf, WorkloadRunner
    stream = torch.cuda.Stream()
    half = TrustedHalf("gpt2_qkv", seqs=2, context=30, room=3, page_tokens=16, stream=stream)
    R = WorkloadRunner("gpt2_qkv", stream=stream, trusted=half, q4_group=64)
    try:
        lens = []
        for _ in range(5):
            R.step()
            torch.cuda.synchronize()
            lens.append(half.lengths.tolist())
        assert lens == [[31] * 2, [32] * 2, [33] * 2, [31] * 2, [32] * 2]
        low = R.layers[0]["ct_low"].clone()
        R.trusted = None
        R.layers[0]["ct_low"].zero_()
        R.step()
        torch.cuda.synchronize()
        assert torch.equal(low, R.layers[0]["ct_low"])
        W = np.stack([half.codes.cpu().numpy() & 15, half.codes.cpu().numpy() >> 4], -1).reshape(half.codes.shape[0], -1)[:, :768].astype(np.float64) - 8
        W *= half.scales.cpu().numpy().astype(np.float64)[:, np.arange(768) // 64]
        x = half.hidden.double().cpu().numpy()
        assert (np.abs(half.logits.double().cpu().numpy() - x @ W.T) <= linear_tolerance(x, x @ W.T, 3 * np.abs(W) + W.std(), "fp32")).all()
        assert torch.isfinite(half.attended.float()).all() and int(half.refs.sum()) == 4
    finally:
        R.close()
        half.close()


@gpu
def test_runner_from_4_bits_beyond_the_cache_budget():
    """What the encoded cache has no room for is encoded from 4 bits inside the call: the same ciphertexts."""
    import torch
    from paper_2606_17421_b200.runner import WorkloadRunner
    out = []
    for budget in (None, 1):
        R = WorkloadRunner("gpt2_qkv", q4_group=32, cache_budget_bytes=budget)
        try:
            assert R.n_fallback_layers() == (0 if budget is None else 1)
            R.step()
            torch.cuda.synchronize()
            out.append(R.layers[0]["ct_low"].clone())
        finally:
            R.close()
    assert torch.equal(*out)


@gpu
def test_attention_keeps_a_nan_to_the_rows_that_see_it(side):
    """Tokens with a NaN in a group of their values or keys: rows that do not see them, and other groups, stay as they are."""
    torch = side.torch
    for D, G, heads in ((64, 32, 2), (128, 128, 12)):
        c = ref.Cache(1, 12, 1, D, G, 16, 1, 10)
        d = fill(side, c, [120], seed=1)
        q = torch.randn((9, heads, D), device="cuda").half()
        st = side.ints([0, 9])

        def run(cache, window):
            out = torch.zeros((9, heads, D), device="cuda").half()
            bf.bf_kv4_attention(side.t, cache.desc, 0, None, st, 1, 9, 120, bf.bf_rows.of(q), heads, bf.bf_rows.of(out), D ** -0.5, window, None)
            return side.host(out)

        for window in (0, 5):
            clean = run(d, window)
            block = c.tables[0, 115 // 16]
            sub = c.pool[0, block, 0, 0]
            keep = sub.copy()
            sub.view(np.float16)[c.vp[115 % 16, (D // G) - 1]] = np.nan                   # the last group of token 115's values
            bad = run(DeviceCache(side, c), window)
            sub[:] = keep
            sees = np.array([115 <= 111 + j and (not window or 115 > 111 + j - window) for j in range(9)])
            assert np.isnan(bad[sees][:, :, D - G:]).all()
            assert np.array_equal(bad[~sees], clean[~sees])
            if G < D:
                assert np.isfinite(bad[sees][:, :, :D - G]).all()
            sub.view(np.float16)[c.kp[115 % 16, 0]] = np.nan                              # its keys
            bad = run(DeviceCache(side, c), window)
            sub[:] = keep
            assert np.isnan(bad[sees]).all() and np.array_equal(bad[~sees], clean[~sees])
    assert status_of(side) == 0


@gpu
def test_cache_calls_on_rows_without_alignment(side):
    """Rows that start anywhere and lie any distance apart: element by element, the same bytes and results."""
    torch = side.torch
    c = ref.Cache(1, 8, 2, 64, 32, 16, 2, 4)
    lens = [50, 33]
    for type in ("bf16", "fp32"):
        d, e = DeviceCache(side, c), DeviceCache(side, c)
        flat = torch.randn(83 * 4 * 67 + 1, device="cuda").to(side.types[type])
        odd = flat[1:].view(83, 4, 67)[:, :, :64]
        even = odd.contiguous()
        st, cs = side.ints([0, 50, 83]), side.ints(lens)
        for cache, x in ((d, odd), (e, even)):
            bf.bf_kv4_grow(side.t, cache.desc, None, cs, 2)
            bf.bf_kv4_append(side.t, cache.desc, 0, None, st, 2, 50, bf.bf_rows.of(x[:, :2]), bf.bf_rows.of(x[:, 2:]))
        assert np.array_equal(side.host(d.pool), side.host(e.pool))
        out = torch.zeros_like(flat)[1:].view(83, 4, 67)[:, :, :64]
        bf.bf_kv4_read(side.t, d.desc, 0, None, st, None, 2, 50, bf.bf_rows.of(out[:, :2]), bf.bf_rows.of(out[:, 2:]))
        flush = torch.zeros_like(even)
        bf.bf_kv4_read(side.t, d.desc, 0, None, st, None, 2, 50, bf.bf_rows.of(flush[:, :2]), bf.bf_rows.of(flush[:, 2:]))
        assert torch.equal(out, flush) and bool((out != 0).any())
        if type == "fp32":
            continue
        res, flush = torch.zeros_like(flat)[1:].view(83, 4, 67)[:, :, :64], torch.zeros_like(even)
        for x, o in ((odd, res), (even, flush)):
            bf.bf_kv4_attention(side.t, d.desc, 0, None, st, 2, 50, 50, bf.bf_rows.of(x), 4, bf.bf_rows.of(o), 0.125)
        assert torch.equal(res, flush)
    assert status_of(side) == 0


@gpu
def test_small_workspace(side):
    """A context with the least workspace: the same results in smaller portions, or a refusal that enqueues nothing."""
    torch = side.torch
    t = bf.bf_trusted_create(1 << 20, side.stream.cuda_stream)
    try:
        rng = np.random.default_rng(1)
        for n, d_in in ((150, 700), (40, 6000), (3, 20000)):
            packed, scales, _, _, _ = draw_matrix(rng, 33, d_in, 128, False)
            codes, sc = side.dev(packed), side.dev(scales)
            M = bf.bf_q4_matrix.of(codes, sc, None, d_in, 128)
            x = torch.randn((n, d_in), device="cuda").bfloat16()
            y, z = torch.zeros((n, 33), device="cuda"), torch.ones((n, 33), device="cuda")
            bf.bf_q4_linear(side.t, M, bf.bf_rows.of(x), n, bf.bf_rows.of(y))
            bf.bf_q4_linear(t, M, bf.bf_rows.of(x), n, bf.bf_rows.of(z))
            assert np.abs(side.host(y) - side.host(z)).max() <= 2.0 ** -18 * np.abs(side.host(y)).max()
        packed, scales, _, _, _ = draw_matrix(rng, 2, 70000, 128, False)
        codes, sc = side.dev(packed), side.dev(scales)
        x, y = torch.randn((2, 70000), device="cuda"), torch.full((2, 2), 3.0, device="cuda")
        refused(bf.BF_ERR_TOO_LARGE, bf.bf_q4_linear, t, bf.bf_q4_matrix.of(codes, sc, None, 70000, 128), bf.bf_rows.of(x), 2, bf.bf_rows.of(y))
        assert (side.host(y) == 3).all()
        c = ref.Cache(1, 300, 1, 64, 64, 16, 2, 150)
        d = fill(side, c, [2000, 1500])
        q = torch.randn((2, 8, 64), device="cuda").half()
        check_attention(side, d, 0, None, [1, 1], q, 8, 0, "fp16", starts_given=False)
        o = torch.zeros_like(q)
        bf.bf_kv4_attention(t, d.desc, 0, None, None, 2, 1, 2000, bf.bf_rows.of(q), 8, bf.bf_rows.of(o), 0.125)
        p = torch.zeros_like(q)
        bf.bf_kv4_attention(side.t, d.desc, 0, None, None, 2, 1, 2000, bf.bf_rows.of(q), 8, bf.bf_rows.of(p), 0.125)
        assert (side.host(o) - side.host(p)).__abs__().max() <= 2.0 ** -9 * np.abs(side.host(p)).max()
    finally:
        bf.bf_trusted_destroy(t)


@gpu
def test_layers_beyond_32_bits_of_offset(side):
    """A layer's pages behind 4 GB of the pool: copies, writes, attention and compaction reach them."""
    torch = side.torch
    T, heads, pages, layers = 256, 8, 40000, 2
    block = bf.bf_kv4_block_bytes(128, 128, T)
    if torch.cuda.mem_get_info()[0] < 3 * layers * pages * heads * block // 2:
        pytest.skip("not enough memory")
    pool = torch.empty((layers, pages, heads, block), dtype=torch.uint8, device="cuda")
    assert pool[0].numel() > 2 ** 33
    tables, lengths, refs = side.ints([[pages - 1, 0], [-1, -1]]), side.ints([300, 0]), torch.zeros(pages, dtype=torch.int32, device="cuda")
    refs[0] = refs[pages - 1] = 1
    cache = bf.bf_kv4_cache.of(pool, tables, lengths, refs, 128, 128, T)
    k, v = (torch.randn((300, heads, 128), device="cuda").half() for _ in range(2))
    st = side.ints([0, 300])
    bf.bf_kv4_append(side.t, cache, 1, None, st, 1, 300, bf.bf_rows.of(k), bf.bf_rows.of(v))
    q = torch.randn((1, heads, 128), device="cuda").half()
    a, b, kk, vv = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    bf.bf_kv4_attention(side.t, cache, 1, None, None, 1, 1, 300, bf.bf_rows.of(q), heads, bf.bf_rows.of(a), 0.1)
    bf.bf_kv4_fork(side.t, cache, src := side.ints([0]), dst := side.ints([1]), 1)
    bf.bf_kv4_free(side.t, cache, src, 1)
    bf.bf_kv4_compact(side.t, cache)
    bf.bf_kv4_attention(side.t, cache, 1, dst, None, 1, 1, 300, bf.bf_rows.of(q), heads, bf.bf_rows.of(b), 0.1)
    bf.bf_kv4_read(side.t, cache, 1, dst, st, None, 1, 300, bf.bf_rows.of(kk), bf.bf_rows.of(vv))
    assert status_of(side) == 0 and side.host(tables).tolist() == [[-1, -1], [0, 1]]
    assert torch.equal(a, b)
    # half a step of the codes, and what rounding low and scale moves (2^-11 of each, the scale up to 15 times)
    for x, held in ((k, kk), (v, vv)):
        span = (x.float().amax(-1, keepdim=True) - x.float().amin(-1, keepdim=True))
        assert bool(((x.float() - held.float()).abs() <= span / 30 + 2.0 ** -10 * (span + x.float().abs().amax(-1, keepdim=True)) + 2.0 ** -11 * held.float().abs()).all())


@gpu
@pytest.mark.parametrize("D,G", [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)])
def test_attention_beside_values_that_do_not_count(side, D, G):
    """Tokens with huge values and next to no weight leave the bits of the others' values alone: single tokens and chunks, huge ones first, last
    and in between, several orders of magnitude in one sub-block."""
    torch = side.torch
    for seed, sizes in enumerate(([30000.0, 0.5], [30000.0, 0.03], [60000.0, 1e-3], [50000.0, 40.0, 0.05], [2000.0, 1.0])):
        rng = np.random.default_rng([D, G, seed])
        c = ref.Cache(1, 24, 1, D, G, 16, 1, 20)
        c.grow([0], [300])
        hidden = {0: 0, 3: -1, 5: 0, 17: -2, 150: 0, 155: 1, 156: -2, 299: 0}               # which token has which size; the rest have the last
        for t in range(300):
            size = sizes[hidden.get(t, -1)]
            k, v = rng.standard_normal((1, D)), rng.uniform(-1, 1, (1, D)) * size
            k[0, 0] = 0.0 if size == sizes[-1] else -100.0
            c.put(0, 0, t, k, v)
        d = DeviceCache(side, c)
        q = torch.from_numpy(rng.standard_normal((12, 4, D))).cuda().half()
        q[:, :, 0] = 12.0                                                                   # exp(-100) and less for what is hidden
        for counts, heads in (([1], 4), ([1], 1), ([2], 4), ([4], 4), ([12], 4)):
            check_attention(side, d, 0, [0], counts, q[:counts[0], :heads], heads, 0, "fp16")
    assert status_of(side) == 0


@gpu
def test_runner_and_trusted_half_on_streams_of_their_own():
    """Each on its own stream: the cache starts over with the right lengths however busy the runner's stream is, and a step is
    over on the runner's stream when it is over on both."""
    import torch
    from paper_2606_17421_b200.runner import TrustedHalf, WorkloadRunner
    half = TrustedHalf("gpt2_qkv", seqs=3, context=30, room=2, page_tokens=16)
    R = WorkloadRunner("gpt2_qkv", trusted=half, q4_group=64)
    try:
        assert half.stream != R.stream
        junk = [torch.full((3,), 7, dtype=torch.int32, device="cuda") for _ in range(50)]    # what the allocator hands out next holds something
        del junk
        lens = []
        for i in range(7):
            torch.cuda.synchronize()
            busy, idle = (R.stream, half.stream) if i % 2 == 0 else (half.stream, R.stream)
            with torch.cuda.stream(busy):
                torch.cuda._sleep(50_000_000)                                               # 25 ms and more
            R.step()
            junk = [torch.full((3,), 9, dtype=torch.int32, device="cuda") for _ in range(50)]
            del junk
            R.stream.synchronize()
            assert half.stream.query()
            lens.append(half.lengths.tolist())
        assert lens == [[n] * 3 for n in (31, 32, 31, 32, 31, 32, 31)]
    finally:
        R.close()
        half.close()


@gpu
def test_free_leaves_a_bad_length_alone(side):
    """A length out of range is reported; length, table and counts stay, so that nothing is handed out over them."""
    c = ref.Cache(1, 6, 1, 64, 64, 16, 3, 3)
    c.grow([0, 1, 2], [20, 16, 40])
    for length in (-1, -2 ** 31, 49, 2 ** 31 - 1):
        d = DeviceCache(side, c)
        d.lengths[0] = length
        bf.bf_kv4_free(side.t, d.desc, a := side.ints([0, 0, 1]), 3)
        assert status_of(side) == bf.BF_ERR_RANGE
        assert side.host(d.lengths).tolist() == [length, 0, 40]
        tables = c.tables.copy()
        refs = c.refs.copy()
        refs[tables[1, 0]] = 0
        tables[1, 0] = -1
        assert np.array_equal(side.host(d.tables), tables) and np.array_equal(side.host(d.refs), refs)


@gpu
@pytest.mark.parametrize("T", [16, 32])
def test_append_does_not_write_to_shared_pages(side, T):
    """Rows that reach back over a branch's own pages: what lies in pages that other sequences name stays, and is reported."""
    torch, Hk, D = side.torch, 2, 64
    c = ref.Cache(2, 12, Hk, D, 32, T, 3, 5)
    d = fill(side, c, [2 * T + 5])
    bf.bf_kv4_fork(side.t, d.desc, a := side.ints([0, 0]), b := side.ints([1, 2]), 2)
    c.fork([0, 0], [1, 2])
    bf.bf_kv4_grow(side.t, d.desc, None, n := side.ints([4, T, 0]), 3)
    c.grow([0, 1, 2], [4, T, 0])
    d.same()
    rng = np.random.default_rng(T)
    # counts of new rows: the branch's own tokens; exactly to the border; over it; over two borders
    for counts, code in (([4, T, 1], 0), ([9, T + 5, 5], 0), ([10, 1, 1], bf.BF_ERR_RANGE), ([1, T + 7, 1], bf.BF_ERR_RANGE), ([T + 11, 2, T + 6], bf.BF_ERR_RANGE)):
        x = rng.standard_normal((sum(counts), 2 * Hk, D)).astype(np.float32)
        dev = side.dev(x)
        starts = np.concatenate([[0], np.cumsum(counts)])
        bf.bf_kv4_append(side.t, d.desc, 1, None, st := side.ints(starts), 3, max(counts), bf.bf_rows.of(dev[:, :Hk]), bf.bf_rows.of(dev[:, Hk:]))
        for i in range(3):
            for j in range(counts[i]):
                t = int(c.lengths[i]) - counts[i] + j
                if c.refs[c.tables[i, t // T]] == 1:
                    c.put(1, i, t, x[starts[i] + j, :Hk].astype(np.float64), x[starts[i] + j, Hk:].astype(np.float64))
        assert status_of(side) == code
        d.same()
    # the other branches end: their pages are this one's own
    bf.bf_kv4_free(side.t, d.desc, e := side.ints([0, 2]), 2)
    c.free([0, 2])
    n = int(c.lengths[1])
    x = rng.standard_normal((n, 2 * Hk, D)).astype(np.float32)
    dev = side.dev(x)
    bf.bf_kv4_append(side.t, d.desc, 0, f := side.ints([1]), st := side.ints([0, n]), 1, n, bf.bf_rows.of(dev[:, :Hk]), bf.bf_rows.of(dev[:, Hk:]))
    for t in range(n):
        c.put(0, 1, t, x[t, :Hk].astype(np.float64), x[t, Hk:].astype(np.float64))
    assert status_of(side) == 0
    d.same()


class Held:
    """A tensor as one on a device looks to the binding: nothing behind its address."""

    def __init__(self, like, device=0):
        self.like, self.device_index, self.dtype, self.shape = like, device, like.dtype, like.shape

    def get_device(self):
        return self.device_index

    def data_ptr(self):
        return 4096

    def stride(self):
        return self.like.stride()

    def numel(self):
        return self.like.numel()

    def is_contiguous(self):
        return self.like.is_contiguous()

    def is_pinned(self):
        return False


def test_calls_refuse_tensors_that_are_too_small(stand_in):
    """What descriptors and lists are made of is compared with what a call reads and writes."""
    torch = pytest.importorskip("torch")
    z = lambda *shape, type=torch.bfloat16: Held(torch.zeros(shape, dtype=type))       # noqa: E731
    ints = lambda *shape: z(*shape, type=torch.int32)                                  # noqa: E731
    R = bf.bf_rows.of
    W = bf.bf_q4_matrix.of(z(50, 48, type=torch.uint8), z(50, 8, type=torch.float16), None, 90, 32)
    lin = lambda x, n, y: refused(bf.BF_ERR_SHAPE, bf.bf_q4_linear, stand_in, W, R(x), n, R(y))    # noqa: E731
    lin(z(4, 90), 5, z(5, 50))                                                         # rows of x, of y
    lin(z(5, 90), 5, z(4, 50))
    lin(z(5, 89), 5, z(5, 50))                                                         # columns of x, of y
    lin(z(5, 90), 5, z(5, 49))
    lin(z(5, 3, 29), 5, z(5, 50))
    lin(z(5, 3, 30), 5, z(5, 2, 24))
    c = bf.bf_kv4_cache.of(z(2, 8, 3, 64 * 16 + 256, type=torch.uint8), ints(4, 5), ints(4), ints(8), 64, 32, 16)
    good = z(6, 3, 64)
    for bad in (z(3, 3, 64), z(6, 2, 64), z(6, 3, 63), z(6, 64), z(6, 192)):
        for k, v in ((good, bad), (bad, good)):
            refused(bf.BF_ERR_SHAPE, bf.bf_kv4_append, stand_in, c, 0, None, None, 4, 1, R(k), R(v))
            refused(bf.BF_ERR_SHAPE, bf.bf_kv4_read, stand_in, c, 0, None, None, None, 4, 1, R(k), R(v))
    query = z(6, 6, 64)
    for bad in (z(3, 6, 64), z(6, 5, 64), z(6, 6, 60), z(6, 384)):
        for q, out in ((query, bad), (bad, query)):
            refused(bf.BF_ERR_SHAPE, bf.bf_kv4_attention, stand_in, c, 0, None, None, 4, 1, 50, R(q), 6, R(out), 1.0, 0, None)
    refused(bf.BF_ERR_SHAPE, bf.bf_kv4_attention, stand_in, c, 0, None, None, 4, 1, 50, R(query), 6, R(query), 1.0, 0, z(4, 5, type=torch.float32))
    # lists: seqs of n, starts of n + 1, counts and first of n
    for seqs, starts in ((ints(3), None), (None, ints(4)), (ints(4), ints(4)), (ints(2, 1), ints(5))):
        refused(bf.BF_ERR_SHAPE, bf.bf_kv4_append, stand_in, c, 0, seqs, starts, 4, 1, R(good), R(good))
        refused(bf.BF_ERR_SHAPE, bf.bf_kv4_read, stand_in, c, 0, seqs, starts, None, 4, 1, R(good), R(good))
        refused(bf.BF_ERR_SHAPE, bf.bf_kv4_attention, stand_in, c, 0, seqs, starts, 4, 1, 50, R(query), 6, R(query), 1.0, 0, None)
    refused(bf.BF_ERR_SHAPE, bf.bf_kv4_read, stand_in, c, 0, None, None, ints(3), 4, 1, R(good), R(good))
    refused(bf.BF_ERR_SHAPE, bf.bf_kv4_grow, stand_in, c, ints(3), None, 4)
    refused(bf.BF_ERR_SHAPE, bf.bf_kv4_grow, stand_in, c, None, ints(3), 4)
    refused(bf.BF_ERR_SHAPE, bf.bf_kv4_fork, stand_in, c, ints(1), ints(2), 2)
    refused(bf.BF_ERR_SHAPE, bf.bf_kv4_fork, stand_in, c, ints(2), ints(1), 2)
    refused(bf.BF_ERR_SHAPE, bf.bf_kv4_free, stand_in, c, ints(1), 2)
    refused(bf.BF_ERR_SHAPE, bf.bf_kv4_compact, stand_in, c, ints(4, 4), None, None)
    refused(bf.BF_ERR_SHAPE, bf.bf_kv4_compact, stand_in, c, None, ints(7), None)
    refused(bf.BF_ERR_SHAPE, bf.bf_kv4_compact, stand_in, c, None, None, ints(0))


def test_calls_refuse_tensors_that_are_elsewhere(stand_in):
    """On the host, or on another device than the context's."""
    torch = pytest.importorskip("torch")
    inv = bf.BF_ERR_INVALID_ARG
    t = ctypes.c_void_p(ctypes.addressof(stand_in))
    t.device = 0
    z = lambda *shape, type=torch.bfloat16: torch.zeros(shape, dtype=type)             # noqa: E731
    R, Z = bf.bf_rows.of, torch.int32
    for at in (lambda x: x, lambda x: Held(x, 1)):
        for where in range(4):
            on = lambda i, x: at(x) if i == where else Held(x)                         # noqa: E731
            W = bf.bf_q4_matrix.of(on(0, z(50, 48, type=torch.uint8)), on(1, z(50, 8, type=torch.float16)), None, 90, 32)
            refused(inv, bf.bf_q4_linear, t, W, R(on(2, z(1, 90))), 1, R(on(3, z(1, 50))))
        for where in range(10):
            c = bf.bf_kv4_cache.of(on(0, z(2, 8, 3, 64 * 16 + 256, type=torch.uint8)), on(1, z(4, 5, type=Z)), on(2, z(4, type=Z)), on(3, z(8, type=Z)), 64, 32, 16)
            q, out, lse = R(on(4, z(6, 3, 64))), R(on(5, z(6, 3, 64))), on(6, z(6, 3, type=torch.float32))
            seqs, starts, first = on(7, z(4, type=Z)), on(8, z(5, type=Z)), on(9, z(4, type=Z))
            if where < 9:
                refused(inv, bf.bf_kv4_attention, t, c, 0, seqs, starts, 4, 1, 50, q, 3, out, 1.0, 0, lse)
            if where != 6:
                refused(inv, bf.bf_kv4_read, t, c, 0, seqs, starts, first, 4, 1, q, out)
            if where < 9 and where != 6:
                refused(inv, bf.bf_kv4_append, t, c, 0, seqs, starts, 4, 1, q, out)
            if where in (0, 1, 2, 3, 7, 9):
                refused(inv, bf.bf_kv4_grow, t, c, seqs, first, 4)
                refused(inv, bf.bf_kv4_fork, t, c, seqs, first, 4)
            if where in (0, 1, 2, 3, 7):
                refused(inv, bf.bf_kv4_free, t, c, seqs, 4)
            if where < 4:
                refused(inv, bf.bf_kv4_compact, t, c)
        c = bf.bf_kv4_cache.of(Held(z(2, 8, 3, 64 * 16 + 256, type=torch.uint8)), Held(z(4, 5, type=Z)), Held(z(4, type=Z)), Held(z(8, type=Z)), 64, 32, 16)
        for tables, refs, live in ((at(z(4, 5, type=Z)), None, None), (None, at(z(8, type=Z)), None), (None, None, at(z(1, type=Z)))):
            refused(inv, bf.bf_kv4_compact, t, c, tables, refs, live)


def test_calls_refuse_no_cache(stand_in):
    r, inv = rows(), bf.BF_ERR_INVALID_ARG
    refused(inv, bf.bf_kv4_append, stand_in, None, 0, None, None, 1, 1, r, r)
    refused(inv, bf.bf_kv4_read, stand_in, None, 0, None, None, None, 1, 1, r, r)
    refused(inv, bf.bf_kv4_attention, stand_in, None, 0, None, None, 1, 1, 1, r, 1, r, 1.0)
    refused(inv, bf.bf_kv4_compact, stand_in, None)
    refused(inv, bf.bf_kv4_grow, stand_in, None, None, None, 1)


@gpu
@pytest.mark.parametrize("n,d_out", [(1, 48), (3, 48), (20, 48), (20, 19000), (64, 2400)])
def test_linear_of_values_near_the_end_of_the_range(side, n, d_out):
    """x next to the smallest normal number, and so large that only the weights bring y back into range: results are normal
    numbers and as exact as any."""
    torch = side.torch
    for xt, size in itertools.product(("fp32", "bf16"), (2.0 ** -110, 2.0 ** -119, 2.0 ** -123, 2.0 ** 121)):
        rng = np.random.default_rng([n, d_out])
        packed, scales, _, W, top = draw_matrix(rng, d_out, 300, 32, False)
        codes, sc = side.dev(packed), side.dev(scales)
        x = (torch.from_numpy(rng.standard_normal((n, 300))) * size).to(side.types[xt]).cuda()
        y = torch.empty((n, d_out), device="cuda")
        bf.bf_q4_linear(side.t, bf.bf_q4_matrix.of(codes, sc, None, 300, 32), bf.bf_rows.of(x), n, bf.bf_rows.of(y))
        xd, got = side.host(x), side.host(y)
        want = xd @ W.T
        # (a sum below the normal range, 2^-126, may be rounded to that range's last place at each of its steps)
        tol = linear_tolerance(xd, want, top, "fp32") + 64 * 2.0 ** -149
        assert (np.abs(got - want) <= tol).all(), (xt, size, np.abs(got - want).max() / size)


def random_tokens(c, lens, seed=0):
    """Sequences of these lengths with any codes and parameters as ordinary keys and values have them, made at once."""
    rng = np.random.default_rng(seed)
    c.grow(list(range(len(lens))), list(lens))
    c.pool[:] = rng.integers(0, 256, c.pool.shape, dtype=np.uint8)
    half = c.pool.view(np.float16)
    for par, low_at in ((c.kp, 1), (c.vp, 4)):
        at = np.unique(par)
        half[..., at] = rng.uniform(0.1, 0.4, (*c.pool.shape[:4], at.size)).astype(np.float16)
        half[..., at + low_at] = rng.uniform(-3, -1, (*c.pool.shape[:4], at.size)).astype(np.float16)


@gpu
@pytest.mark.parametrize("D,G", [(64, 32), (128, 128)])
def test_attention_of_queries_near_the_end_of_the_range(side, D, G):
    """Scores of 10^36: finite in 32 bits, so the token with the largest is the answer, and log-sum-exp is its score."""
    torch = side.torch
    for length in (50, 5000):
        c = ref.Cache(1, length // 16 + 2, 1, D, G, 16, 1, length // 16 + 1)
        random_tokens(c, [length])
        d = DeviceCache(side, c)
        k, v = c.get(0, 0, length)
        vt = c.top(0, 0, length)[1]
        for size in (2.0 ** 80, 2.0 ** 110, 2.0 ** 119, 2.0 ** 122):
            q = (torch.randn((12, 2, D), device="cuda") * size).bfloat16()
            qd = side.host(q)
            for rows in (1, 3, 12):
                st = side.ints([0, rows])
                out, lse = torch.zeros((rows, 2, D), device="cuda").bfloat16(), torch.zeros((rows, 2), device="cuda")
                bf.bf_kv4_attention(side.t, d.desc, 0, None, st, 1, rows, length, bf.bf_rows.of(q[:rows]), 2, bf.bf_rows.of(out), D ** -0.5, 0, lse)
                o, l = side.host(out), side.host(lse)
                for j, h in itertools.product(range(rows), range(2)):
                    n = length - rows + j + 1
                    s = D ** -0.5 * (k[:n, 0] @ qd[j, h])
                    at = int(s.argmax())
                    # (next to a tie the answer is a mixture; none of these are: gaps are 10^30 and more)
                    assert np.abs(o[j, h] - v[at, 0]).max() <= (2.0 ** -8 + 2.0 ** -10) * vt[at, 0].max(), (length, size, rows)
                    assert abs(l[j, h] - s[at]) <= 2.0 ** -16 * np.abs(s).max()
    assert status_of(side) == 0


@gpu
def test_attention_scale_that_brings_scores_back_into_range(side):
    """q beyond what a score could be, a scale as small: ordinary scores, and the other way round."""
    torch = side.torch
    c = ref.Cache(1, 10, 2, 64, 32, 16, 1, 8)
    random_tokens(c, [100])
    d = DeviceCache(side, c)
    base = torch.randn((5, 4, 64), device="cuda")
    for e in (-100, -60, 60, 100, 114, 122):
        q = (base * 2.0 ** e).bfloat16()
        for rows in (1, 5):
            check_attention(side, d, 0, [0], [rows], q[:rows], 4, 0, "bf16", scale=0.125 * 2.0 ** -e)
    assert status_of(side) == 0


@pytest.mark.parametrize("name,fused,calls", [("qwen3_step", False, ["q", "k", "v", "*", "o", "gate", "up", "down"]), ("qwen3_step", True, ["q+k+v", "*", "o", "gate+up", "down"]),
                                              ("gpt2_step", True, ["qkv", "*", "out_proj", "ffn_up", "ffn_down"]), ("gpt2_qkv", True, ["qkv", "*"]),
                                              ("llama3_layer", False, ["q", "k", "v", "*", "o", "gate", "up", "down"])])
def test_attention_follows_q_k_and_v(name, fused, calls):
    """The order of a step's work, stacked projections or not: attention of a layer once all it reads is there."""
    from types import SimpleNamespace

    from paper_2606_17421_b200 import workloads as wl
    from paper_2606_17421_b200.runner import WorkloadRunner
    w = wl.WORKLOADS[name]
    units = [wl.Layer(nm, d_in, 0, ms[0].input) for nm, d_in, ms in wl.fuse_shared_inputs(w.layers, w.plan.D)] if fused else w.layers
    R, did = WorkloadRunner.__new__(WorkloadRunner), []
    R.layers = [dict(layer=L, rep=rep) for rep in range(w.n_repeat) for L in units]
    R.stream = "one"
    R.trusted = SimpleNamespace(stream="one", begin=lambda: did.append("<"), attend=lambda rep: did.append(("*", rep)), finish=lambda: did.append(">"))
    R._call = lambda e: did.append((e["layer"].name, e["rep"]))
    R.step()
    assert did == ["<"] + [(c, rep) for rep in range(w.n_repeat) for c in calls] + [">"]


def test_attention_of_layers_with_one_input():
    """Layers that are nothing but q, k and v, one after the other."""
    from types import SimpleNamespace

    from paper_2606_17421_b200 import workloads as wl
    from paper_2606_17421_b200.runner import WorkloadRunner
    for units in ([wl.Layer("qkv", 8, 24)], [wl.Layer(x, 8, 8, "attn") for x in "qkv"]):
        R, did = WorkloadRunner.__new__(WorkloadRunner), []
        R.layers = [dict(layer=L, rep=rep) for rep in range(3) for L in units]
        R.stream = "one"
        R.trusted = SimpleNamespace(stream="one", begin=lambda: None, attend=lambda rep: did.append("*"), finish=lambda: None)
        R._call = lambda e: did.append(e["layer"].name)
        R.step()
        assert did == ([L.name for L in units] + ["*"]) * 3


def test_trusted_half_refuses_and_ends(monkeypatch):
    """No room for a step's token is refused before anything is made; a context that found something wrong is destroyed all the same."""
    from paper_2606_17421_b200.runner import TrustedHalf
    for kw in (dict(room=0), dict(seqs=0), dict(context=0), dict(room=-1)):
        with pytest.raises(ValueError):
            TrustedHalf("gpt2_qkv", **kw)
    half, gone = TrustedHalf.__new__(TrustedHalf), []
    half.ctx = "context"

    def found(t):
        raise bf.BifrostError(bf.BF_ERR_RANGE, "bf_trusted_status")

    monkeypatch.setattr(bf, "bf_trusted_status", found)
    monkeypatch.setattr(bf, "bf_trusted_destroy", gone.append)
    refused(bf.BF_ERR_RANGE, half.close)
    assert gone == ["context"]


def product_in_64_bits(torch, codes, scales, offs, d_in, group, x):
    """(y, what linear_tolerance's `top` gives for |x|, and for the largest of a row), by pieces on the device."""
    col = torch.arange(d_in, device="cuda")
    ys, mags, bigs = [], [], []
    xd = x.double()
    for at in range(0, codes.shape[0], 2048):
        some = slice(at, at + 2048)
        code = (codes[some][:, col // 2].int() >> (4 * (col % 2)) & 15).double()
        s = scales[some][:, col // group].double()
        z = offs[some][:, col // group].double() if offs is not None else torch.zeros_like(s)
        ys.append(xd @ (s * (code - 8) + z).t())
        top = s * 23 + z.abs()
        mags.append(xd.abs() @ top.t())
        bigs.append(xd.abs().amax(1, keepdim=True) * top.sum(1))
    return [torch.cat(a, 1).cpu().numpy() for a in (ys, mags, bigs)]


def check_product(side, t, n, d_in, d_out, group, offsets, xt, yt, strided=False, x=None, seed=0):
    torch = side.torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    groups = -(-d_in // group)
    codes = torch.randint(0, 256, (d_out, -(-d_in // 32) * 16), generator=gen, device="cuda", dtype=torch.uint8)
    scales = (torch.rand((d_out, -(-groups // 8) * 8), generator=gen, device="cuda") * 0.009 + 0.001).half()
    offs = (torch.randn(scales.shape, generator=gen, device="cuda") * 0.02).half() if offsets else None
    for a in (scales, offs):
        if a is not None:
            a[:, groups:] = float("nan")
    if x is None:
        x = torch.randn((n, d_in), generator=gen, device="cuda")
    x = x.to(side.types[xt])
    pad = torch.full((n + 1, d_out + 11), 5.0, device="cuda").to(side.types[yt])
    if strided:                                                                              # odd strides, odd starts
        x, y = torch.nn.functional.pad(x, (7, 2))[:, 7:7 + d_in], pad[:, 3:3 + d_out]
    else:
        y = pad[:, :d_out]
    bf.bf_q4_linear(t, bf.bf_q4_matrix.of(codes, scales, offs, d_in, group), bf.bf_rows.of(x), n, bf.bf_rows.of(y))
    want, mag, big = product_in_64_bits(torch, codes, scales, offs, d_in, group, x)
    got, at = side.host(y), 3 if strided else 0
    tol = HALF_STEP[yt] * np.abs(want) + 2.0 ** -22 * (d_in / 16 + d_in / 32 + 24) * mag + 2.0 ** -24 * big + TINY[yt]
    fine = np.isfinite(side.host(x)).all(1)
    assert (np.abs(got[:n] - want)[fine] <= tol[fine]).all(), (np.abs(got[:n] - want) - tol)[fine].max()
    assert not np.isfinite(got[:n][~fine]).any()
    rest = side.host(pad)
    assert (rest[n] == 5).all() and (rest[:, :at] == 5).all() and (rest[:, at + d_out:] == 5).all()


WIDE = [(12, 333, 19001, 64), (20, 600, 18950, 32), (30, 1000, 19000, 128), (64, 333, 2400, 128), (100, 520, 2401, 64)]


@gpu
@pytest.mark.parametrize("n,d_in,d_out,group", WIDE)
def test_linear_of_many_outputs_strided(side, n, d_in, d_out, group):
    """Rows without alignment through the products of 128 rows of W at a time."""
    for i, (xt, yt) in enumerate((("bf16", "fp32"), ("fp32", "fp16"), ("fp16", "bf16"))):
        if xt == "fp32" and d_out > 18000:
            n = max(n // 2, 9)
        check_product(side, side.t, n, d_in, d_out, group, i == 1, xt, yt, strided=True, seed=i)
    bf.bf_trusted_status(side.t)


@gpu
@pytest.mark.parametrize("n,d_in,d_out,group", WIDE)
def test_linear_of_many_outputs_with_extreme_rows(side, n, d_in, d_out, group):
    """Rows of zeros, tiny and huge values; NaN and infinities stay in their rows."""
    torch = side.torch
    for xt in ("fp32", "bf16", "fp16"):
        rows = n // 2 if xt == "fp32" else n
        x = torch.randn((rows, d_in), device="cuda")
        x[0] = 0
        if xt != "fp16":
            x[1] *= 1e-30
            x[2] *= 1e30
        x[3, ::7] *= 1e3
        x[4, d_in - 1] = float("nan")
        x[5, 3] = float("-inf")
        check_product(side, side.t, rows, d_in, d_out, group, xt == "bf16", xt, "fp32", x=x)
    bf.bf_trusted_status(side.t)


@gpu
@pytest.mark.parametrize("n,d_in,d_out,group,xt", [(150, 6000, 2400, 128, "bf16"), (90, 6000, 2333, 64, "fp32"), (40, 8000, 19000, 128, "bf16"), (17, 16500, 19001, 64, "fp16"),
                                                  (70, 8000, 19000, 32, "bf16")])
def test_linear_of_many_outputs_in_a_small_workspace(side, n, d_in, d_out, group, xt):
    """More rows than the workspace holds at once, and narrower chunks of them, through the products of 128 rows of W at a time."""
    t = bf.bf_trusted_create(1 << 20, side.stream.cuda_stream)
    try:
        check_product(side, t, n, d_in, d_out, group, False, xt, "fp32")
        bf.bf_trusted_status(t)
    finally:
        bf.bf_trusted_destroy(t)


@gpu
@pytest.mark.parametrize("length,D,G", [(20000, 64, 32), (76001, 64, 64), (40000, 128, 64)])
def test_attention_of_many_splits(side, length, D, G):
    """One sequence and one key head, so that its tokens are split over more blocks than a warp has lanes."""
    torch = side.torch
    pages = -(-length // 64)
    c = ref.Cache(1, pages + 1, 1, D, G, 64, 1, pages)
    random_tokens(c, [length], seed=length)
    d = DeviceCache(side, c)
    q = torch.randn((6, 2, D), device="cuda").half()
    check_attention(side, d, 0, None, [1], q[:1], 2, 0, "fp16", starts_given=False)
    check_attention(side, d, 0, None, [3], q[:3], 2, 15000, "fp16")
    check_attention(side, d, 0, None, [6], q, 2, 0, "fp16")
    assert status_of(side) == 0


def test_descriptors_take_attributes_and_pinned_memory(stand_in):
    """A caller may hang what has to live as long on a descriptor; memory that the device reaches on the host is let through."""
    torch = pytest.importorskip("torch")
    x = torch.zeros(2, 64)
    rows_, W = bf.bf_rows.of(x), bf.bf_q4_matrix.of(torch.zeros(4, 16, dtype=torch.uint8), torch.zeros(4, 8, dtype=torch.float16), None, 32, 32)
    c = bf.bf_kv4_cache.of(torch.zeros(1, 2, 1, 64 * 16 + 128, dtype=torch.uint8), *(torch.zeros(s, dtype=torch.int32) for s in ((1, 1), (1,), (2,))), 64, 64, 16)
    for d in (rows_, W, c, rows(), matrix(), cache()):
        d.keep = x
    pinned = Held(x, -1)
    pinned.is_pinned = lambda: True
    assert bf.bf_rows.of(pinned).device is None and bf._common(pinned, pinned) is None and bf._common(Held(x), pinned) == 0
    assert bf._common(Held(x), Held(x, 1)) == -1 and bf._common(Held(x, -1), Held(x, -1)) == -1


@gpu
def test_runner_and_trusted_half_in_one_graph():
    """A step captured on the runner's stream takes the half's stream with it: replays go on where eager steps ended."""
    import torch
    from paper_2606_17421_b200.runner import TrustedHalf, WorkloadRunner
    half = TrustedHalf("gpt2_qkv", seqs=2, context=20, room=12, page_tokens=16)
    R = WorkloadRunner("gpt2_qkv", trusted=half)
    try:
        R.step()
        R.step()
        torch.cuda.synchronize()
        assert half.lengths.tolist() == [22, 22]
        low, logits = R.layers[0]["ct_low"].clone(), half.logits.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=R.stream):
            R.step()
        torch.cuda.synchronize()
        assert half.lengths.tolist() == [22, 22]
        for i in range(3):
            R.layers[0]["ct_low"].zero_()
            half.logits.zero_()
            half.attended.fill_(float("nan"))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert half.lengths.tolist() == [23 + i] * 2 and int(half.refs.sum()) == 4
            assert torch.equal(low, R.layers[0]["ct_low"]) and torch.equal(logits, half.logits) and bool(torch.isfinite(half.attended.float()).all())
        bf.bf_trusted_status(half.ctx)
    finally:
        R.close()
        half.close()
