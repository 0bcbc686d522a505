"""The serving operators (ssd_kvq_*, ssd_rope_axes, ssd_sample_logits) against plain 64-bit implementations
(tests/serve_util.py), at the sizes, masks and strides where they can go wrong."""
import ctypes
from concurrent.futures import ThreadPoolExecutor

import numpy as np
import pytest

import paper_2606_20543_amd as ssd
from tests import gpu_util as G
from tests import serve_util as S

pytestmark = pytest.mark.gpu


class Dev:
    """Device arrays of one test, freed with it."""

    def __init__(self):
        self.all = []

    def __call__(self, host):
        a = G.DeviceArray(np.ascontiguousarray(host))
        self.all.append(a)
        return a

    def free(self):
        for a in self.all:
            a.free()


@pytest.fixture
def dev():
    d = Dev()
    yield d
    d.free()


def upload(a, host):
    host = np.ascontiguousarray(host)
    assert host.nbytes == a.nbytes
    assert G.DeviceArray.hip().hipMemcpy(a.ptr, host.ctypes.data, a.nbytes, 1) == 0


def typed(x, dtype):
    """(array as the device holds it, its values in float64)."""
    x = np.asarray(x, np.float32)
    if dtype == "bf16":
        b = S.bf16_bits(x)
        return b, S.bf16_value(b).astype(np.float64)
    return x, x.astype(np.float64)


def values(a, dtype):
    h = a.numpy()
    return (S.bf16_value(h) if dtype == "bf16" else h).astype(np.float64)


def code(dtype):
    return ssd.SSD_BF16 if dtype == "bf16" else ssd.SSD_F32


# ---------------------------------------------------------------- block tables and slots
def slot_case(rng, B, block, width, most_held, most_fresh, short=0, pad=0, cut=0):
    held = rng.integers(0, most_held + 1, B).astype(np.int32)
    fresh = rng.integers(0, most_fresh + 1, B).astype(np.int32)
    blocks = int(sum(min(-(-int(h + f) // block), width) for h, f in zip(held, fresh)))
    ids = rng.permutation(blocks + 9).astype(np.int32)
    table, at = np.full((B, width), -7, np.int32), 0
    for b in range(B):
        n = min(-(-int(held[b]) // block), width)
        table[b, :n] = ids[at:at + n]
        at += n
    pool = ids[at:]
    if short:
        pool = pool[:max(0, blocks - at - short)]
    return held, fresh, pool, table, max(0, int(fresh.sum()) + pad - cut)


SLOTS = [  # B, block, width, held, fresh, short of blocks, padded rows, rows cut
    (1, 16, 1, 0, 1, 0, 0, 0), (1, 16, 4, 15, 2, 0, 3, 0), (7, 16, 9, 100, 40, 0, 0, 0), (8, 32, 20, 500, 1, 0, 1, 0),
    (9, 64, 70, 4352, 0, 0, 4, 0), (64, 64, 69, 4352, 1, 0, 0, 0), (65, 128, 40, 3000, 700, 0, 17, 0),
    (300, 16, 12, 150, 30, 0, 5, 0), (33, 16, 4, 90, 60, 0, 2, 0), (20, 16, 30, 200, 90, 11, 6, 0), (5, 32, 9, 64, 90, 0, 0, 40),
    (1, 16, 5000, 9000, 60000, 0, 700, 0), (40, 64, 60, 800, 3000, 0, 20000, 0), (3, 128, 600, 0, 30000, 40, 0, 900),
    (700, 32, 90, 2000, 40, 0, 33000, 0)]


@pytest.mark.parametrize("B,block,width,held,fresh,short,pad,cut", SLOTS)
def test_slots(dev, B, block, width, held, fresh, short, pad, cut):
    rng = np.random.default_rng(B * 100 + block + fresh)
    h, f, pool, table, n = slot_case(rng, B, block, width, held, fresh, short, pad, cut)
    if B > 5:
        h[3], f[4] = -5, -2  # count as 0
        table[3] = np.maximum(table[3], 0)
    want = S.slots(h, f, pool, table, block, n)
    p = ssd.ssd_kvq_slot_params(B, block, width, len(pool), n)
    ins = [dev(x) for x in (h, f, pool if len(pool) else np.zeros(1, np.int32))]
    t = dev(table)
    outs = [dev(np.full(max(1, x), 99, np.int32)) for x in (B, B + 1, n, n, 1)]
    for _ in range(2):  # again: the same
        ssd.ssd_kvq_slots(p, *[x.ptr for x in ins], t.ptr, *[x.ptr for x in outs])
        got = [t.numpy()] + [x.numpy() for x in outs]
        for name, a in zip(("table", "lens", "cu", "slots", "positions", "used"), got):
            w = want[name]
            assert np.array_equal(a.reshape(-1)[:w.size], w.reshape(-1)), name


# ---------------------------------------------------------------- rotary positions
ROPE = [  # dtype, T, heads, kv, D, section, extra row length, first element off
    ("f32", 1, 4, 4, 64, (8, 12, 12), 0, 0), ("bf16", 1, 16, 16, 128, (16, 24, 24), 0, 0),
    ("bf16", 67, 32, 8, 128, (16, 24, 24), 8, 0), ("f32", 33, 5, 1, 64, (32,), 4, 0),
    ("bf16", 5, 3, 1, 96, (7, 9, 11, 3), 1, 1), ("f32", 7, 2, 2, 64, (0, 5, 10), 3, 1),
    ("bf16", 9, 8, 2, 128, (16, 16), 0, 0), ("f32", 4, 1, 1, 2, (1,), 0, 0), ("f32", 3, 2, 1, 1024, (500, 12), 0, 0),
    ("bf16", 130, 4, 2, 64, (8, 8, 16), 64, 0)]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("dtype,T,heads,kv,D,section,extra,off", ROPE)
def test_rope_axes(dev, dtype, T, heads, kv, D, section, extra, off, in_place):
    rng = np.random.default_rng(T + D)
    theta = 1e4
    cq, ck = heads * D, kv * D
    ld = cq + ck + extra
    raw, x = typed(rng.standard_normal(off + T * ld) * 3, dtype)
    pos = rng.integers(-50, 5000, (len(section), T)).astype(np.int32)
    pos[0, 0], pos[-1, -1] = 2 ** 31 - 1, -2 ** 31
    es = raw.itemsize
    src, P = dev(raw), dev(pos)
    rows = x[off:].reshape(T, ld)
    q, k = rows[:, :cq].reshape(T, heads, D), rows[:, cq:cq + ck].reshape(T, kv, D)
    p = ssd.ssd_rope_params(n_heads=heads, n_kv_heads=kv, head_dim=D, dtype=code(dtype), n_axes=len(section), theta=theta)
    for i, n in enumerate(section):
        p.section[i] = n
    p.ld_q = p.ld_k = ld
    qa = src.ptr + off * es
    if in_place:
        p.ld_q_out = p.ld_k_out = ld
        ssd.ssd_rope_axes(p, T, qa, qa + cq * es, P.ptr, qa, qa + cq * es)
        got = values(src, dtype)
        assert np.array_equal(got[:off], x[:off])
        got = got[off:].reshape(T, ld)
        assert np.array_equal(got[:, cq + ck:], rows[:, cq + ck:])  # the gap between rows stays
        gq, gk = got[:, :cq].reshape(T, heads, D), got[:, cq:cq + ck].reshape(T, kv, D)
    else:
        p.ld_q_out, p.ld_k_out = cq + extra, ck
        qo, ko = dev(np.zeros(T * (cq + extra), raw.dtype)), dev(np.zeros(T * ck, raw.dtype))
        ssd.ssd_rope_axes(p, T, qa, qa + cq * es, P.ptr, qo.ptr, ko.ptr)
        assert np.array_equal(src.numpy(), raw)
        gq = values(qo, dtype).reshape(T, -1)
        assert not gq[:, cq:].any()
        gq, gk = gq[:, :cq].reshape(T, heads, D), values(ko, dtype).reshape(T, kv, D)
    half = sum(section)
    for got, want, v in ((gq, S.rope(q, pos, section, theta), q), (gk, S.rope(k, pos, section, theta), k)):
        # a factor is off by its own rounding, the half turns' (pi 2^-25) and sincospi's few units: 6 units of 2^-24 with
        # the product and the sum; a far position's float64 angle by 2^31 2^-52 rounded a few times
        size = np.abs(v).copy()
        size[..., :half] += np.abs(v[..., half:2 * half])
        size[..., half:2 * half] += np.abs(v[..., :half])
        tol = size * (6 * 2.0 ** -24 + 2.0 ** 31 * 2.0 ** -50) + (np.abs(want) * 2.0 ** -8 if dtype == "bf16" else 0)
        worst = float((np.abs(got - want) - tol).max())
        assert worst <= 0
        assert np.array_equal(got[..., 2 * half:], v[..., 2 * half:])


# ---------------------------------------------------------------- cache writes
def cache_arrays(dev, rng, n_blocks, kv, block, D, live=True):
    """A cache of finite codes, and the same for the plain implementation."""
    def codes(shape):
        c = rng.integers(0, 256, shape).astype(np.uint8)
        c[(c & 127) == 127] = 5
        return c
    k, v = codes((n_blocks, kv, block, D)), codes((n_blocks, kv, D, block))
    ke, ve = (rng.integers(116, 122, (n_blocks, kv)).astype(np.uint8) for _ in range(2))
    arrs = [dev(x) for x in (k, v, ke, ve)]
    c = ssd.ssd_kvq_cache(*[x.ptr for x in arrs], n_blocks, block, kv, D)
    plain = S.Cache(n_blocks, kv, block, D)
    plain.load(k, v, ke, ve)
    return c, arrs, plain


def assert_cache(arrs, plain):
    k, v, ke, ve = [x.numpy() for x in arrs]
    assert np.array_equal(ke, plain.ke) and np.array_equal(ve, plain.ve)
    assert np.array_equal(S.E4M3[k], plain.k)
    assert np.array_equal(S.E4M3[v].swapaxes(2, 3), plain.v)


def rows_of(rng, n, kv, D, dtype, ld, spread=1.0):
    x = rng.standard_normal((n, ld)) * np.exp(rng.standard_normal((n, 1)) * spread)
    raw, val = typed(x, dtype)
    return raw, val[:, :kv * D].reshape(n, kv, D)


APPEND = [  # dtype, block, kv, D, runs (block, offset, length), extra row length
    ("bf16", 16, 1, 64, [(0, 0, 1)], 0),
    ("bf16", 64, 8, 128, [(3, 0, 64), (1, 17, 1), (0, 63, 1), (2, 5, 30)], 0),
    ("f32", 32, 4, 64, [(4, 31, 1), (0, 0, 32), (1, 0, 7), (2, 8, 24)], 4),
    ("f32", 128, 2, 128, [(1, 0, 128), (0, 1, 127), (2, 100, 3)], 1),
    ("bf16", 128, 3, 64, [(2, 77, 51), (0, 0, 128), (1, 0, 65)], 3),
    ("bf16", 16, 5, 128, [(6, 15, 1), (5, 0, 16), (4, 0, 16), (0, 2, 3), (1, 1, 15)], 8),
    ("f32", 64, 1, 128, [(i, (i * 13) % 64, 1) for i in range(40)], 0)]


@pytest.mark.parametrize("dtype,block,kv,D,runs,extra", APPEND)
@pytest.mark.parametrize("spread", [0.5, 6.0])
def test_append(dev, dtype, block, kv, D, runs, extra, spread):
    rng = np.random.default_rng(block + D)
    c, arrs, plain = cache_arrays(dev, rng, 41, kv, block, D)
    slots = []
    for p, o, n in runs:  # between the runs rows that are skipped
        slots += list(range(p * block + o, p * block + o + n)) + [-1]
    slots = np.array(slots + [41 * block, 2 ** 31 - 1, -2 ** 31], np.int32)
    n, ld = len(slots), kv * D + extra
    k, kval = rows_of(rng, n, kv, D, dtype, ld, spread)
    v, vval = rows_of(rng, n, kv, D, dtype, ld, spread)
    p = ssd.ssd_kvq_append_params(code(dtype), n, ld, ld)
    ds, dk, dv = dev(slots), dev(k), dev(v)
    plain.append(slots, kval, vval)
    for _ in range(2):  # the same rows again: nothing changes
        ssd.ssd_kvq_append(c, p, ds.ptr, dk.ptr, dv.ptr)
        assert_cache(arrs, plain)


@pytest.mark.parametrize("dtype,block,D,rows,extra", [
    ("bf16", 16, 64, 2100, 0), ("f32", 32, 128, 2500, 0), ("bf16", 64, 128, 17000, 0), ("bf16", 128, 128, 16500, 8),
    ("f32", 128, 128, 17000, 4), ("f32", 128, 64, 5000, 0), ("bf16", 32, 64, 16400, 1)])
def test_append_long(dev, dtype, block, D, rows, extra):
    """Prompts of many blocks between single tokens and skipped rows: every length of the windows that look for runs."""
    rng = np.random.default_rng(rows + block)
    n_blocks = 2 * rows // block + 80
    c, arrs, plain = cache_arrays(dev, rng, n_blocks, 1, block, D)
    pages, slots = iter(rng.permutation(n_blocks).tolist()), []
    while len(slots) < rows:
        kind = rng.integers(4)
        if kind == 0:
            slots += [-1] * int(rng.integers(1, 70))
        elif kind == 1:  # single tokens of several requests
            slots += [next(pages) * block + int(rng.integers(block)) for _ in range(int(rng.integers(1, 9)))]
        else:  # a prompt behind held tokens
            off, left = int(rng.integers(block)), int(rng.integers(1, 20 * block))
            while left > 0:
                n = min(block - off, left)
                p = next(pages) * block
                slots += range(p + off, p + off + n)
                off, left = 0, left - n
    slots = np.array(slots[:rows], np.int32)
    k, kval = rows_of(rng, rows, 1, D, dtype, D + extra, 3.0)
    v, vval = rows_of(rng, rows, 1, D, dtype, D + extra, 3.0)
    plain.append(slots, kval, vval)
    ssd.ssd_kvq_append(c, ssd.ssd_kvq_append_params(code(dtype), rows, D + extra, D + extra), dev(slots).ptr,
                       dev(k).ptr, dev(v).ptr)
    assert_cache(arrs, plain)


def test_append_special_values(dev):
    """Zeros, subnormal and huge magnitudes, infinities, NaN, values at 448 and half way between codes."""
    rng = np.random.default_rng(3)
    block, kv, D = 16, 9, 64
    c, arrs, plain = cache_arrays(dev, rng, 4, kv, block, D)
    x = np.zeros((5, kv, D), np.float32)
    x[:, 1] = 1e-42
    x[:, 2] = rng.standard_normal((5, D)) * 1e-30
    x[:, 3] = rng.standard_normal((5, D)) * 1e37
    x[:, 4] = np.where(rng.random((5, D)) < 0.2, np.inf, rng.standard_normal((5, D)))
    x[:, 5] = np.where(rng.random((5, D)) < 0.2, np.nan, rng.standard_normal((5, D)))
    x[:, 6] = np.where(rng.random((5, D)) < 0.5, -np.inf, np.nan)
    x[:, 7] = np.resize(np.array([448, -448, 447.99, 17, 18, 19, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -6, -0.0]), (5, D))
    x[:, 8] = np.resize(np.array([448.1, 1, 1.0625, 1.1875, 480, 464]), (5, D))
    for slots in (np.arange(16, 21), np.arange(40, 45)):
        slots = slots.astype(np.int32)
        plain.append(slots, x.astype(np.float64), -x.astype(np.float64))
        ssd.ssd_kvq_append(c, ssd.ssd_kvq_append_params(ssd.SSD_F32, 5, kv * D, kv * D), dev(slots).ptr,
                           dev(x).ptr, dev(-x).ptr)
        assert_cache(arrs, plain)


def test_append_nothing(dev):
    rng = np.random.default_rng(4)
    c, arrs, plain = cache_arrays(dev, rng, 3, 2, 16, 64)
    ssd.ssd_kvq_append(c, ssd.ssd_kvq_append_params(ssd.SSD_F32, 0, 128, 128), None, None, None)
    ssd.ssd_kvq_append(c, ssd.ssd_kvq_append_params(ssd.SSD_F32, 1, 128, 128), dev(np.array([-1], np.int32)).ptr,
                       dev(np.ones(128, np.float32)).ptr, dev(np.ones(128, np.float32)).ptr)
    assert_cache(arrs, plain)


@pytest.mark.parametrize("dtype,D,block", [("bf16", 128, 64), ("f32", 128, 32), ("bf16", 64, 32), ("f32", 64, 64), ("bf16", 128, 128)])
@pytest.mark.parametrize("requests,step", [(1, 1), (2, 1), (1, 3), (2, 5), (9, 1)])
def test_append_where_the_scale_grows(dev, dtype, D, block, requests, step):
    """A few requests fill a block each from its first token, `step` rows a call: every call finds a larger magnitude, so
    the older codes of both sides are rounded again while the new ones are stored beside them, in the same words."""
    rng = np.random.default_rng(block + D + 10 * requests + step)
    kv, rows = 24, requests * step
    c, arrs, plain = cache_arrays(dev, rng, requests + 2, kv, block, D)
    pages = rng.permutation(requests + 2)[:requests]
    p = ssd.ssd_kvq_append_params(code(dtype), rows, kv * D, kv * D)
    calls = -(-block // step)
    growth = np.exp2(12.0 / calls)  # 12 steps of the exponent from first to last
    raw = [[], []]
    for i in range(calls):
        size = growth ** i * (1 + 0.2 * rng.random((rows, kv, 1)))
        for side in raw:
            side.append(typed((rng.uniform(-1, 1, (rows, kv, D)) * size).reshape(rows, kv * D), dtype))
    dk, dv = (dev(np.stack([x[0] for x in side])) for side in raw)
    slots = np.full((calls, rows), -1, np.int32)
    for i in range(calls):
        n = min(step, block - i * step)
        for b in range(requests):
            slots[i, b * step:b * step + n] = pages[b] * block + i * step + np.arange(n)
    ds = dev(slots)
    es = raw[0][0][0].itemsize
    for i in range(calls):
        at = i * rows * kv * D * es
        ssd.ssd_kvq_append(c, p, ds.ptr + i * rows * 4, dk.ptr + at, dv.ptr + at)
        plain.append(slots[i], *(side[i][1].reshape(rows, kv, D) for side in raw))
        if i % 8 == 1 or i == calls - 1:
            assert_cache(arrs, plain)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,block,off", [(128, 64, 1), (128, 64, 5), (64, 128, 127), (128, 128, 66), (64, 32, 3), (128, 16, 15)])
def test_append_behind_small_tokens(dev, dtype, D, block, off):
    """One new token, one call a block, in many blocks whose older tokens have a far smaller scale."""
    rng = np.random.default_rng(block + off)
    kv, n_blocks = 16, 60
    c, arrs, plain = cache_arrays(dev, rng, n_blocks, kv, block, D)
    for a in arrs[2:]:
        upload(a, np.full((n_blocks, kv), 118, np.uint8))
    plain.ke[:], plain.ve[:] = 118, 118
    (k, kval), (v, vval) = (typed(rng.standard_normal((n_blocks, kv * D)) * 40.0, dtype) for _ in range(2))
    dk, dv, es = dev(k), dev(v), k.itemsize
    slots = (np.arange(n_blocks) * block + off).astype(np.int32)
    ds = dev(slots)
    p = ssd.ssd_kvq_append_params(code(dtype), 1, kv * D, kv * D)
    for i in range(n_blocks):
        ssd.ssd_kvq_append(c, p, ds.ptr + 4 * i, dk.ptr + i * kv * D * es, dv.ptr + i * kv * D * es)
    for i in range(n_blocks):
        plain.append(slots[i:i + 1], kval[i:i + 1].reshape(1, kv, D), vval[i:i + 1].reshape(1, kv, D))
    assert (plain.ve > 118).all()
    assert_cache(arrs, plain)


# ---------------------------------------------------------------- attention
def attend_case(dev, rng, dtype, heads, kv, D, block, reqs, width=None, extra=0, hide=(), max_q=None, max_len=None,
                q_scale=1.0, scale=None):
    """reqs: (len, rows) of every request.  Returns (got, want, tol) by row, and the arrays."""
    B = len(reqs)
    lens = np.array([r[0] for r in reqs], np.int32)
    cu = np.concatenate([[0], np.cumsum([r[1] for r in reqs])]).astype(np.int32)
    rows = int(cu[-1]) + 3  # three rows of no request
    need = [max(0, -(-int(x) // block)) for x in lens]
    W = width or max(1, max(need))
    n_blocks = sum(need) + 2
    c, arrs, plain = cache_arrays(dev, rng, n_blocks, kv, block, D)
    ids, at = rng.permutation(n_blocks).astype(np.int32), 0
    table = np.full((B, W), -1, np.int32)
    for b in range(B):
        n = min(need[b], W)
        table[b, :n] = ids[at:at + n]
        at += n
    for b, j, what in hide:
        table[b, j] = what
    ld = heads * D + extra
    raw, val = typed(rng.standard_normal((rows, ld)) * q_scale, dtype)
    q = val[:, :heads * D].reshape(rows, heads, D)
    mark, _ = typed(np.full((rows, ld), 77.0), dtype)
    scale = scale or D ** -0.5
    p = ssd.ssd_kvq_attn_params(code(dtype), B, rows, heads, max_q or max(1, max(r[1] for r in reqs)),
                                max_len or max(1, int(lens.max())), W, ld, ld, scale, 0)
    p.workspace_bytes = ssd.ssd_kvq_workspace(c, p)
    work = dev(np.full(max(16, p.workspace_bytes), 0xFF, np.uint8))  # NaN bit patterns
    dq, do = dev(raw), dev(mark)
    dcu, dl, dt = dev(cu), dev(lens), dev(table)
    ssd.ssd_kvq_attention(c, p, dq.ptr, dcu.ptr, dl.ptr, dt.ptr, do.ptr, work.ptr)
    got = values(do, dtype).reshape(rows, ld)
    assert (got[:, heads * D:] == 77.0).all()  # the gap between rows stays
    got = got[:, :heads * D].reshape(rows, heads, D)
    want, tol = S.attention(plain, q, cu, lens, table, scale, dtype == "bf16")
    return got, want, tol, (c, p, dq, dcu, dl, dt, do, work, table, lens, cu, plain, q)


def assert_attend(got, want, tol):
    none = np.isnan(want).all((1, 2))
    kept, nan = bool((got[none] == 77.0).all()), bool(np.isnan(got).any())
    assert kept and not nan  # rows of no request stay as they were
    over = np.abs(got - want) - tol
    at = np.unravel_index(np.nanargmax(over), over.shape)
    worst = float(over[at])
    assert worst <= 0, (worst, at, float(got[at]), float(want[at]), float(tol[at]))


ATTEND = [  # dtype, heads, kv, D, block, (len, rows) of every request
    ("bf16", 16, 16, 128, 32, [(412, 1)]),
    ("bf16", 8, 2, 128, 64, [(1, 1), (2, 1), (63, 1), (64, 1), (65, 1), (1000, 1), (0, 0), (257, 1)]),
    ("bf16", 32, 8, 128, 64, [(700, 24), (64, 64), (3, 3), (130, 0), (515, 5)]),
    ("f32", 4, 4, 64, 16, [(97, 33), (33, 33), (200, 1), (1100, 7)]),
    ("f32", 6, 2, 128, 128, [(300, 2), (129, 17)]),
    ("bf16", 4, 1, 64, 16, [(31, 16), (500, 65), (16, 1)]),
    ("bf16", 7, 1, 128, 128, [(2100, 3)]),
    ("f32", 3, 3, 64, 32, [(1, 1)]),
    ("bf16", 40, 2, 64, 64, [(150, 13), (77, 1)]),
    ("bf16", 8, 8, 128, 64, [(140, 130)]),
    ("f32", 8, 1, 128, 64, [(5000, 1), (17, 1), (4097, 1)])]


@pytest.mark.parametrize("dtype,heads,kv,D,block,reqs", ATTEND)
def test_attention(dev, dtype, heads, kv, D, block, reqs):
    rng = np.random.default_rng(heads + D + block)
    got, want, tol, _ = attend_case(dev, rng, dtype, heads, kv, D, block, reqs, extra=0)
    assert_attend(got, want, tol)


MANY = [  # heads, kv, D, block, table width, (len, rows) of every request, hidden entries, more
    # (wide tables and many requests: sizes at which the waves of a workgroup split the rows, 256 and 128 of them)
    (32, 8, 128, 64, 68, [(1500, 64), (903, 50), (0, 0), (64, 64), (3, 8), (705, 33), (129, 1), (1000, 40)], [], {}),
    (32, 8, 128, 64, 68, [(1400, 64), (900, 63), (0, 2), (65, 64), (448, 60), (705, 33), (130, 17), (3, 8)],
     [(0, 3, -1), (0, 22, 10 ** 6), (1, 0, -2 ** 31), (4, 6, -1)], dict(extra=3)),
    (32, 8, 128, 32, 128, [(1500, 80), (700, 66), (81, 80), (5, 1), (333, 40), (0, 0), (900, 8), (64, 70)],
     [(1, 2, -1)], dict(q_scale=60.0)),
    (32, 8, 64, 16, 272, [(1300, 64), (200, 50), (64, 64), (63, 64), (705, 33), (129, 1), (900, 40), (2, 2)],
     [(4, 0, -1), (4, 1, -1)], dict(extra=1, scale=-0.3)),
    (32, 8, 64, 128, 34, [(1200, 80), (900, 66), (128, 80), (5, 6), (333, 40), (0, 0), (900, 8), (64, 70)], [],
     dict(max_q=79)),
    (16, 16, 128, 64, 256, [(2600, 130), (131, 130), (700, 20)], [(0, 40, -1)], dict(max_len=9000)),
    (24, 8, 128, 128, 128, [(2000, 90), (91, 90), (1, 1)], [], dict(max_len=10 ** 9))]


@pytest.mark.parametrize("heads,kv,D,block,width,reqs,hide,more", MANY)
def test_attention_many_rows(dev, heads, kv, D, block, width, reqs, hide, more):
    rng = np.random.default_rng(heads + D + block)
    more = dict(dict(max_len=width * block), **more)
    got, want, tol, (c, p, dq, dcu, dl, dt, do, work, table, lens, *_) = attend_case(
        dev, rng, "bf16", heads, kv, D, block, reqs, width=width, hide=hide, **more)
    if "max_q" in more:  # rows past it are not computed
        at = 0
        for _, n in reqs:
            want[at + more["max_q"]:at + max(n, more["max_q"])] = np.nan
            at += n
    assert_attend(got, want, tol)
    # in place, with anything in the codes that no row sees
    k, v = dev.all[0].numpy().copy().reshape(c.n_blocks, kv, block, D), dev.all[1].numpy().copy().reshape(c.n_blocks, kv, D, block)
    ke, ve = dev.all[2].numpy().copy().reshape(c.n_blocks, kv), dev.all[3].numpy().copy().reshape(c.n_blocks, kv)
    used = {}
    for b, L in enumerate(lens):
        for j in range(min(width, -(-int(L) // block))):
            used[int(table[b, j])] = min(block, int(L) - block * j)
    for pg in range(c.n_blocks):
        n = used.get(pg, 0)
        k[pg, :, n:], v[pg, :, :, n:] = 0x7F, 0xFF
        if n == 0:
            ke[pg], ve[pg] = 255, 255
    for a, x in zip(dev.all[:4], (k, v, ke, ve)):
        upload(a, x)
    before = values(dq, "bf16").reshape(-1, p.ld_q)
    ssd.ssd_kvq_attention(c, p, dq.ptr, dcu.ptr, dl.ptr, dt.ptr, dq.ptr, work.ptr)
    after = values(dq, "bf16").reshape(-1, p.ld_q)
    none = np.isnan(want).all((1, 2))
    assert (after[none] == before[none]).all() and (after[:, heads * D:] == before[:, heads * D:]).all()
    assert np.array_equal(after[~none][:, :heads * D].reshape(-1, heads, D), got[~none])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_strides_and_wrong_hints(dev, dtype):
    """Rows with a gap, a max_len hint far too small and far too large."""
    for max_len in (1, 10 ** 9):
        rng = np.random.default_rng(8)
        got, want, tol, _ = attend_case(dev, rng, dtype, 8, 2, 128, 32, [(600, 9), (50, 1), (1500, 2)], extra=3, max_len=max_len)
        assert_attend(got, want, tol)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_rows_that_see_nothing(dev, dtype):
    """Rows before position 0, requests of length 0, hidden blocks, lengths past the table, rows past max_q."""
    rng = np.random.default_rng(9)
    got, want, tol, _ = attend_case(dev, rng, dtype, 4, 2, 64, 16, [(3, 8), (0, 2), (40, 3), (16, 2)],
                                    hide=[(2, 1, -1), (2, 0, 10 ** 6), (3, 0, -2 ** 31)])
    assert_attend(got, want, tol)
    assert not got[0:5].any() and not got[8:10].any()  # rows 0-4 sit before position 0, request 1 is empty
    # a table narrower than the length: positions past it are seen by none
    got, want, tol, _ = attend_case(dev, rng, dtype, 4, 2, 64, 16, [(100, 4), (20, 1)], width=3)
    assert_attend(got, want, tol)
    # rows past max_q are not computed
    got, want, tol, _ = attend_case(dev, rng, dtype, 4, 2, 64, 16, [(100, 6), (20, 1)], max_q=4)
    want[4:6] = np.nan
    assert_attend(got, want, tol)


def test_attention_bad_row_offsets(dev):
    """cu that leaves the array's rows: those rows are skipped."""
    rng = np.random.default_rng(10)
    _, _, _, (c, p, dq, dcu, dl, dt, do, work, table, lens, cu, plain, q) = attend_case(dev, rng, "f32", 4, 2, 64, 16,
                                                                                       [(30, 2), (30, 4)])
    for bad in ([-2, 2, 6], [0, 2, 10 ** 6], [5, 3, 200], [2 ** 31 - 1, -2 ** 31, 4]):
        upload(dcu, np.array(bad, np.int32))
        upload(do, np.full(q.size, 77.0, np.float32))
        ssd.ssd_kvq_attention(c, p, dq.ptr, dcu.ptr, dl.ptr, dt.ptr, do.ptr, work.ptr)
        got = values(do, "f32").reshape(q.shape)
        want, tol = S.attention(plain, q, [max(-10, min(x, 10 ** 4)) for x in bad], lens, table, 64 ** -0.5, False) \
            if bad[0] != 2 ** 31 - 1 else (None, None)
        if want is not None and bad[1] - bad[0] <= p.max_q and bad[2] - bad[1] <= p.max_q:
            assert_attend(got, want, tol)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_large_scores(dev, dtype):
    """Scores of thousands (one key takes nearly all the weight), a negative and a zero scale."""
    rng = np.random.default_rng(11)
    for kw in (dict(q_scale=60.0), dict(scale=-0.3), dict(scale=1e-30)):
        got, want, tol, _ = attend_case(dev, rng, dtype, 4, 2, 128, 64, [(333, 5), (90, 1)], **kw)
        assert_attend(got, want, tol)


def test_attention_in_place_and_stale_nan(dev):
    """out may be q; codes and exponents of positions past a request's length may hold anything."""
    rng = np.random.default_rng(12)
    got, want, tol, (c, p, dq, dcu, dl, dt, do, work, table, lens, cu, plain, q) = attend_case(
        dev, rng, "bf16", 8, 2, 64, 32, [(70, 5), (33, 1), (32, 2)])
    assert_attend(got, want, tol)
    k, v = (x.reshape(c.n_blocks, 2, 32, 64) for x in (dev.all[0].numpy(), dev.all[1].numpy()))
    k, v = k.copy(), v.reshape(c.n_blocks, 2, 64, 32).copy()
    ke, ve = dev.all[2].numpy().copy(), dev.all[3].numpy().copy()
    used = set()
    for b, L in enumerate(lens):
        for j in range(-(-int(L) // 32)):
            pg, n = table[b, j], min(32, int(L) - 32 * j)
            used.add(int(pg))
            k[pg, :, n:] = 0x7F
            v[pg, :, :, n:] = 0xFF
    for pg in set(range(c.n_blocks)) - used:
        k[pg], v[pg], ke[pg], ve[pg] = 0x7F, 0x7F, 255, 255
    for a, x in zip(dev.all[:4], (k, v, ke, ve)):
        upload(a, x)
    ssd.ssd_kvq_attention(c, p, dq.ptr, dcu.ptr, dl.ptr, dt.ptr, dq.ptr, work.ptr)
    again = values(dq, "bf16").reshape(q.shape)
    live = ~np.isnan(want).all((1, 2))
    assert np.array_equal(again[live], got[live])
    assert np.array_equal(again[~live], q[~live])


class Raw:
    """Device memory whose contents nobody reads before they are written."""

    def __init__(self, nbytes):
        p = ctypes.c_void_p()
        assert G.DeviceArray.hip().hipMalloc(ctypes.byref(p), nbytes) == 0
        self.ptr = p.value

    def put(self, at, host):
        host = np.ascontiguousarray(host)
        assert G.DeviceArray.hip().hipMemcpy(self.ptr + at, host.ctypes.data, host.nbytes, 1) == 0

    def get(self, at, shape, dtype):
        out = np.empty(shape, dtype)
        assert G.DeviceArray.hip().hipDeviceSynchronize() == 0
        assert G.DeviceArray.hip().hipMemcpy(out.ctypes.data, self.ptr + at, out.nbytes, 2) == 0
        return out

    def free(self):
        assert G.DeviceArray.hip().hipFree(self.ptr) == 0


@pytest.mark.parametrize("fresh,hint", [(1, 700), (64, 4352), (80, 4352)])
def test_offsets_past_32_bits(dev, fresh, hint):
    """Blocks behind the first 4 GiB of the codes, and rows of queries that far apart: the bits that a small cache and
    close rows give."""
    rng = np.random.default_rng(fresh)
    B, heads, kv, D, block, few = 8, 32, 8, 128, 128, 40
    many = 2 ** 32 // (kv * D * block) + few
    lens = np.array([fresh + int(x) for x in rng.integers(0, 500, B)], np.int32)
    width = -(-hint // block)
    need = [-(-int(x) // block) for x in lens]
    assert sum(need) <= few
    table, at = np.full((B, width), -1, np.int32), 0
    for b in range(B):
        table[b, :need[b]] = range(at, at + need[b])
        at += need[b]
    slots = np.concatenate([table[b, np.arange(x) // block] * block + np.arange(x) % block for b, x in enumerate(lens)])
    n, cols, rows = len(slots), kv * D, B * fresh
    k, _ = typed(rng.standard_normal((n, cols)), "bf16")
    v, _ = typed(rng.standard_normal((n, cols)), "bf16")
    q, _ = typed(rng.standard_normal((rows, heads * D)), "bf16")
    cu, dl, dk, dv = dev(np.arange(0, rows + 1, fresh).astype(np.int32)), dev(lens), dev(k), dev(v)
    outs, keep = [], []
    for blocks, shift, ld in ((few, 0, heads * D), (many, many - few, 2 ** 32 // (2 * (rows - 1)) // 8 * 8 + 64)):
        mem = [Raw(blocks * kv * block * D) for _ in range(2)] + [Raw(blocks * kv) for _ in range(2)] + [Raw(rows * ld * 2) for _ in range(2)]
        keep += mem
        c = ssd.ssd_kvq_cache(*[x.ptr for x in mem[:4]], blocks, block, kv, D)
        ssd.ssd_kvq_append(c, ssd.ssd_kvq_append_params(ssd.SSD_BF16, n, cols, cols), dev((slots + shift * block).astype(np.int32)).ptr,
                           dk.ptr, dv.ptr)
        for r in range(rows):
            mem[4].put(r * ld * 2, q[r])
        p = ssd.ssd_kvq_attn_params(ssd.SSD_BF16, B, rows, heads, fresh, hint, width, ld, ld, D ** -0.5, 0)
        p.workspace_bytes = ssd.ssd_kvq_workspace(c, p)
        work = dev(np.zeros(max(16, p.workspace_bytes), np.uint8))
        ssd.ssd_kvq_attention(c, p, mem[4].ptr, cu.ptr, dl.ptr, dev(np.where(table < 0, -1, table + shift).astype(np.int32)).ptr,
                              mem[5].ptr, work.ptr)
        outs.append([np.stack([mem[5].get(r * ld * 2, heads * D, np.uint16) for r in range(rows)])] +
                    [mem[i].get(shift * kv * block * D, few * kv * block * D, np.uint8).reshape(few, kv, -1)[:at] for i in range(2)] +
                    [mem[i].get(shift * kv, (few, kv), np.uint8)[:at] for i in (2, 3)])
    for x in keep:
        x.free()
    assert np.array_equal(outs[0][0], outs[1][0])
    full = np.zeros((at, block), bool)  # (codes behind a request's end were never written)
    full.reshape(-1)[slots] = True
    for i, tokens in ((1, lambda a: a.reshape(at, kv, block, D).transpose(0, 2, 1, 3)), (2, lambda a: a.reshape(at, kv, D, block).transpose(0, 3, 1, 2))):
        assert np.array_equal(tokens(outs[0][i])[full], tokens(outs[1][i])[full])
    assert np.array_equal(outs[0][3], outs[1][3]) and np.array_equal(outs[0][4], outs[1][4])


# ---------------------------------------------------------------- sampling
def run_sample(dev, logits, u, V, ld, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, rows=None):
    R = len(u)
    p = ssd.ssd_sample_params(vocab=V, ld=ld, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p)
    if rows:
        p.temperatures, p.top_ks, p.top_ps, p.min_ps = [dev(x).ptr for x in rows]
    tok, prob = dev(np.full(R, 99, np.int32)), dev(np.full(R, 99, np.float32))
    ssd.ssd_sample_logits(p, R, dev(logits).ptr, dev(np.asarray(u, np.float32)).ptr, tok.ptr, prob.ptr)
    return tok.numpy(), prob.numpy()


def check_sample(dev, logits, u, V, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, rows=None):
    tok, prob = run_sample(dev, logits, u, V, logits.shape[1], temperature, top_k, top_p, min_p, rows)
    for r in range(len(u)):
        T, k, tp, mp = [x[r] for x in rows] if rows else (temperature, top_k, top_p, min_p)
        want, wp = S.sample(logits[r, :V], float(np.float32(u[r])), float(T), int(k), float(tp), float(mp))
        assert tok[r] == want, (r, tok[r], want, T, k, tp, mp)
        # float64 throughout, weights to 2^-46 of the largest, one rounding to fp32
        assert abs(prob[r] - wp) <= wp * (2.0 ** -24 + V * 2.0 ** -45) + 1e-30


def logit_rows(rng, R, V, extra=0):
    x = rng.standard_normal((R, V + extra)) * rng.uniform(0.5, 3.0, (R, 1))
    x[np.arange(R), rng.integers(0, V, R)] += rng.uniform(0, 8, R)
    return x.astype(np.float32)


@pytest.mark.parametrize("V,extra", [(1, 0), (2, 5), (33, 0), (1000, 3), (1024, 0), (8192, 8), (16384, 0), (16387, 1),
                                     (32768, 0), (33001, 0), (65536, 0), (262144, 0)])
def test_sample(dev, V, extra):
    rng = np.random.default_rng(V)
    x = logit_rows(rng, 6, V, extra)
    u = rng.random(6)
    for kw in (dict(), dict(temperature=0.7, top_k=50), dict(top_p=0.9), dict(min_p=0.05, temperature=1.3),
               dict(top_k=max(1, V // 2), top_p=0.5, min_p=0.01), dict(temperature=0.0), dict(top_k=1), dict(top_p=0.0),
               dict(min_p=2.0), dict(top_k=V + 5, top_p=2.0, min_p=-1.0), dict(temperature=50.0, top_p=0.99)):
        check_sample(dev, x, u, V, **kw)


def test_sample_rows_of_their_own(dev):
    rng = np.random.default_rng(7)
    R, V = 200, 5000
    x = logit_rows(rng, R, V)
    rows = (rng.choice([0.0, 0.5, 1.0, 1.5, -1.0, np.nan, np.inf], R).astype(np.float32), rng.choice([0, 1, 7, 400, 4999, -3], R).astype(np.int32),
            rng.choice([1.0, 0.9, 0.3, 0.0, np.nan], R).astype(np.float32), rng.choice([0.0, 0.1, 1.0, np.nan], R).astype(np.float32))
    check_sample(dev, x, rng.random(R), V, rows=rows)


def test_sample_ties_and_special_values(dev):
    rng = np.random.default_rng(8)
    V = 6000
    x = np.zeros((18, V), np.float32)
    x[1] = np.where(rng.random(V) < 0.5, 1.0, 0.0)           # two values, thousands of ties each
    x[2] = np.round(rng.standard_normal(V) * 2) / 2           # a few values
    x[3] = -np.inf                                            # nothing to draw
    x[4] = np.nan
    x[5, ::3], x[5, 1::3] = np.nan, -np.inf
    x[6, 17] = np.inf
    x[7, [5, 99, 4000]] = np.inf                              # ties of the largest finite number
    x[8] = -np.inf
    x[8, 1234] = -3e38                                        # one code left
    x[9] = np.where(rng.random(V) < 0.5, 1e-45, 0.0)          # subnormal differences
    x[10] = rng.choice([3.4e38, -3.4e38, 0.0], V)
    x[11] = rng.standard_normal(V) * 1e-38
    x[12] = -np.exp2(-rng.integers(0, 140, V).astype(np.float64))   # many scales
    x[13] = np.linspace(-40, 0, V)                            # weights that vanish
    x[14] = -1e30
    x[15, :] = 5.0
    x[15, V - 1] = 5.0000005
    x[16] = np.where(np.arange(V) % 2, -0.0, 0.0)             # signed zeros are equal
    x[17] = rng.standard_normal(V)
    u = np.array([0.0, 0.5, 0.999, 0.3, 0.3, 0.7, 0.9, 0.5, 0.9, 0.2, 0.6, 0.4, 0.8, 0.99999994, 0.25, 0.5, 0.75, 0.1])
    for kw in (dict(), dict(top_k=1500), dict(top_k=2999), dict(top_p=0.37), dict(top_k=2000, top_p=0.61), dict(min_p=0.5),
               dict(temperature=3e38, top_k=2500), dict(temperature=1e-300, top_p=0.5), dict(temperature=0.0)):
        check_sample(dev, x, u, V, **kw)
    # uniforms at and outside the ends
    y = logit_rows(rng, 5, V)
    for top in (dict(), dict(top_p=0.8)):
        tok, _ = run_sample(dev, y, [1.0, 7.0, np.nan, -3.0, np.inf], V, V, **top)
        for r, uu in enumerate((1.0, 1.0, 0.0, 0.0, 1.0)):
            assert tok[r] == S.sample(y[r], uu, 1.0, 0, top.get("top_p", 1.0), 0.0)[0]


def test_sample_frequencies(dev):
    """Draws over a grid of uniforms fall on each code as often as its weight says (the inverse CDF is exact)."""
    V, R = 7, 4096
    l = np.array([0.3, -1.0, 2.0, 0.0, 1.0, -np.inf, 0.7], np.float32)
    x = np.tile(l, (R, 1))
    u = ((np.arange(R) + 0.5) / R).astype(np.float32)
    tok, _ = run_sample(dev, x, u, V, V)
    w = np.exp(l.astype(np.float64) - l.max())
    assert np.all(np.abs(np.bincount(tok, minlength=V) - R * w / w.sum()) <= 1.0)
    assert np.all(np.diff(tok) >= 0)


# ---------------------------------------------------------------- together
def step(rng, dev, cache, plain, heads, kv, D, block, dtype, held, fresh, table, pool, V):
    """One step of a server: lengths -> slots -> rotary -> append -> attention -> sampling; checks every stage."""
    B, n = len(held), int(sum(fresh))
    pad = n + 2
    W = table.shape[1]
    h, f, dp, dt = dev(np.array(held, np.int32)), dev(np.array(fresh, np.int32)), dev(pool), dev(table)
    lens, cu, slots, pos, used = (dev(np.zeros(x, np.int32)) for x in (B, B + 1, pad, pad, 1))
    ssd.ssd_kvq_slots(ssd.ssd_kvq_slot_params(B, block, W, len(pool), pad), h.ptr, f.ptr, dp.ptr, dt.ptr, lens.ptr, cu.ptr,
                      slots.ptr, pos.ptr, used.ptr)
    want = S.slots(held, fresh, pool, table, block, pad)
    C = (heads + 2 * kv) * D
    raw, val = typed(rng.standard_normal((pad, C)), dtype)
    axes = rng.integers(0, 100, (3, pad)).astype(np.int32)
    qkv, dpos = dev(raw), dev(axes)
    es = raw.itemsize
    rp = ssd.ssd_rope_params(n_heads=heads, n_kv_heads=kv, head_dim=D, dtype=code(dtype), n_axes=3, theta=1e4, ld_q=C, ld_k=C,
                             ld_q_out=C, ld_k_out=C)
    rp.section[0], rp.section[1], rp.section[2] = D // 8, 3 * D // 16, 3 * D // 16
    ka, va = qkv.ptr + heads * D * es, qkv.ptr + (heads + kv) * D * es
    ssd.ssd_rope_axes(rp, pad, qkv.ptr, ka, dpos.ptr, qkv.ptr, ka)
    ssd.ssd_kvq_append(cache, ssd.ssd_kvq_append_params(code(dtype), pad, C, C), slots.ptr, ka, va)
    p = ssd.ssd_kvq_attn_params(code(dtype), B, pad, heads, max(fresh), max(a + b for a, b in zip(held, fresh)), W, C, heads * D,
                                D ** -0.5, 0)
    p.workspace_bytes = ssd.ssd_kvq_workspace(cache, p)
    work, out = dev(np.zeros(max(16, p.workspace_bytes), np.uint8)), dev(np.zeros((pad, heads * D), raw.dtype))
    ssd.ssd_kvq_attention(cache, p, qkv.ptr, cu.ptr, lens.ptr, dt.ptr, out.ptr, work.ptr)
    u, tok = rng.random(pad).astype(np.float32), dev(np.zeros(pad, np.int32))
    logits = logit_rows(rng, pad, V)
    ssd.ssd_sample_logits(ssd.ssd_sample_params(vocab=V, ld=V, temperature=0.9, top_k=40, top_p=0.9, min_p=0.01), pad,
                          dev(logits).ptr, dev(u).ptr, tok.ptr)
    for name, a in (("table", dt), ("lens", lens), ("cu", cu), ("slots", slots), ("positions", pos), ("used", used)):
        assert np.array_equal(a.numpy(), want[name]), name
    # the rotated rows as the device holds them feed the plain cache and attention
    got = values(qkv, dtype).reshape(pad, C)
    x = val[:, :(heads + kv) * D].reshape(pad, heads + kv, D)
    turned = S.rope(x, axes, tuple(rp.section)[:3], 1e4)
    err = np.abs(got[:, :(heads + kv) * D].reshape(pad, heads + kv, D) - turned)
    worst = float((err - np.abs(turned) * (2.0 ** -8 if dtype == "bf16" else 0)).max())
    assert worst <= 2.0 ** -20 * np.abs(x).max()
    q, k, v = (y.reshape(pad, -1, D) for y in np.split(got, [heads * D, (heads + kv) * D], axis=1))
    plain.append(want["slots"], k, v)
    o, tol = S.attention(plain, q, want["cu"], want["lens"], want["table"], D ** -0.5, dtype == "bf16")
    go = values(out, dtype).reshape(pad, heads, D)
    worst = float((np.abs(go[:n] - o[:n]) - tol[:n]).max())
    assert worst <= 0 and not go[n:].any()
    assert list(tok.numpy()) == [S.sample(logits[r], float(u[r]), 0.9, 40, 0.9, 0.01)[0] for r in range(pad)]
    return want


@pytest.mark.parametrize("dtype,heads,kv,D,block", [("bf16", 8, 2, 128, 32), ("f32", 4, 4, 64, 16)])
def test_steps_of_a_server(dev, dtype, heads, kv, D, block):
    """A prefill step, decode steps, a verify round that is taken back and written again, and a request that ends."""
    rng = np.random.default_rng(5)
    n_blocks, W, B = 40, 8, 4
    cache, arrs, plain = cache_arrays(dev, rng, n_blocks, kv, block, D)
    free = rng.permutation(n_blocks).astype(np.int32)
    table, held = np.full((B, W), -1, np.int32), [0] * B
    for fresh, keep in (([37, 5, 70, 16], None), ([1, 1, 1, 1], None), ([9, 9, 0, 9], [2, 9, 0, 0]), ([4, 1, 9, 1], None)):
        want = step(rng, dev, cache, plain, heads, kv, D, block, dtype, held, fresh, table, free, 700)
        table, free = want["table"], free[int(want["used"][0]):]
        grown = keep or fresh
        for b in range(B):  # blocks that the kept tokens do not need go back
            have = -(-(held[b] + grown[b]) // block)
            back = [x for x in table[b, have:] if x >= 0]
            table[b, have:] = -1
            free = np.concatenate([np.array(back, np.int32), free])
        held = [a + b for a, b in zip(held, grown)]
    assert_cache(arrs, plain)


def test_captured_step_replays(dev):
    """slots -> append -> attention -> sampling on one stream, captured once and replayed on new inputs, with the
    eager calls between the replays."""
    hip = G.DeviceArray.hip()
    vp = ctypes.c_void_p
    stream, graph, exe = vp(), vp(), vp()
    assert hip.hipStreamCreate(ctypes.byref(stream)) == 0
    heads, kv, D, block, B, W, V = 8, 2, 128, 32, 5, 70, 3000
    rng = np.random.default_rng(6)
    c, arrs, plain = cache_arrays(dev, rng, B * W, kv, block, D)
    start = [a.numpy() for a in arrs]
    table = rng.permutation(B * W).astype(np.int32).reshape(B, W)
    held, fresh = rng.integers(1500, 2200, B).astype(np.int32), np.ones(B, np.int32)

    def inputs(i):
        r = np.random.default_rng(100 + i)
        return [S.bf16_bits(r.standard_normal((B, heads * D))), S.bf16_bits(r.standard_normal((B, kv * D))),
                S.bf16_bits(r.standard_normal((B, kv * D))), logit_rows(r, B, V), r.random(B).astype(np.float32)]

    ins = [dev(x) for x in inputs(0)]
    dh, df, dt = dev(held), dev(fresh), dev(table)
    lens, cu, slots, pos, used, tok = (dev(np.zeros(x, np.int32)) for x in (B, B + 1, B, B, 1, B))
    out = dev(np.zeros((B, heads * D), np.uint16))
    pa = ssd.ssd_kvq_append_params(ssd.SSD_BF16, B, kv * D, kv * D)
    p = ssd.ssd_kvq_attn_params(ssd.SSD_BF16, B, B, heads, 1, 2300, W, heads * D, heads * D, D ** -0.5, 0)
    p.workspace_bytes = ssd.ssd_kvq_workspace(c, p)
    work = dev(np.full(max(16, p.workspace_bytes), 0xFF, np.uint8))
    sp = ssd.ssd_kvq_slot_params(B, block, W, 0, B)
    ps = ssd.ssd_sample_params(vocab=V, ld=V, temperature=1.0, top_p=0.9)

    def load(i):
        for a, x in zip(ins, inputs(i)):
            upload(a, x)
        for a, x in zip(arrs, start):
            upload(a, x)
        upload(out, np.zeros((B, heads * D), np.uint16))

    def calls():
        q, k, v, logits, u = [a.ptr for a in ins]
        ssd.ssd_kvq_slots(sp, dh.ptr, df.ptr, None, dt.ptr, lens.ptr, cu.ptr, slots.ptr, pos.ptr, used.ptr, stream.value)
        ssd.ssd_kvq_append(c, pa, slots.ptr, k, v, stream.value)
        ssd.ssd_kvq_attention(c, p, q, cu.ptr, lens.ptr, dt.ptr, out.ptr, work.ptr, stream.value)
        ssd.ssd_sample_logits(ps, B, logits, u, tok.ptr, None, stream.value)

    def state():
        return [a.numpy() for a in (slots, out, tok, *arrs)]

    try:
        want = []
        for i in range(3):
            load(i)
            calls()
            want.append(state())
        assert not np.array_equal(want[0][1], want[1][1])
        assert hip.hipStreamBeginCapture(stream, 0) == 0
        calls()
        assert hip.hipStreamEndCapture(stream, ctypes.byref(graph)) == 0
        assert hip.hipGraphInstantiate(ctypes.byref(exe), graph, None, None, ctypes.c_size_t(0)) == 0
        for i in (2, 0, 1, 1):
            load(i)
            assert hip.hipGraphLaunch(exe, stream) == 0
            assert all(np.array_equal(a, b) for a, b in zip(state(), want[i])), i
            load((i + 1) % 3)
            calls()
            assert all(np.array_equal(a, b) for a, b in zip(state(), want[(i + 1) % 3])), i
    finally:
        if exe:
            hip.hipGraphExecDestroy(exe)
        if graph:
            hip.hipGraphDestroy(graph)
        hip.hipStreamDestroy(stream)


def test_two_streams_at_once(dev):
    """Two threads, each with a stream, arrays and a workspace of its own, on one card: what each gives alone."""
    hip = G.DeviceArray.hip()
    heads, kv, D, block, V = 32, 8, 128, 64, 20000
    streams = [ctypes.c_void_p() for _ in range(2)]
    calls, outs = [], []
    for i, reqs in enumerate(([(1500, 64), (903, 50), (64, 64), (705, 33), (1000, 40), (600, 64), (300, 60), (1200, 64)],
                              [(2000, 1), (900, 1), (3000, 1), (64, 1)])):
        assert hip.hipStreamCreate(ctypes.byref(streams[i])) == 0
        rng = np.random.default_rng(70 + i)
        _, _, _, (c, p, dq, dcu, dl, dt, do, work, *_) = attend_case(dev, rng, "bf16", heads, kv, D, block, reqs, width=68, max_len=4352)
        B, R = len(reqs), 6
        ps = ssd.ssd_sample_params(vocab=V, ld=V, temperature=1.0, top_k=500, top_p=0.9)
        logits, u = dev(logit_rows(rng, R, V)), dev(rng.random(R).astype(np.float32))
        tok, prob = dev(np.zeros(R, np.int32)), dev(np.zeros(R, np.float32))
        ps_rope = ssd.ssd_rope_params(heads, heads, D, ssd.SSD_BF16, 3, (16, 24, 24), p.ld_q, p.ld_out, p.ld_q, p.ld_q, 1e4)
        pos = dev(rng.integers(0, 5000, 3 * p.n_rows).astype(np.int32))
        qo, ko = dev(np.zeros((p.n_rows, p.ld_q), np.uint16)), dev(np.zeros((p.n_rows, p.ld_q), np.uint16))

        def call(c=c, p=p, a=(dq, dcu, dl, dt, do, work), ps=ps, b=(logits, u, tok, prob), pr=ps_rope, e=(pos, qo, ko), st=streams[i]):
            ssd.ssd_kvq_attention(c, p, *[x.ptr for x in a], st.value)
            ssd.ssd_rope_axes(pr, p.n_rows, a[0].ptr, a[4].ptr, *[x.ptr for x in e], st.value)
            ssd.ssd_sample_logits(ps, R, *[x.ptr for x in b], st.value)
        calls.append(call)
        outs.append((do, qo, ko, tok, prob))
    try:
        alone = []
        for f, o in zip(calls, outs):
            f()
            alone.append([x.numpy() for x in o])
        with ThreadPoolExecutor(2) as pool:
            for _ in range(3):
                list(pool.map(lambda f: [f() for _ in range(10)], calls))
                for o, want in zip(outs, alone):
                    assert all(np.array_equal(x.numpy(), w) for x, w in zip(o, want))
    finally:
        for st in streams:
            if st:
                hip.hipStreamDestroy(st)


def test_refused_arrays(dev):
    """Host memory, arrays that end early and misaligned ones are refused before any launch."""
    a = dev(np.zeros(64, np.int32))
    host = np.zeros(64, np.float32)
    lg = dev(np.zeros((2, 32), np.float32))
    p = ssd.ssd_sample_params(vocab=32, ld=32, temperature=1.0, top_p=1.0)
    for bad in ((2, host, lg.ptr, a.ptr), (3, lg.ptr, lg.ptr, a.ptr), (2, lg.ptr + 2, lg.ptr, a.ptr), (1, lg.ptr, host, a.ptr),
                (1, lg.ptr, lg.ptr, host)):
        with pytest.raises(ssd.SSDError) as e:
            ssd.ssd_sample_logits(p, *bad)
        assert e.value.status == ssd.SSD_E_INVAL and "array of the current device" in ssd.ssd_last_error()
    ssd.ssd_sample_logits(p, 2, lg.ptr, lg.ptr, a.ptr)
    rng = np.random.default_rng(1)
    c, arrs, _ = cache_arrays(dev, rng, 3, 2, 16, 64)
    rows = dev(np.zeros((4, 128), np.float32))
    ok = ssd.ssd_kvq_append_params(ssd.SSD_F32, 4, 128, 128)
    ssd.ssd_kvq_append(c, ok, a.ptr, rows.ptr, rows.ptr)
    c.n_blocks = 400000  # past the cache's arrays
    with pytest.raises(ssd.SSDError) as e:
        ssd.ssd_kvq_append(c, ok, a.ptr, rows.ptr, rows.ptr)
    assert e.value.status == ssd.SSD_E_INVAL and "cache k" in ssd.ssd_last_error()
