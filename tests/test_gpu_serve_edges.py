"""The serving operators at the edges of what their calls allow: scores and magnitudes near the ends of fp32, row offsets
that leave the arrays, very many requests, unaligned outputs, errors that others left behind."""
import ctypes
import dataclasses

import numpy as np
import pytest

import paper_2606_20543_amd as ssd
import synth
from tests import gpu_util as G
from tests import serve_util as S
from tests.test_gpu_serve_ops import Dev, Raw, cache_arrays, code, slot_case, typed, upload, values

pytestmark = pytest.mark.gpu


@pytest.fixture
def dev():
    d = Dev()
    yield d
    d.free()


def attend(dev, c, dtype, q, cu, lens, table, scale, max_q=None, max_len=None, heads=None, in_place=False):
    """One call on rows of q [n][heads][D] as the device holds them; rows that it leaves alone hold 77."""
    n, heads, D = q.shape
    p = ssd.ssd_kvq_attn_params(code(dtype), len(lens), n, heads, max_q or max(1, int(np.diff(cu).max())),
                                max_len or max(1, int(max(lens))), table.shape[1], heads * D, heads * D, scale, 0)
    p.workspace_bytes = ssd.ssd_kvq_workspace(c, p)
    work = dev(np.full(max(16, p.workspace_bytes), 0xFF, np.uint8))  # NaN bit patterns
    out = dev(typed(np.full((n, heads, D), 77.0), dtype)[0])
    i32 = lambda x: dev(np.asarray(x, np.int32)).ptr  # noqa: E731
    ssd.ssd_kvq_attention(c, p, dev(q).ptr, i32(cu), i32(lens), i32(table), out.ptr, work.ptr)
    return values(out, dtype)


# dtype, heads, kv, D, block, table width, (len, rows) of every request, whether the hint is the table's width
# (a wide table splits the keys into shares; bf16 calls with many rows of many requests split the rows between waves)
EQUAL = [("f32", 4, 4, 64, 16, 20, [(300, 3), (1, 1), (65, 65)], False), ("f32", 8, 2, 128, 64, 90, [(500, 1), (90, 2)], True),
         ("bf16", 16, 16, 128, 32, 13, [(412, 1), (70, 3)], False), ("bf16", 8, 2, 64, 128, 60, [(1000, 1), (1, 1), (200, 20)], True),
         ("bf16", 32, 8, 128, 64, 68, [(400, 64), (100, 50), (64, 64), (3, 3), (305, 33), (129, 1), (500, 40), (80, 64)], True),
         ("bf16", 32, 8, 64, 16, 272, [(300, 64), (200, 50), (64, 64), (63, 63), (205, 33), (129, 1), (300, 40), (2, 2)], True)]


@pytest.mark.parametrize("dtype,heads,kv,D,block,width,reqs,wide", EQUAL)
@pytest.mark.parametrize("log2,negative", [(12, False), (21, False), (25, True), (28, False), (33, True), (66, False), (101, False),
                                           (126, False), (126, True)])
def test_attention_scores_of_any_size(dev, dtype, heads, kv, D, block, width, reqs, wide, log2, negative):
    """Keys of all ones or all minus ones under equal queries: scores +-1.5 2^log2, exact and equal but for their sign, the
    low ones first.  Of what a row sees, the larger scores share the weight: the mean of their values.

    Weights of equal scores are equal to fp32's roundings: the sums are off by (n + 16) 2^-24 of the magnitudes, fp16
    weights of bf16 calls by 2^-11, the result by its rounding."""
    rng = np.random.default_rng(log2 + D)
    B, lens = len(reqs), [r[0] for r in reqs]
    cu = np.concatenate([[0], np.cumsum([r[1] for r in reqs])])
    need = [-(-x // block) for x in lens]
    n_blocks = sum(need) + 1
    table, at, ids = np.full((B, width), -1, np.int32), 0, rng.permutation(n_blocks)
    for b in range(B):
        table[b, :need[b]] = ids[at:at + need[b]]
        at += need[b]
    c, arrs, plain = cache_arrays(dev, rng, n_blocks, kv, block, D)
    low = [np.concatenate([np.ones(min(70, x // 2 + 1), bool), rng.random(max(0, x - min(70, x // 2 + 1))) < 0.5]) for x in lens]
    k = np.full((n_blocks, kv, block, D), 0x38, np.uint8)  # 1
    for b in range(B):
        for p in np.nonzero(low[b])[0]:
            k[table[b, p // block], :, p % block] = 0xB8
    e = log2 // 2
    upload(arrs[0], k)
    upload(arrs[2], np.full((n_blocks, kv), 127 + e, np.uint8))
    q = typed(np.full((int(cu[-1]), heads, D), (-1.5 if negative else 1.5) * 2.0 ** (log2 - e - D.bit_length() + 1)), dtype)[0]
    # (scale 1: 1.5 2^(log2 - e) / D, D times, by 2^e; a negative scale gives the same scores)
    got = attend(dev, c, dtype, q, cu, lens, table, -1.0 if negative else 1.0, max_len=width * block if wide else None)
    g, u = heads // kv, 2.0 ** -24
    V = plain.v * np.exp2(plain.ve - 127.0)[:, :, None, None]  # [blocks][kv][block][D]
    for b in range(B):
        pg, at = table[b, np.arange(lens[b]) // block], np.arange(lens[b]) % block
        for i in range(reqs[b][1]):
            seen = np.arange(lens[b]) <= lens[b] - reqs[b][1] + i
            most = seen & ~low[b] if (seen & ~low[b]).any() else seen
            v = V[pg[most], :, at[most]]  # [n][kv][D]
            want, mag = (np.repeat(x.mean(0), g, 0) for x in (v, np.abs(v)))
            tol = mag * ((lens[b] + 16) * u + (2.0 ** -11 if dtype == "bf16" else 0)) + np.abs(want) * (2.0 ** -8 if dtype == "bf16" else 0)
            worst = float((np.abs(got[cu[b] + i] - want) - tol).max())
            assert worst <= 0, (b, i, worst)


@pytest.mark.parametrize("dtype,heads,kv,D,block,width,reqs,wide", EQUAL)
@pytest.mark.parametrize("scale,q_scale", [(0.0, 1.0), (-0.0, 1e34), (0.0, 1e34), (1e-40, 1e34), (-1e-42, 1e36), (2e-45, 1e3)])
def test_attention_tiny_scales(dev, dtype, heads, kv, D, block, width, reqs, wide, scale, q_scale):
    """A scale of zero gives every seen key the same weight, one below fp32's normal range its own; hidden blocks stay hidden."""
    rng = np.random.default_rng(D + block)
    B, lens = len(reqs), [r[0] for r in reqs]
    cu = np.concatenate([[0], np.cumsum([r[1] for r in reqs])])
    need = [-(-x // block) for x in lens]
    c, arrs, plain = cache_arrays(dev, rng, sum(need) + 1, kv, block, D)
    table, at, ids = np.full((B, width), -1, np.int32), 0, rng.permutation(sum(need) + 1)
    for b in range(B):
        table[b, :need[b]] = ids[at:at + need[b]]
        at += need[b]
    table[0, need[0] // 2] = -1
    table[B - 1, 0] = 10 ** 6
    q, val = typed(rng.standard_normal((int(cu[-1]), heads, D)) * q_scale, dtype)
    got = attend(dev, c, dtype, q, cu, lens, table, scale, max_len=width * block if wide else None)
    want, tol = S.attention(plain, val, cu, lens, table, scale, dtype == "bf16")
    # the scale (its product with log2 e) is one of fp32: off by at most a step of 2^-149 below the normal range, and so
    # scores by that times q.k; exp of that less one, twice, of sum p |v|, which is at most the largest |v|
    top = 448.0 * np.exp2(plain.ve.max() - 127.0)
    qk = np.abs(val).sum(2).max() * np.abs(plain.k * np.exp2(plain.ke - 127.0)[:, :, None, None]).max()
    d = qk * (2.0 ** -148 if abs(scale) < 2.0 ** -126 else 0)
    assert d < 1e-3
    worst = float((np.abs(got - want) - tol - 4 * d * top).max())
    assert worst <= 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cu,max_q", [([-2, 2, 6], 4), ([0, 2, 10 ** 6], 4), ([5, 3, 200], 4), ([2 ** 31 - 1, -2 ** 31, 4], 4),
                                      ([0, 9, 9], 4), ([9, 12, 9], 4), ([7, 11, 20], 20), ([-5, -1, 3], 20), ([2, 2, 2], 1)])
def test_attention_row_offsets_anywhere(dev, dtype, cu, max_q):
    """Rows that cu puts outside the array are skipped, rows past max_q are not computed, and no other row is written."""
    rng = np.random.default_rng(10)
    heads, kv, D, block, rows = 4, 2, 64, 16, 9
    c, arrs, plain = cache_arrays(dev, rng, 5, kv, block, D)
    table, lens = np.array([[3, 1], [0, 4]], np.int32), [30, 25]
    q, val = typed(rng.standard_normal((rows, heads, D)), dtype)
    got = attend(dev, c, dtype, q, cu, lens, table, 0.125, max_q=max_q)
    want, tol = np.full(q.shape, np.nan), np.zeros(q.shape)
    for b in range(2):
        n = cu[b + 1] - cu[b]
        if not 0 < n < 2 ** 24:  # (2^32: all of its first rows lie before the array)
            continue
        w, t = S.attention(plain, val, [cu[b], cu[b + 1]], lens[b:b + 1], table[b:b + 1], 0.125, dtype == "bf16")
        for r in range(max(0, cu[b]), min(rows, cu[b + 1], cu[b] + max_q)):
            want[r], tol[r] = w[r], t[r]
    none = np.isnan(want)
    assert (got[none] == 77.0).all()
    assert (np.abs(got - want) <= tol)[~none].all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D,rows,off", [(64, 5, 0), (128, 1, 0), (128, 16, 0), (64, 3, 8)])
def test_append_and_read_the_largest_magnitudes(dev, dtype, D, rows, off):
    """Magnitudes to the end of fp32 (bf16): an exponent of 247, where codes above 240 would stand for more than the type
    holds.  Values and infinities end at 240, and the attention over them is finite."""
    rng = np.random.default_rng(D + rows)
    kv, block = 6, 16
    c, arrs, plain = cache_arrays(dev, rng, 3, kv, block, D)
    x = rng.standard_normal((rows, kv, D))
    big = np.float32(3.3895313892515355e38)  # the largest bf16
    x[:, 0] *= 1e37
    x[:, 1] = np.where(rng.random((rows, D)) < 0.3, big, x[:, 1])
    x[:, 2] = np.where(rng.random((rows, D)) < 0.3, -big, np.clip(x[:, 2] * 2.5e37, -1e38, 1e38))
    x[:, 3] = np.where(rng.random((rows, D)) < 0.3, np.inf, np.clip(x[:, 3] * 2e38, -big, big))
    x[:, 4] = np.resize(np.array([2.0 ** 127 * 1.75, 2.0 ** 127 * 1.6, -2.0 ** 127, 3e38]), (rows, D))
    x[:, 5] = np.resize(np.array([2.0 ** 127 * 1.765625, -np.inf, 2.0 ** 127 * 1.9375, 2.0 ** 127 * 1.875, 2.0 ** 127 * 1.8125]), (rows, D))
    x[0, 1:3, 0] = big
    x = x.astype(np.float32)
    if dtype == "f32":
        x[0, 1, 1] = np.finfo(np.float32).max
    raw, val = typed(x, dtype)
    slots = (block + off + np.arange(rows)).astype(np.int32)
    dk, dv = dev(raw), dev(raw[:, ::-1].copy())
    ssd.ssd_kvq_append(c, ssd.ssd_kvq_append_params(code(dtype), rows, kv * D, kv * D), dev(slots).ptr, dk.ptr, dv.ptr)
    k, v, ke, ve = [a.numpy() for a in arrs]
    for h in range(kv):
        for codes, exps, head, old in ((S.E4M3[k[1, h, off:off + rows]], ke, h, plain.ke), (S.E4M3[v[1, h]].T[off:off + rows], ve, kv - 1 - h, plain.ve)):
            y = val[:, head]
            s = max(S.exponent(np.abs(y[np.isfinite(y)]).max()), old[1, h] if off else 1)
            assert exps[1, h] == s
            top = 240.0 if s == 247 else 448.0
            assert np.array_equal(codes, S.e4m3_round(np.clip(y * 2.0 ** (127 - s), -top, top)))
    stands = np.abs(S.E4M3[k[1]][:, off:off + rows] * np.exp2(ke[1] - 127.0)[:, None, None]).max()
    assert (ke[1] == 247).any() and stands <= big
    if off:
        return
    # The attention that sees the first token returns its values.  (Sums are fp32, and 2 * 240 * 2^120 is past it: a row that
    # sees several such values has no finite sum.)
    q = typed(np.zeros((1, kv, D)), dtype)[0]
    got = attend(dev, c, dtype, q, [0, 1], [1], np.array([[1]]), 1.0)
    want = (S.E4M3[v[1]][:, :, 0] * np.exp2(ve[1] - 127.0)[:, None])[None]
    worst = float((np.abs(got - want) - np.abs(want) * (2.0 ** -8 + 2.0 ** -11 + 32 * 2.0 ** -24)).max())
    assert worst <= 0


def slots_of(held, fresh, pool, table, block, n_rows):
    """tests/serve_util.py's slots without loops over requests; lengths and positions end at the largest int32."""
    top = 2 ** 31 - 1
    B, W = table.shape
    held, fresh = np.maximum(held.astype(np.int64), 0), np.maximum(fresh.astype(np.int64), 0)
    lens = held + fresh
    have, want = np.minimum(-(-held // block), W), np.minimum(-(-lens // block), W)
    take = want - have
    start, cu = np.cumsum(take) - take, np.concatenate([[0], np.cumsum(fresh)])
    total = int(take.sum())
    served = np.concatenate([pool.astype(np.int64), np.full(max(0, total - len(pool)), -1)])
    table = table.copy()
    b = np.repeat(np.arange(B), take)
    table[b, have[b] + np.arange(total) - start[b]] = served[:total]
    n = min(n_rows, int(cu[-1]))
    slots, positions = np.full(n_rows, -1, np.int64), np.full(n_rows, -1, np.int64)
    b = np.searchsorted(cu[1:], np.arange(n), side="right")
    p = held[b] + np.arange(n) - cu[b]
    page = np.where(p // block < W, table[b, np.minimum(p // block, W - 1)], -1)
    positions[:n] = np.minimum(p, top)
    slots[:n] = np.where(page >= 0, page.astype(np.int64) * block + p % block, -1)
    return dict(table=table, lens=np.minimum(lens, top), cu=np.minimum(cu, top), slots=slots, positions=positions,
                used=np.array([total]))


MANY_REQUESTS = [  # B, block, width, held, fresh, short of blocks, padded rows, rows cut
    (2049, 16, 6, 90, 2, 0, 5, 0), (4097, 32, 3, 60, 5, 40, 0, 17), (8192, 16, 5, 90, 2, 0, 5, 0),
                 (8193, 16, 5, 90, 2, 30, 0, 5), (10000, 128, 2, 200, 90, 0, 3000, 0), (33333, 64, 4, 300, 1, 0, 0, 0),
    (100000, 16, 5, 70, 3, 1000, 9, 0), (262144, 32, 2, 30, 1, 0, 0, 100), (2 ** 20 - 1, 16, 3, 40, 1, 0, 1, 0), (2 ** 20, 16, 2, 30, 2, 9, 0, 0)]


@pytest.mark.parametrize("B,block,width,held,fresh,short,pad,cut", MANY_REQUESTS)
def test_slots_of_many_requests(dev, B, block, width, held, fresh, short, pad, cut):
    rng = np.random.default_rng(B + block)
    h, f, pool, table, n = slot_case(rng, B, block, width, held, fresh, short, pad, cut)
    h[3], f[4] = -5, -2  # count as 0
    table[3] = np.maximum(table[3], 0)
    f[B // 2] = 900  # a prompt among them, past the table's width
    n += 900
    if B < 5000:
        want = slots_of(h, f, pool, table, block, n)
        for name, w in S.slots(h, f, pool, table, block, n).items():
            assert np.array_equal(want[name], w), name
    h[rng.integers(0, B, 9)] = 2 ** 31 - 1
    want = slots_of(h, f, pool, table, block, n)
    p = ssd.ssd_kvq_slot_params(B, block, width, len(pool), n)
    ins = [dev(x) for x in (h, f, pool)]
    t = dev(table)
    outs = [dev(np.full(max(1, x), 99, np.int32)) for x in (B, B + 1, n, n, 1)]
    for _ in range(2):  # again: the same
        ssd.ssd_kvq_slots(p, *[x.ptr for x in ins], t.ptr, *[x.ptr for x in outs])
        for name, a in zip(("table", "lens", "cu", "slots", "positions", "used"), [t] + outs):
            w = want[name].reshape(-1)
            assert np.array_equal(a.numpy().reshape(-1)[:w.size], w), name


def test_slots_time_grows_with_the_requests(dev):
    """2^20 single tokens: a few passes over some 20 MB.  Summing all lengths in every workgroup took 4 TB of reads."""
    hip = G.DeviceArray.hip()
    B = 2 ** 20
    h, f = dev(np.full(B, 15, np.int32)), dev(np.full(B, 2, np.int32))
    pool, table = dev(np.arange(B, dtype=np.int32)), dev(np.zeros((B, 2), np.int32))
    outs = [dev(np.zeros(x, np.int32)) for x in (B, B + 1, 2 * B, 2 * B, 1)]
    p = ssd.ssd_kvq_slot_params(B, 16, 2, B, 2 * B)
    start, stop = ctypes.c_void_p(), ctypes.c_void_p()
    assert hip.hipEventCreate(ctypes.byref(start)) == 0 and hip.hipEventCreate(ctypes.byref(stop)) == 0
    ms = ctypes.c_float()
    for _ in range(2):
        assert hip.hipEventRecord(start, None) == 0
        ssd.ssd_kvq_slots(p, h.ptr, f.ptr, pool.ptr, table.ptr, *[x.ptr for x in outs])
        assert hip.hipEventRecord(stop, None) == 0 and hip.hipEventSynchronize(stop) == 0
        assert hip.hipEventElapsedTime(ctypes.byref(ms), start, stop) == 0
    hip.hipEventDestroy(start), hip.hipEventDestroy(stop)
    assert outs[4].numpy()[0] == B
    assert ms.value < 20.0  # (some 0.1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_session_rows_at_any_element(dtype):
    """A layer's cached rows into arrays that start on an element, not on 16 bytes: the rows an aligned array gets, and
    nothing around them."""
    shape = synth.TINY if dtype == "f32" else dataclasses.replace(synth.M1B, n_layers=2)
    pair = G.Pair(shape, oracle=False)
    B, P = 3, 19
    sess = ssd.ssd_prefill(pair.model, B, P, synth.prompt(shape, B, P).astype(np.int32), P + 4, 4)
    raw = np.uint16 if dtype == "bf16" else np.float32
    n = B * P * shape.n_kv_heads * shape.head_dim
    aligned = [G.DeviceArray(np.zeros(n, raw)) for _ in range(2)]
    odd = [G.DeviceArray(np.full(n + 16, 3, raw)) for _ in range(2)]
    try:
        ssd.ssd_session_read_kv(sess, 1, P, aligned[0].ptr, aligned[1].ptr)
        for ka, va in ((1, 3), (0, 5), (7, 8)):
            for a in odd:
                upload(a, np.full(n + 16, 3, raw))
            es = np.dtype(raw).itemsize
            ssd.ssd_session_read_kv(sess, 1, P, odd[0].ptr + ka * es, odd[1].ptr + va * es)
            for a, want, at in zip(odd, aligned, (ka, va)):
                got = a.numpy()
                assert np.array_equal(got[at:at + n], want.numpy())
                assert (got[:at] == 3).all() and (got[at + n:] == 3).all()
        with pytest.raises(ssd.SSDError) as e:  # inside an element
            ssd.ssd_session_read_kv(sess, 1, P, odd[0].ptr + 1, odd[1].ptr)
        assert e.value.status == ssd.SSD_E_INVAL
    finally:
        for a in aligned + odd:
            a.free()
        ssd.ssd_free_session(sess)
        pair.close()


def test_an_error_of_an_earlier_call_is_not_this_ones(dev):
    """An error that other code of the thread left behind (a copy that the runtime refused) does not fail a call that works."""
    hip = G.DeviceArray.hip()
    rng = np.random.default_rng(4)
    c, arrs, plain = cache_arrays(dev, rng, 3, 2, 16, 64)
    rows, ints, out = dev(np.ones((4, 128), np.float32)), dev(np.arange(16, dtype=np.int32)), dev(np.zeros((4, 128), np.float32))
    i32 = [dev(np.zeros(16, np.int32)) for _ in range(6)]
    rope = ssd.ssd_rope_params(2, 2, 64, ssd.SSD_F32, 1, (32,), 128, 128, 128, 128, 1e4)
    attn = ssd.ssd_kvq_attn_params(ssd.SSD_F32, 1, 4, 2, 1, 16, 1, 128, 128, 0.125, 0)
    calls = [lambda: ssd.ssd_kvq_slots(ssd.ssd_kvq_slot_params(2, 16, 2, 4, 4), ints.ptr, ints.ptr, ints.ptr, *[x.ptr for x in i32]),
             lambda: ssd.ssd_rope_axes(rope, 4, rows.ptr, rows.ptr, ints.ptr, out.ptr, arrs[0].ptr),
             lambda: ssd.ssd_kvq_append(c, ssd.ssd_kvq_append_params(ssd.SSD_F32, 4, 128, 128), ints.ptr, rows.ptr, rows.ptr),
             lambda: ssd.ssd_kvq_attention(c, attn, rows.ptr, ints.ptr, ints.ptr, i32[0].ptr, out.ptr),
             lambda: ssd.ssd_sample_logits(ssd.ssd_sample_params(vocab=128, ld=128, temperature=1.0, top_p=1.0), 4, rows.ptr, rows.ptr, ints.ptr)]
    shape = synth.TINY
    pair = G.Pair(shape, oracle=False)
    sess = ssd.ssd_prefill(pair.model, 1, 5, synth.prompt(shape, 1, 5).astype(np.int32), 9, 4)
    axes = dev(np.zeros((2, 4), np.int32))
    row = dev(np.zeros((2, 5 * shape.n_kv_heads * shape.head_dim), np.float32))
    half = shape.head_dim // 4
    calls += [lambda: ssd.ssd_session_set_axes(sess, (half, half), axes.ptr),
              lambda: ssd.ssd_session_sample(sess, ssd.ssd_sample_params(temperature=1.0, top_p=1.0), rows.ptr, ints.ptr),
              lambda: ssd.ssd_session_read_kv(sess, 0, 5, row.ptr, row.ptr + row.nbytes // 2)]
    try:
        for call in calls:
            assert hip.hipMemcpy(None, None, 16, 1) != 0
            call()
        assert hip.hipDeviceSynchronize() == 0
    finally:
        hip.hipGetLastError()
        ssd.ssd_free_session(sess)
        pair.close()


@pytest.mark.parametrize("width,hint", [(4, None), (90, 5000)])
def test_attention_largest_queries(dev, width, hint):
    """fp32 queries past the largest bf16 (255 2^120), keys small enough that scores stay ordinary: the three operands of a
    query carry all of its bits."""
    rng = np.random.default_rng(21)
    heads, kv, D, block, L = 4, 2, 64, 64, 150
    c, arrs, plain = cache_arrays(dev, rng, 4, kv, block, D)
    upload(arrs[2], np.full((4, kv), 5, np.uint8))  # keys of some 2^-115
    plain.ke[:] = 5
    q = (rng.standard_normal((3, heads, D)) * 1e37).astype(np.float32)
    top = np.finfo(np.float32).max
    q[0, :, 3], q[1, :, 7], q[2, 0, 60] = top, -top, np.nextafter(np.float32(3.3953e38), np.float32(np.inf))
    table = np.full((1, width), -1, np.int32)
    table[0, :3] = [2, 0, 3]
    got = attend(dev, c, "f32", q, [0, 3], [L], table, 2.0 ** -8, max_len=hint)
    want, tol = S.attention(plain, q.astype(np.float64), [0, 3], [L], table, 2.0 ** -8, False)
    assert float((np.abs(got - want) - tol).max()) <= 0


def test_rope_of_the_most_tokens(dev):
    """2^25 - 1 tokens of heads of 684: the launch holds them (92 GB, in place); the first, the last and some rows between."""
    T, D = 2 ** 25 - 1, 684
    rng = np.random.default_rng(22)
    x, val = typed(rng.standard_normal((2, 1, 1, D)), "bf16")
    pos = np.zeros((1, T), np.int32)
    at = [0, 1, 2, 3, 4, T // 2, T - 4, T - 3, T - 2, T - 1]
    pos[0, at] = [0, 5, 17, 4000, 3, 99999, 12, 7, 2 ** 31 - 1, 1234]
    p = ssd.ssd_rope_params(1, 1, D, ssd.SSD_BF16, 1, (D // 2,), D, D, D, D, 1e4)
    dp, mem = dev(pos), []
    try:
        for side in x:
            mem.append(Raw(T * D * 2))
            for t in at:
                mem[-1].put(t * D * 2, side)
        ssd.ssd_rope_axes(p, T, mem[0].ptr, mem[1].ptr, dp.ptr, mem[0].ptr, mem[1].ptr)
        for side, m in zip(val, mem):
            for t in at:
                want = S.rope(side, pos[:, t:t + 1], (D // 2,), 1e4)
                got = S.bf16_value(m.get(t * D * 2, (1, 1, D), np.uint16)).astype(np.float64)
                size = np.abs(side) + np.abs(np.roll(side, D // 2, -1))
                assert (np.abs(got - want) <= size * (6 * 2.0 ** -24 + 2.0 ** 31 * 2.0 ** -50) + np.abs(want) * 2.0 ** -8).all(), t
    finally:
        for m in mem:
            m.free()
