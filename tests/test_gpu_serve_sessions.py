"""The session side of the serving operators: sampling from a session's carry, rotary positions with several axes
in its passes (against the oracle with the same positions), and its cache handed to the 8-bit one."""
import dataclasses

import numpy as np
import pytest

import paper_2606_20543_amd as ssd
import synth
from oracle import decode as Dc
from oracle import model as M
from tests import gpu_util as G
from tests import serve_util as S

pytestmark = pytest.mark.gpu

BF16 = dataclasses.replace(synth.M1B, n_layers=2)
P, W = 16, 8


@pytest.fixture(scope="module", params=["f32", "bf16"])
def pair(request):
    p = G.Pair(synth.TINY if request.param == "f32" else BF16, gain_std=0.1)
    yield p
    p.close()


def grid_axes(n, t0):
    """Positions behind a prompt of t0 tokens on (time, height, width): a grid of W columns."""
    i = np.arange(n)
    return np.stack([np.full(n, t0), t0 + i // W, t0 + i % W]).astype(np.int32)


def sections(D):
    return (D // 8, 3 * D // 16, 3 * D // 16)


def axes_rope(axes, section):
    """oracle.model.rope with the positions behind the prompt looked up in axes [3][max_ctx - P]."""
    which = np.repeat(np.arange(len(section)), section)

    def rope(x, pos, inv_freq):
        half = x.shape[-1] // 2
        at = np.empty(pos.shape + (half,))
        for j in range(half):
            at[..., j] = np.where(pos < P, pos, axes[which[j]][np.maximum(pos - P, 0)])
        c, s = np.cos(at * inv_freq)[:, :, None, :], np.sin(at * inv_freq)[:, :, None, :]
        a, b = x[..., :half], x[..., half:]
        return np.concatenate([a * c - b * s, b * c + a * s], -1)
    return rope


def block(shape, B, K, seed):
    return (synth.random_codes(shape, (B, K), seed=seed) + shape.img_lo).astype(np.int32)


def test_session_axes_against_the_oracle(pair, monkeypatch):
    """A committed row and a verify round behind it; raster positions on all axes change nothing."""
    shape, B, K = pair.shape, 2, W
    n = 3 * W
    pre = synth.prompt(shape, B, P).astype(np.int32)
    axes, sec = grid_axes(n, P), sections(shape.head_dim)
    blocks = [block(shape, B, K, 1), block(shape, B, K, 2)]

    def run(prepare):
        sess = ssd.ssd_prefill(pair.model, B, P, pre, P + n, K)
        prepare(sess)
        a = G.gpu_verify(sess, shape, blocks[0], G.vparams(commit=1))["logits"]
        b = G.gpu_verify(sess, shape, blocks[1], G.vparams())["logits"]
        if prepare is grid:  # too late now
            with pytest.raises(ssd.SSDError) as e:
                ssd.ssd_session_set_axes(sess, sec, axes)
            assert e.value.status == ssd.SSD_E_STATE
        ssd.ssd_free_session(sess)
        return np.concatenate([a, b], 1)

    def grid(sess):
        ssd.ssd_session_set_axes(sess, sec, axes[::-1].copy())  # the next call replaces it
        ssd.ssd_session_set_axes(sess, sec, axes)

    def raster(sess):
        ssd.ssd_session_set_axes(sess, sec, np.tile(np.arange(P, P + n, dtype=np.int32), (3, 1)))

    plain, same, turned = run(lambda s: None), run(raster), run(grid)
    assert np.array_equal(plain, same)
    with monkeypatch.context() as m:
        m.setattr(M, "rope", axes_rope(axes, sec))
        os_ = Dc.prefill(pair.om, pre, P + n)
        want = []
        for i, blk in enumerate(blocks):
            lg, _ = M.forward(pair.om, os_.cache, blk, os_.f)
            want.append(lg)
            os_.f[:] += K
    want = np.concatenate(want, 1)
    tol = G.TOL[shape.dtype]
    assert float(np.abs(turned - want).max()) < tol
    assert float(np.abs(plain - want).max()) > 20 * tol  # the positions matter


def test_session_axes_refusals(pair):
    shape = pair.shape
    pre = synth.prompt(shape, 1, P).astype(np.int32)
    sess = ssd.ssd_prefill(pair.model, 1, P, pre, P + 4, 4)
    ok = np.zeros((3, 4), np.int32)
    half = shape.head_dim // 2
    for sec in ((half + 1, 0), (half, 1), (-1, half + 1), (), (1,) * 5):
        with pytest.raises(ssd.SSDError) as e:
            ssd.ssd_session_set_axes(sess, sec, ok)
        assert e.value.status == ssd.SSD_E_INVAL
    with pytest.raises(ssd.SSDError):
        ssd.ssd_session_set_axes(sess, (half,), None)
    ssd.ssd_session_set_axes(sess, (half,), ok)
    ssd.ssd_free_session(sess)


@pytest.mark.parametrize("guided", [False, True])
def test_session_sample(pair, guided):
    """The draws are those of the plain sampler on the session's own carry; a sampled decode of several tokens."""
    shape, B = pair.shape, 4
    pre = synth.prompt(shape, B, P).astype(np.int32)
    sess = ssd.ssd_prefill(pair.model, B, P, pre, P + 8, 1)
    n = B // 2 if guided else B
    if guided:
        ssd.ssd_session_set_cfg(sess, 3.0)
    rng = np.random.default_rng(1)
    p = ssd.ssd_sample_params(temperature=0.8, top_k=300, top_p=0.9, min_p=0.001)
    u, tok, prob = (G.DeviceArray(np.zeros(n, t)) for t in (np.float32, np.int32, np.float32))
    try:
        for _ in range(4):
            draw = rng.random(n).astype(np.float32)
            assert G.DeviceArray.hip().hipMemcpy(u.ptr, draw.ctypes.data, u.nbytes, 1) == 0
            carry = np.zeros((n, shape.v_img), np.float32)
            ssd.ssd_get_carry(sess, carry)
            ssd.ssd_session_sample(sess, p, u.ptr, tok.ptr, prob.ptr)
            got, gp = tok.numpy(), prob.numpy()
            for b in range(n):
                want, wp = S.sample(carry[b], float(draw[b]), 0.8, 300, 0.9, 0.001)
                assert got[b] == want + shape.img_lo and abs(gp[b] - wp) <= wp * 2.0 ** -23
            G.gpu_verify(sess, shape, got[:, None], G.vparams(commit=1))
        with pytest.raises(ssd.SSDError) as e:
            ssd.ssd_session_sample(sess, p, np.zeros(n, np.float32), tok.ptr)
        assert e.value.status == ssd.SSD_E_INVAL
        bad = ssd.ssd_sample_params(temperature=-1.0, top_p=1.0)
        with pytest.raises(ssd.SSDError):
            ssd.ssd_session_sample(sess, bad, u.ptr, tok.ptr)
    finally:
        for a in (u, tok, prob):
            a.free()
        ssd.ssd_free_session(sess)


def test_session_cache_as_rows_and_in_eight_bits(pair):
    """Every layer's cached rows against the oracle's cache, then slots, 8-bit cache and attention on them."""
    shape, B, block_ = pair.shape, 2, 32
    n_prompt = 37
    pre = synth.prompt(shape, B, n_prompt).astype(np.int32)
    sess = ssd.ssd_prefill(pair.model, B, n_prompt, pre, n_prompt + 8, 8)
    os_ = Dc.prefill(pair.om, pre, n_prompt + 8)
    blk = block(shape, B, 5, 3)
    G.gpu_verify(sess, shape, blk, G.vparams(commit=1))
    Dc.commit(os_, blk)
    n = n_prompt + 5
    kv, D, heads = shape.n_kv_heads, shape.head_dim, shape.n_heads
    bf16 = shape.dtype == "bf16"
    raw = np.uint16 if bf16 else np.float32
    arrs = [G.DeviceArray(np.zeros((B, n, kv, D), raw)) for _ in range(2)]
    try:
        for layer in range(shape.n_layers):
            ssd.ssd_session_read_kv(sess, layer, n, arrs[0].ptr, arrs[1].ptr)
            for a, want in zip(arrs, (os_.cache.k, os_.cache.v)):
                got = a.numpy()
                got = (S.bf16_value(got) if bf16 else got).astype(np.float64)
                w = want[layer, :, :, :n].swapaxes(1, 2)
                # one rounding of values that agree to the logits' tolerance: a step of bf16, or fp32 sums
                assert (np.abs(got - w) <= np.abs(w) * (2.0 ** -7 if bf16 else 0) + (1e-3 if bf16 else 1e-4)).all()
        # the prompt's rows of a shorter read are the same
        k_all = arrs[0].numpy()
        ssd.ssd_session_read_kv(sess, shape.n_layers - 1, 3, arrs[1].ptr, arrs[0].ptr)
        assert np.array_equal(arrs[1].numpy().reshape(-1)[:B * 3 * kv * D].reshape(B, 3, kv, D), k_all[:, :3])
        ssd.ssd_session_read_kv(sess, 0, n, arrs[0].ptr, arrs[1].ptr)
        k, v = ((S.bf16_value(a.numpy()) if bf16 else a.numpy()).astype(np.float64).reshape(B * n, kv, D) for a in arrs)
        dev = []

        def put(x):
            dev.append(G.DeviceArray(np.ascontiguousarray(x)))
            return dev[-1]
        Wd = -(-n // block_)
        held, fresh = np.zeros(B, np.int32), np.full(B, n, np.int32)
        pool, table = np.arange(B * Wd, dtype=np.int32)[::-1].copy(), np.full((B, Wd), -1, np.int32)
        dh, df, dp, dt = put(held), put(fresh), put(pool), put(table)
        lens, cu, slots, pos, used = (put(np.zeros(x, np.int32)) for x in (B, B + 1, B * n, B * n, 1))
        ssd.ssd_kvq_slots(ssd.ssd_kvq_slot_params(B, block_, Wd, len(pool), B * n), dh.ptr, df.ptr, dp.ptr, dt.ptr, lens.ptr, cu.ptr,
                          slots.ptr, pos.ptr, used.ptr)
        cache = [put(np.zeros((B * Wd, kv, block_, D), np.uint8)), put(np.zeros((B * Wd, kv, D, block_), np.uint8)),
                 put(np.zeros((B * Wd, kv), np.uint8)), put(np.zeros((B * Wd, kv), np.uint8))]
        c = ssd.ssd_kvq_cache(*[x.ptr for x in cache], B * Wd, block_, kv, D)
        dtype = ssd.SSD_BF16 if bf16 else ssd.SSD_F32
        ssd.ssd_kvq_append(c, ssd.ssd_kvq_append_params(dtype, B * n, kv * D, kv * D), slots.ptr, arrs[0].ptr, arrs[1].ptr)
        plain = S.Cache(B * Wd, kv, block_, D)
        plain.append(slots.numpy(), k, v)
        assert np.array_equal(S.E4M3[cache[0].numpy()], plain.k) and np.array_equal(cache[2].numpy(), plain.ke)
        rng = np.random.default_rng(2)
        q = rng.standard_normal((B, heads, D)).astype(np.float32)
        qraw = S.bf16_bits(q) if bf16 else q
        q = (S.bf16_value(qraw) if bf16 else q).astype(np.float64)
        p = ssd.ssd_kvq_attn_params(dtype, B, B, heads, 1, n, Wd, heads * D, heads * D, D ** -0.5, 0)
        p.workspace_bytes = ssd.ssd_kvq_workspace(c, p)
        work, out, cq = put(np.zeros(max(16, p.workspace_bytes), np.uint8)), put(np.zeros((B, heads, D), raw)), put(
            np.arange(B + 1, dtype=np.int32))
        ssd.ssd_kvq_attention(c, p, put(qraw).ptr, cq.ptr, lens.ptr, dt.ptr, out.ptr, work.ptr)
        got = out.numpy()
        got = (S.bf16_value(got) if bf16 else got).astype(np.float64)
        want, tol = S.attention(plain, q, np.arange(B + 1), lens.numpy(), dt.numpy(), D ** -0.5, bf16)
        assert float((np.abs(got - want) - tol).max()) <= 0
        # and near the attention over the unrounded rows: e4m3 keeps four significant bits
        for b in range(B):
            for h in range(heads):
                kk, vv = (x.reshape(B, n, kv, D)[b, :, h // (heads // kv)] for x in (k, v))
                s = kk @ q[b, h] / np.sqrt(D)
                w = np.exp(s - s.max())
                ref = (w / w.sum()) @ vv
                assert np.abs(got[b, h] - ref).max() <= 0.15 * np.abs(vv).max()
        for bad in ((-1, 1), (shape.n_layers, 1), (0, 0), (0, n + 1)):
            with pytest.raises(ssd.SSDError) as e:
                ssd.ssd_session_read_kv(sess, *bad, arrs[0].ptr, arrs[1].ptr)
            assert e.value.status == ssd.SSD_E_INVAL
        for a in dev:
            a.free()
    finally:
        for a in arrs:
            a.free()
        ssd.ssd_free_session(sess)


def test_session_calls_refuse_null(pair):
    L = ssd.lib()
    assert L.ssd_session_sample(None, None, None, None, None) == ssd.SSD_E_INVAL
    assert L.ssd_session_set_axes(None, 1, None, None) == ssd.SSD_E_INVAL
    assert L.ssd_session_read_kv(None, 0, 1, None, None) == ssd.SSD_E_INVAL
