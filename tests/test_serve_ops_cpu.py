"""The serving operators without a GPU: struct layouts, the refusals that need no device, and the plain
implementations that their GPU tests compare with (against closed forms)."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import paper_2606_20543_amd as ssd
from tests import serve_util as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STRUCTS = (ssd.ssd_kvq_cache, ssd.ssd_kvq_slot_params, ssd.ssd_rope_params, ssd.ssd_kvq_append_params, ssd.ssd_kvq_attn_params,
           ssd.ssd_sample_params)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(ssd.LIB_PATH):
        from paper_2606_20543_amd import _build
        _build.build()
    return ssd.lib()


def test_struct_layouts_match_header(tmp_path):
    lines = []
    for s in STRUCTS:
        lines.append(f'printf("%zu\\n", sizeof({s.__name__}));')
        lines += [f'printf("%zu\\n", offsetof({s.__name__}, {f[0]}));' for f in s._fields_]
    src = tmp_path / "layout.c"
    src.write_text(f'#include <stdio.h>\n#include <stddef.h>\n#include "{ROOT}/include/ssd.h"\nint main(void) {{\n' +
                   "\n".join(lines) + "\nreturn 0;\n}\n")
    exe = tmp_path / "layout"
    subprocess.check_call(["gcc", str(src), "-o", str(exe)])
    got = [int(x) for x in subprocess.check_output([str(exe)]).decode().split()]
    want = []
    for s in STRUCTS:
        want += [ctypes.sizeof(s)] + [getattr(s, f[0]).offset for f in s._fields_]
    assert got == want


def refused(fn, args, word):
    with pytest.raises(ssd.SSDError) as e:
        fn(*args)
    assert e.value.status == ssd.SSD_E_INVAL and word in ssd.ssd_last_error(), ssd.ssd_last_error()


def change(s, **kw):
    t = type(s).from_buffer_copy(s)
    for k, v in kw.items():
        if k == "section":
            for i, x in enumerate(v):
                t.section[i] = x
        else:
            setattr(t, k, v)
    return t


X = 0x1000  # an address that no call may reach


def test_slots_refusals(lib):
    p = ssd.ssd_kvq_slot_params(4, 16, 8, 10, 20)
    a = [X] * 9
    for kw in (dict(block=0), dict(block=24), dict(block=256), dict(n_seqs=0), dict(table_width=0), dict(n_pool=-1), dict(n_rows=-1)):
        refused(ssd.ssd_kvq_slots, [change(p, **kw)] + a, "block =" if "block" in kw else "must be positive")
    refused(ssd.ssd_kvq_slots, [change(p, n_seqs=2 ** 20 + 1)] + a, "2^20")
    for i in range(9):
        refused(ssd.ssd_kvq_slots, [p] + a[:i] + [None] + a[i + 1:], "NULL")
    assert lib.ssd_kvq_slots(None, *[None] * 10) == ssd.SSD_E_INVAL


def test_rope_refusals(lib):
    p = ssd.ssd_rope_params(n_heads=4, n_kv_heads=2, head_dim=64, dtype=ssd.SSD_BF16, n_axes=3, ld_q=256, ld_k=128, ld_q_out=256,
                            ld_k_out=128, theta=1e4)
    p.section[0], p.section[1], p.section[2] = 8, 12, 12
    a = [X] * 5
    for kw, word in ((dict(dtype=7), "dtype"), (dict(n_heads=0), "n_heads"), (dict(n_kv_heads=-1), "n_heads"),
                     (dict(head_dim=1), "head_dim"), (dict(head_dim=2048), "head_dim"), (dict(n_axes=0), "n_axes"),
                     (dict(n_axes=5), "n_axes"), (dict(section=(8, -1, 9)), "section"), (dict(section=(0, 0, 0)), "pairs"),
                     (dict(section=(8, 13, 12)), "pairs"), (dict(section=(2 ** 31 - 1, 2 ** 31 - 1, 2)), "pairs"),
                     (dict(theta=0.0), "theta"), (dict(theta=float("nan")), "theta"), (dict(theta=float("inf")), "theta"),
                     (dict(ld_q=255), "row lengths"), (dict(ld_k_out=1), "row lengths"), (dict(ld_q_out=300), "in place")):
        refused(ssd.ssd_rope_axes, [change(p, **kw), 3] + a, word)
    refused(ssd.ssd_rope_axes, [p, 0] + a, "T = 0")
    refused(ssd.ssd_rope_axes, [p, 2 ** 25] + a, "T = 33554432")
    for i in range(5):
        refused(ssd.ssd_rope_axes, [p, 3] + a[:i] + [None] + a[i + 1:], "NULL")


CACHE = dict(k=X, v=X, k_exp=X, v_exp=X, n_blocks=9, block=16, n_kv_heads=2, head_dim=64)
BAD_CACHE = ((dict(block=8), "block"), (dict(head_dim=96), "head_dim"), (dict(n_kv_heads=0), "n_kv_heads"),
             (dict(n_blocks=0), "n_blocks"), (dict(n_blocks=2 ** 28), "n_blocks"))


def test_append_refusals(lib):
    c, p = ssd.ssd_kvq_cache(**CACHE), ssd.ssd_kvq_append_params(ssd.SSD_F32, 5, 128, 128)
    for kw, word in BAD_CACHE:
        refused(ssd.ssd_kvq_append, (change(c, **kw), p, X, X, X), word)
    for kw, word in ((dict(dtype=2), "dtype"), (dict(n_rows=-1), "n_rows"), (dict(n_rows=2 ** 29), "launch"), (dict(ld_k=127), "row lengths"), (dict(ld_v=0), "row lengths")):
        refused(ssd.ssd_kvq_append, (c, change(p, **kw), X, X, X), word)
    for i in range(3):
        refused(ssd.ssd_kvq_append, [c, p] + [X] * i + [None] + [X] * (2 - i), "NULL")
    for f in ("k", "v", "k_exp", "v_exp"):
        refused(ssd.ssd_kvq_append, (change(c, **{f: None}), p, X, X, X), "NULL")
    assert lib.ssd_kvq_append(None, ctypes.byref(p), None, None, None, None) == ssd.SSD_E_INVAL


def test_attention_refusals(lib):
    c = ssd.ssd_kvq_cache(**CACHE)
    p = ssd.ssd_kvq_attn_params(ssd.SSD_BF16, 3, 5, 4, 2, 100, 7, 256, 256, 0.125, 0)
    p.workspace_bytes = ssd.ssd_kvq_workspace(c, p)
    a = [X] * 6
    cases = [(change(c, **kw), p, word) for kw, word in BAD_CACHE]
    cases += [(c, change(p, **kw), word) for kw, word in (
        (dict(dtype=-1), "dtype"), (dict(n_seqs=0), "positive"), (dict(n_rows=0), "positive"), (dict(max_q=0), "positive"),
        (dict(max_len=0), "positive"), (dict(table_width=0), "positive"), (dict(n_heads=5), "n_heads"), (dict(n_heads=0), "n_heads"),
        (dict(n_seqs=2 ** 15, max_q=2 ** 14), "2^31"), (dict(n_seqs=2 ** 23, max_q=1), "2^24"), (dict(table_width=2 ** 27), "2^30"), (dict(ld_q=255), "row lengths"), (dict(ld_out=255), "row lengths"),
        (dict(scale=float("nan")), "scale"), (dict(scale=1e300), "scale"))]
    for cc, pp, word in cases:
        refused(ssd.ssd_kvq_attention, [cc, pp] + a, word)
        refused(ssd.ssd_kvq_workspace, [cc, pp], word)
    for i in range(5):
        refused(ssd.ssd_kvq_attention, [c, p] + a[:i] + [None] + a[i + 1:], "NULL")
    refused(ssd.ssd_kvq_attention, [c, change(p, workspace_bytes=-1)] + a, "workspace")
    refused(ssd.ssd_kvq_attention, [c, change(p, ld_out=300), X, X, X, X, X, X], "in place")


def test_sample_refusals(lib):
    p = ssd.ssd_sample_params(vocab=100, ld=100, temperature=1.0, top_p=1.0)
    a = [X] * 3
    nan, inf = float("nan"), float("inf")
    for kw, word in ((dict(vocab=0), "vocab"), (dict(vocab=2 ** 18 + 1, ld=2 ** 19), "vocab"), (dict(ld=99), "ld"),
                     (dict(temperature=-1.0), "temperature"), (dict(temperature=nan), "temperature"), (dict(temperature=inf), "temperature"),
                     (dict(top_p=nan), "top_p"), (dict(min_p=nan), "min_p")):
        refused(ssd.ssd_sample_logits, [change(p, **kw), 2] + a, word)
    refused(ssd.ssd_sample_logits, [p, 0] + a, "R = 0")
    refused(ssd.ssd_sample_logits, [p, 2 ** 22] + a, "R = 4194304")
    for i in range(3):
        refused(ssd.ssd_sample_logits, [p, 2] + a[:i] + [None] + a[i + 1:], "NULL")


def test_addresses_that_are_no_device_arrays(lib):
    """Host memory (and, here, no GPU at all) is refused before anything is launched."""
    host = np.zeros(4096, np.float32)
    p = ssd.ssd_sample_params(vocab=8, ld=8, temperature=1.0, top_p=1.0)
    refused(ssd.ssd_sample_logits, [p, 2, host, host, host], "needs an aligned array of the current device")


# ---------------------------------------------------------------- the plain implementations
def test_e4m3_values():
    assert np.nanmax(S.E4M3) == 448.0 and S.E4M3[1] == 2.0 ** -9 and S.E4M3[8] == 2.0 ** -6 and S.E4M3[0x38] == 1.0
    v = np.unique(S.E4M3[~np.isnan(S.E4M3)])
    assert np.array_equal(S.e4m3_round(v), v)
    mid = (v[1:] + v[:-1]) / 2  # ties go to the code with an even last bit
    even = {x for c, x in enumerate(S.E4M3) if c % 2 == 0}
    assert all(x in even for x in S.e4m3_round(mid))
    assert np.array_equal(S.e4m3_round(mid + 1e-9 * np.abs(mid) + 1e-12), v[1:])


def test_exponents():
    for e in (1, 100, 127, 200):
        s = 2.0 ** (e - 127)
        assert S.exponent(448 * s) == e and S.exponent(448 * s * (1 + 2.0 ** -20)) == e + 1 and S.exponent(225 * s) == e
    assert S.exponent(0.0) == 1 and S.exponent(3.4028234e38) == 247


def test_plain_rope():
    """Equal positions on all axes are the one-axis rotation; a quarter turn; norms stay."""
    rng = np.random.default_rng(0)
    x = rng.standard_normal((6, 2, 16))
    pos = rng.integers(0, 99, 6)
    a = S.rope(x, np.stack([pos] * 3), (2, 3, 3), 1e4)
    assert np.allclose(a, S.rope(x, pos[None], (8,), 1e4), atol=1e-13)
    assert np.allclose((a ** 2).sum(-1), (x ** 2).sum(-1))
    one = S.rope(np.array([[[1.0, 0.0]]]), np.array([[1]]), (1,), 1e4)
    assert np.allclose(one, [[[np.cos(1), np.sin(1)]]])


def test_plain_append_and_attention():
    """One key: the output is its value; equal keys: the mean; a block's scale grows with what is appended."""
    c = S.Cache(3, 1, 4, 2)
    c.append([4], np.array([[[1.0, 2.0]]]), np.array([[[3.0, -6.0]]]))
    q = np.array([[[5.0, -1.0]]])
    t = np.array([[1]])
    out, _ = S.attention(c, q, [0, 1], [1], t, 1.0, False)
    assert np.array_equal(out, [[[3.0, -6.0]]])
    c.append([5], np.array([[[1.0, 2.0]]]), np.array([[[448.0, 2.0]]]))
    assert c.ve[1, 0] == 127 and c.v[1, 0, 0].tolist() == [3.0, -6.0]
    out, _ = S.attention(c, q, [0, 1], [2], t, 1.0, False)
    assert np.allclose(out, [[[225.5, -2.0]]])
    c.append([4], np.array([[[1.0, 2.0]]]), np.array([[[0.5, 0.25]]]))  # offset 0 sets the exponent anew
    assert c.ve[1, 0] == S.exponent(0.5)


def test_plain_slots():
    t = np.array([[5, -1, -1], [-1, -1, -1]])
    w = S.slots([3, 0], [2, 5], [8, 9, 7], t, 4, 9)
    assert w["table"].tolist() == [[5, 8, -1], [9, 7, -1]] and w["lens"].tolist() == [5, 5] and w["cu"].tolist() == [0, 2, 7]
    assert w["slots"].tolist() == [23, 32, 36, 37, 38, 39, 28, -1, -1] and w["positions"].tolist() == [3, 4, 0, 1, 2, 3, 4, -1, -1]
    assert w["used"].tolist() == [3]


def test_plain_sampling():
    l = np.log(np.array([0.1, 0.4, 0.2, 0.3]))
    f = lambda u, **k: S.sample(l, u, k.get("T", 1.0), k.get("k", 0), k.get("p", 1.0), k.get("m", 0.0))  # noqa: E731
    assert [f(u)[0] for u in (0.0, 0.09, 0.11, 0.49, 0.51, 0.69, 0.71, 0.999)] == [0, 0, 1, 1, 2, 2, 3, 3]
    assert f(0.99, k=1)[0] == 1 and f(0.0, k=2)[0] == 1 and f(0.99, k=2)[0] == 3
    assert {f(u, p=0.65)[0] for u in np.linspace(0, 0.999, 50)} == {1, 3} and f(0.5, p=0.39) == (1, 1.0)
    assert {f(u, m=0.6)[0] for u in np.linspace(0, 0.999, 50)} == {1, 3} and f(0.3, T=0.0) == (1, 1.0)
    assert abs(f(0.99, p=0.65)[1] - 3 / 7) < 1e-12
