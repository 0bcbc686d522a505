"""Refusals of the serving operators at the edges of fp32 and of the address space, without a GPU."""
import pytest

import paper_2606_20543_amd as ssd
from tests.test_serve_ops_cpu import CACHE, X, change, lib, refused  # noqa: F401


@pytest.mark.parametrize("scale", [2.4e38, -3.4e38, 1e39, float("inf"), float("nan")])
def test_scales_past_fp32(lib, scale):  # noqa: F811
    """Scores are formed in units of log 2: the scale times 1 / ln 2 has to be a number of fp32."""
    c = ssd.ssd_kvq_cache(**CACHE)
    p = ssd.ssd_kvq_attn_params(ssd.SSD_BF16, 3, 5, 4, 2, 100, 7, 256, 256, scale, 1 << 30)
    refused(ssd.ssd_kvq_workspace, [c, p], "scale")
    refused(ssd.ssd_kvq_attention, [c, p] + [X] * 6, "scale")
    for ok in (2.3e38, -2.3e38, 0.0, -0.0, 1e-300):
        ssd.ssd_kvq_workspace(c, change(p, scale=ok))


FAR = (2 ** 61, 2 ** 60 + 4, 2 ** 62 - 1, 2 ** 63 - 1)  # with 4-byte elements rows 1 and 2 wrap, or pass the address space


@pytest.mark.parametrize("ld", FAR)
def test_row_lengths_past_the_address_space(lib, ld):  # noqa: F811
    """Rows so far apart that their offsets pass 64 bits are refused by the name of their array (without a GPU every
    other array is refused for that), not taken for the few bytes that the product leaves."""
    rope = ssd.ssd_rope_params(n_heads=4, n_kv_heads=2, head_dim=64, dtype=ssd.SSD_F32, n_axes=1, section=(32,), ld_q=256, ld_k=256,
                               ld_q_out=256, ld_k_out=256, theta=1e4)
    a = [X + 4096 * i for i in range(5)]
    for f, word in (("ld_q", "q:"), ("ld_k", "k:"), ("ld_q_out", "q_out:"), ("ld_k_out", "k_out:")):
        refused(ssd.ssd_rope_axes, [change(rope, **{f: ld}), 3] + a, word)
    c = ssd.ssd_kvq_cache(**CACHE)
    p = ssd.ssd_kvq_append_params(ssd.SSD_F32, 3, 128, 128)
    refused(ssd.ssd_kvq_append, [c, change(p, ld_k=ld), X, X, X], "k:")
    refused(ssd.ssd_kvq_append, [c, change(p, ld_v=ld), X, X, X], "v:")
    p = ssd.ssd_kvq_attn_params(ssd.SSD_F32, 1, 3, 4, 1, 16, 1, 256, 256, 0.125, 0)
    refused(ssd.ssd_kvq_attention, [c, change(p, ld_q=ld)] + a, "q:")
    refused(ssd.ssd_kvq_attention, [c, change(p, ld_out=ld)] + a, "out:")
    p = ssd.ssd_sample_params(vocab=100, ld=ld, temperature=1.0, top_p=1.0)
    refused(ssd.ssd_sample_logits, [p, 3, X, X, X], "logits:")
    # one row has no distance to the next
    with pytest.raises(ssd.SSDError):
        ssd.ssd_sample_logits(p, 1, X, X, X)
    assert "logits:" not in ssd.ssd_last_error()
