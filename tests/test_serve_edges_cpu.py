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
