"""Which windowed calls of few rows go without a workspace, that is to clusters: host only, no GPU."""
import pytest
import torch

BF, HF, FP = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def a2sf():
    from paper_2407_20485_b200 import build

    build.build()
    from paper_2407_20485_b200 import binding

    return binding


@pytest.mark.parametrize("B,H,G,d,dtype,c,window,clusters", [
    # short parts of a unit, or few units
    (1, 32, 1, 128, BF, 1, 205, True), (1, 8, 1, 128, BF, 1, 4000, True), (1, 32, 1, 128, BF, 1, 4000, True), (8, 8, 4, 128, HF, 4, 4096, True),
    (4, 37, 1, 128, FP, 1, 300, True), (1, 14, 1, 128, FP, 1, 4000, True), (37, 8, 1, 128, BF, 1, 450, True), (1, 37, 1, 128, BF, 1, 1000, True),
    # more units than fit at once
    (149, 1, 1, 128, FP, 1, 300, False), (297, 1, 1, 128, BF, 1, 300, False),
    # long parts: one long sequence among short ones would make all wait
    (32, 8, 1, 128, BF, 1, 4096, False), (16, 8, 1, 128, BF, 1, 4096, False), (32, 8, 1, 128, BF, 1, 1500, False), (37, 4, 1, 128, FP, 1, 2000, False),
    # more clusters of this size than fit, or a device left idle
    (1, 16, 1, 128, FP, 1, 4096, False), (1, 37, 1, 128, FP, 1, 4096, False), (1, 75, 1, 128, FP, 1, 4096, False), (1, 35, 1, 128, BF, 1, 4096, False),
    (2, 37, 1, 128, BF, 1, 4096, False), (1, 38, 1, 128, BF, 1, 4096, False)])
def test_clusters_serve_where_they_fit_and_their_parts_are_short(a2sf, B, H, G, d, dtype, c, window, clusters):
    cache = a2sf.PagedCache(B, H, d, dtype, 16, 1, 1024, group=G, device="cpu")
    size = cache.attend_window_workspace_bytes(c, window, 0)
    assert (size == 256) == clusters and size >= 256
