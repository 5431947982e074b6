"""Which kernel a windowed attention call takes, seen from outside: by the size of its workspace, the kernels it launches, and the
list of cut items that the tcgen05 form leaves in the workspace.  Tests that are meant for one form assert it."""
import torch

# form: B, H, G, d, dtype, past, c, window, sinks; B, H, G and c choose a form together with the slots that are seen
FORMS = {
    "cluster": (2, 3, 2, 128, torch.bfloat16, 700, 2, 600, 4), "cluster, 64": (1, 5, 1, 64, torch.float16, 3000, 1, 2500, 0),
    "cluster, 16 rows": (1, 2, 4, 128, torch.float16, 3000, 4, 2800, 20), "cluster, 32 bits": (1, 3, 3, 64, torch.float32, 900, 2, 800, 2),
    "whole": (40, 10, 1, 128, torch.bfloat16, 300, 1, 180, 4), "whole, 64": (40, 8, 2, 64, torch.float16, 300, 2, 200, 0),
    "whole, 32 bits": (30, 10, 2, 128, torch.float32, 300, 1, 180, 7),
    "list": (40, 10, 1, 64, torch.bfloat16, 2000, 1, 1900, 4), "list, 16 rows": (40, 10, 4, 128, torch.float16, 1500, 4, 1200, 9),
    "list, 32 bits": (40, 8, 1, 128, torch.float32, 1200, 1, 1100, 0),
    "mma": (20, 8, 1, 128, torch.bfloat16, 300, 40, 200, 3), "mma, large tiles": (60, 10, 1, 64, torch.bfloat16, 60, 64, 20, 4),
    "mma, pieces": (1, 2, 2, 64, torch.float16, 3000, 30, 2600, 1), "mma, 32 bits": (20, 8, 1, 128, torch.float32, 200, 40, 60, 5),
    "mma, 32 bits, pieces": (1, 2, 2, 64, torch.float32, 3000, 30, 2600, 0),
    "tcgen05": (4, 12, 1, 128, torch.bfloat16, 500, 300, 450, 4), "tcgen05, 64": (4, 30, 3, 64, torch.float16, 700, 200, 600, 20),
    "tcgen05, cut": (1, 4, 4, 128, torch.float16, 5000, 64, 4096, 4), "tcgen05, cut, 64": (1, 8, 1, 64, torch.bfloat16, 9000, 1000, 3500, 1),
}


def tcgen05_bytes(B, H, G, d, c):
    """Workspace of the tcgen05 form: a list entry for each of 148 CTAs, and where fewer than 888 items may be cut, two partial results
    of 256 rows for each."""
    pad = lambda n: -(-n // 256) * 256  # noqa: E731
    pair = 2 * (128 // G)
    return pad(148 * 16) + (pad(296 * 256 * 8) + pad(296 * 256 * d * 4) if B * H * -(-c // pair) < 888 else 0)


def attend(a2sf, cache, q, window, sinks, lens=None, out=None, lse=None):
    """One call -> out, lse and its form."""
    c, fp32 = q.shape[2], cache.dtype == torch.float32
    size = cache.attend_window_workspace_bytes(c, window, sinks)
    ws = a2sf.torch.empty((size,), dtype=torch.uint8, device="cuda").zero_()      # the binding's torch: in the debug sweep it puts guard words around
    before = a2sf.a2sf_kernel_launch_count()
    out, lse = cache.a2sf_paged_attend_window(q, window, sinks, lens=lens, out=out, lse=lse, workspace=ws)
    launches = a2sf.a2sf_kernel_launch_count() - before
    torch.cuda.synchronize()
    if c * cache.group <= (8 if fp32 else 16):
        form = "cluster" if size == 256 else "whole" if launches == 1 else "list"
    elif not fp32 and size == tcgen05_bytes(cache.B, cache.H, cache.group, cache.d, c):
        cut = bool((ws[: 148 * 16].view(torch.int32).view(148, 4)[:, 3] > 0).any())
        form = "tcgen05, cut" if cut else "tcgen05"
    else:
        form = "mma" if launches == 1 else "mma, pieces"
    return out, lse, form


def expected(name):
    """The form that attend() reports for a name of FORMS."""
    parts = name.split(", ")
    return parts[0] + "".join(", " + x for x in parts[1:] if x in ("cut", "pieces"))
