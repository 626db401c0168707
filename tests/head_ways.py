"""Calls of grouped-head attention that say which kernel ran, and how its row tiles were cut."""
import numpy as np
import torch

from head_cases import HeadCase  # noqa: F401

STEP = 64                      # tokens of a step of the kernel of many rows
WHOLE = 2 ** 31 // 2 - 1       # steps of a piece where no row tile is cut


def run_way(c, dev, form, causal=True, y_dtype=torch.bfloat16, lse=True):
    """(y, lse) of the case, and "few", "whole" or "cut" (up to 64 requests; of more "cut" or None).

    The kernel of many rows leaves the steps of a piece at the workspace's word B + 1, that of few rows nothing there."""
    from paper_2606_29982_amd import caee
    a = c.arguments(dev, form, causal, y_dtype)
    y = torch.full((c.T + 2, c.H, c.D), 7.0, dtype=y_dtype, device=dev)
    lbuf = torch.full((c.T + 8, c.H), 7.0, dtype=torch.float32, device=dev)
    print("case", form, causal, y_dtype, c.seq[:8], c.new[:8], len(c.seq), c.H, c.G, c.D, flush=True)
    caee.head_attention(y=y[1:c.T + 1], lse=lbuf[4:c.T + 4] if lse else None, **a)
    torch.cuda.synchronize()
    assert torch.all(y[0] == 7.0) and torch.all(y[c.T + 1] == 7.0), "write outside y"
    assert torch.all(lbuf[:4] == 7.0) and torch.all(lbuf[c.T + 4:] == 7.0), "write outside lse"
    B = len(c.seq)
    per = int(a["ws"][4 * (B + 1):4 * (B + 2)].view(torch.int32)[0])
    longest = max(-(-int(s) // STEP) for s, n in zip(c.seq, c.new) if n > 0)
    if 0 <= per < longest:
        way = "cut"
    elif B > 64:
        way = None
    else:
        way = "few" if per == -1 else "whole"
    got = y[1:c.T + 1].float().cpu().numpy().astype(np.float64), lbuf[4:c.T + 4].cpu().numpy()
    return got, way
