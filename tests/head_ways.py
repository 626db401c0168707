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


def bf16_parts(x, n):
    """x [float64] as the sum of n bf16 numbers, each the nearest to what the ones before it leave."""
    total = torch.zeros_like(x)
    for _ in range(n):
        total = total + (x - total).to(torch.bfloat16).double()
    return total


def with_weight_parts(c, parts, y_dtype, causal=True):
    """The case's results in float64 but for the softmax weights, which are rounded to `parts` bf16 numbers before the
    values' sums (their own sum is of the weights themselves), and the result's rounding."""
    y = torch.zeros(c.T, c.H, c.D, dtype=torch.float64)
    r = c.H // c.G
    for b in range(len(c.seq)):
        k, v = c.k[b].double(), c.v[b].double()
        for i in range(int(c.new[b])):
            seen = torch.from_numpy(c.sees(b, i, causal))
            if not seen.any():
                continue
            for g in range(c.G):
                h = slice(g * r, (g + 1) * r)
                s = c.scale * (c.q[int(c.cu_new[b]) + i, h].double() @ k[seen, g].t())
                w = torch.exp(s - s.amax(1, keepdim=True))
                y[int(c.cu_new[b]) + i, h] = (bf16_parts(w, parts) @ v[seen, g]) / w.sum(1, keepdim=True)
    return y.to(y_dtype).double().numpy()


def _rms(a):
    return float(np.sqrt((a * a).mean()))


def precise(y, ref, y_dtype, parts):
    """Whether results are as near to the definition as weights of `parts` bf16 numbers let them be, over all values.

    32-bit results, three parts (24 bits and more): a score of a few units is rounded up to D / 16 times by 2^-24 of
    it at most, some 2^-22.5 as they fall, its power of two, the sums and the quotient by 2^-24 each: 2^-21 in all.  Two
    parts leave up to 2^-16 of a weight, some 2^-19 as they fall.
    bf16 results: the rounding of the definition itself, of which two parts are off by no more than a hundredth.  Weights of
    one part are off by as much as the result's rounding is, and independently: sqrt(2) of it in all, and at most 1.5."""
    off = _rms(y - ref) / _rms(ref)
    if y_dtype == torch.float32:
        return off <= 2.0 ** -21
    rounded = _rms(torch.from_numpy(ref).to(torch.bfloat16).double().numpy() - ref) / _rms(ref)
    return off <= (1.01 if parts > 1 else 1.5) * rounded
