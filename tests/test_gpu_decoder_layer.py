"""The decoder layer of examples/: the paged cache, the 8-bit projections, the
latent attention and the MoE layer together."""
import numpy as np
import pytest
import torch

from examples.decoder_layer import DecoderLayer, Pages, SHAPES
from paper_2606_29982_amd import caee

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def _layer(n_pages, block, seed=1):
    shape, heads, q_rank = SHAPES["tiny"]
    return DecoderLayer(shape, heads, q_rank, n_pages, block, DEV, seed=seed), shape.d


def _tokens(new):
    return torch.tensor(new, dtype=torch.int32, device=DEV)


def test_steps_agree_with_the_whole_prompt():
    """Attention over tokens that came in three steps, and over the same at once.

    Both sides quantise the same values to 8 bits up to the forms' rounding (3e-3 of a row, rms, on either side),
    which moves about a tenth of the codes of the output projection by a step of 1/16: sqrt(0.1) / 16 = 2e-2 of the
    attention's part, rms.  Allowed: 5e-2."""
    block, lens, parts = 16, [70, 33, 5], [[64, 30, 3], [5, 0, 1], [1, 3, 1]]
    layer, d = _layer(40, block)
    x = [torch.randn((n, d), device=DEV).bfloat16() for n in lens]

    whole = Pages(3, 20, block, 80, DEV)
    plan = whole.step(_tokens(lens), sum(lens))
    at_once = layer.attention(torch.cat(x), plan, whole.table, max(lens), sum(lens)).split(lens)

    pages, ctx, got = Pages(3, 20, block, 80, DEV), [0, 0, 0], [[], [], []]
    for new in parts:
        rows = torch.cat([x[b][ctx[b]:ctx[b] + n] for b, n in enumerate(new)])
        plan = pages.step(_tokens(new), sum(new))
        ctx = [c + n for c, n in zip(ctx, new)]
        assert plan["seq_len"].tolist() == ctx and int(plan["lacking"][0]) == 0
        for b, y in enumerate(layer.attention(rows, plan, pages.table, max(new), sum(ctx)).split(new)):
            got[b].append(y)
    for b in range(3):
        a, g = at_once[b].double() - x[b].double(), torch.cat(got[b]).double() - x[b].double()
        assert float((a - g).square().mean().sqrt()) <= 5e-2 * float(a.square().mean().sqrt())


def test_serving_loop():
    block, prompts, steps = 16, [31, 1, 16, 90], 5
    n_pages = sum(-(-(n + steps) // block) for n in prompts)
    layer, d = _layer(n_pages, block, seed=2)
    pages = Pages(4, n_pages, block, 100, DEV)
    x, new, cached = torch.randn((sum(prompts), d), device=DEV).bfloat16(), _tokens(prompts), 0
    for s in range(steps + 1):
        cached += x.shape[0]
        plan = pages.step(new, x.shape[0])
        y = layer(x, plan, pages.table, max(prompts) if s == 0 else 1, cached)
        assert torch.isfinite(y).all()
        x, new = y[(plan["cu_new"][1:] - 1).long()], torch.ones_like(new)
    assert int(plan["free_head"][0]) == n_pages and int(plan["lacking"][0]) == 0
    assert pages.ctx.tolist() == [n + steps for n in prompts]
    used = pages.table[pages.table >= 0].cpu().numpy()
    assert np.array_equal(np.sort(used), np.arange(n_pages))       # every page once


def test_layer_needs_its_pages():
    """Without a free page a token has no slot; the plan says how many pages lack."""
    pages = Pages(1, 1, 16, 64, DEV)
    plan = pages.step(_tokens([20]), 20)
    assert int(plan["lacking"][0]) == 1 and plan["slots"].tolist()[16:] == [-1] * 4
    assert caee.Latent(4, 128, 64, 512, 128, 1.0).form == "auto"
