"""The paging calls, the head store and the attention as a serving loop runs
them: prompts, decode steps, a verified tree of drafts, in one cache, each step
against a program that keeps every request's keys and values in float64."""
import numpy as np
import pytest
import torch

from examples.decoder_layer import HeadsLayer, Pages, SHAPES
from head_cases import HALF_BF16, make_cache, store_ref
from paper_2606_29982_amd import caee

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
BF = torch.bfloat16


class Server:
    def __init__(self, B, H, G, D, block, layout, rope, norm, seed):
        g = torch.Generator().manual_seed(seed)
        self.B, self.H, self.G, self.D, self.block = B, H, G, D, block
        self.freq = torch.from_numpy(10000.0 ** (-np.arange(0, rope, 2) / rope))
        self.wq, self.wk = ((1 + 0.2 * torch.randn(D, generator=g)) if norm else None for _ in range(2))
        n = 200
        self.kc, self.vc = make_cache(n, block, G, D, layout, DEV)
        self.table = torch.full((B, 64), -1, dtype=torch.int32, device=DEV)
        self.free = torch.randperm(n, generator=g).to(torch.int32).to(DEV)
        self.ctx, self.head = torch.zeros(B, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
        self.att = caee.Heads(heads=H, kv_heads=G, dim=D, scale=D ** -0.5)
        self.k, self.v = [[] for _ in range(B)], [[] for _ in range(B)]      # rows as the cache should hold them
        self.g = g

    def step(self, new, depth=None, tree=None, keep=True):
        """A step in which request b has new[b] tokens, at `depth` past its cached ones (None: one after the other)."""
        B, H, G, D = self.B, self.H, self.G, self.D
        T, pad = sum(new), 3
        wide = torch.randn(T + pad, (H + 2 * G) * D, generator=self.g).to(BF)
        dev = wide.to(DEV)
        q, k, v = (w.view(T + pad, -1, D) for w in dev.split([H * D, G * D, G * D], 1))
        new_dev = torch.tensor(new, dtype=torch.int32, device=DEV)
        plan = caee.alloc_paged_plan(B, T + pad, DEV)
        caee.paged_plan(self.block, self.ctx, new_dev, self.table, self.free, self.head, plan)
        position = plan["position"]
        if depth is not None:
            base = self.ctx.repeat_interleave(new_dev.long())
            position = torch.cat([base + torch.tensor(depth, dtype=torch.int32, device=DEV),
                                  torch.full((pad,), -1, dtype=torch.int32, device=DEV)])
        to = lambda a: None if a is None else a.to(DEV)  # noqa: E731
        caee.head_store(q, k, v, plan["slots"], q, self.kc, self.vc, q_norm=to(self.wq), k_norm=to(self.wk),
                        position=position, freq=to(self.freq))
        held = [len(r) for r in self.k]
        max_kv = sum(held) + T
        words = None
        if tree is not None:
            words = torch.zeros(T + pad, tree.shape[1], dtype=torch.int32, device=DEV)
            words[:T] = torch.from_numpy(tree.view(np.int32)).to(DEV)
        y = torch.full((T + pad, H, D), 7.0, dtype=BF, device=DEV)
        ws = caee.alloc_head_workspace(self.att, T + pad, B, max(new), max_kv, DEV, tree=tree is not None)
        caee.head_attention(self.att, q, self.kc, self.vc, self.table, plan, y, ws, max(new), max_kv, tree=words)
        torch.cuda.synchronize()
        assert int(plan["lacking"][0]) == 0
        slots = plan["slots"][:T].cpu()
        at = slots // self.block, slots % self.block
        self._check(wide, position.cpu(), new, tree, q.cpu(), self.kc.cpu()[at], self.vc.cpu()[at], y.cpu())
        if keep:
            self.ctx, self.head = plan["seq_len"], plan["free_head"]
        else:               # a program that takes the step back: its own lengths and head go on
            self.k, self.v = [r[:n] for r, n in zip(self.k, held)], [r[:n] for r, n in zip(self.v, held)]
        return plan

    def _check(self, wide, position, new, tree, q, k_new, v_new, y):
        H, G, D, T = self.H, self.G, self.D, sum(new)
        rq, rk, rv = (w.view(wide.shape[0], -1, D) for w in wide.split([H * D, G * D, G * D], 1))
        for got, x, w in ((q, rq, self.wq), (k_new, rk[:T], self.wk)):
            want, size = store_ref(x, w, self.freq, position[:len(x)], False, 1e-6)
            assert torch.all((got.double() - want).abs() <= HALF_BF16 * want.abs() + 2.0 ** -20 * size + 1e-30)
        assert torch.equal(v_new, rv[:T])
        r, t0 = H // G, 0
        for b, n in enumerate(new):
            held = len(self.k[b])
            self.k[b] += list(k_new[t0:t0 + n].double())
            self.v[b] += list(v_new[t0:t0 + n].double())
            for i in range(n):
                t = t0 + i
                seen = list(range(held + i + 1)) if tree is None else list(range(held)) + [
                    held + j for j in range(n) if tree[t, j // 32] >> np.uint32(j % 32) & 1]
                k, v = torch.stack([self.k[b][j] for j in seen]), torch.stack([self.v[b][j] for j in seen])
                for g in range(G):
                    h, kk, vv = slice(g * r, (g + 1) * r), k[:, g], v[:, g]
                    qd = q[t, h].double()
                    p = torch.softmax((qd @ kk.t()) * D ** -0.5, 1)
                    ref, mag = p @ vv, p @ vv.abs()
                    # as check_heads: the weights' errors (their rounding, the score's), then the result's rounding
                    score = (qd.abs() @ kk.abs().t()).amax(1, keepdim=True) * D ** -0.5
                    off = 2 * (HALF_BF16 + 2.0 ** -16 * score + 2.0 ** -20) * mag
                    tol = off + HALF_BF16 * (1 + 2 * HALF_BF16) * (ref.abs() + off) + 1e-30
                    assert torch.all((y[t, h].double() - ref).abs() <= tol)
            t0 += n
        assert torch.all(y[T:] == 0)


@pytest.mark.parametrize("H,G,D,block,layout,rope,norm", [
    (8, 2, 128, 16, "token", 128, True), (12, 4, 64, 64, "head", 32, False), (8, 8, 128, 7, "joint", 64, True)])
def test_prompts_decode_and_drafts(H, G, D, block, layout, rope, norm):
    s = Server(3, H, G, D, block, layout, rope, norm, seed=H + block)
    s.step([40, 17, 1])
    s.step([1, 1, 1])
    s.step([1, 33, 0])
    # a tree of five drafts for two requests: 0 - (1 - 3, 2 - 4), checked and taken back
    tree = np.zeros((10, 1), np.uint32)
    for r in range(2):
        for i, up in enumerate((None, 0, 0, 1, 2)):
            tree[5 * r + i] = (0 if up is None else tree[5 * r + up, 0]) | np.uint32(1 << i)
    s.step([5, 0, 5], depth=[0, 1, 1, 2, 2] * 2, tree=tree, keep=False)
    s.step([3, 1, 3])                # the accepted path, one after the other, in the same pages
    for _ in range(3):
        s.step([1, 1, 1])


def test_decoder_layer_steps_agree_with_the_whole_prompt():
    """Attention over tokens that came in three steps, and over the same at once.

    Queries, keys and values are the same in both; the attention's results differ by their roundings (2^-8 of a value
    and of its addends), which moves about a tenth of the codes of the output projection by a step of 1/16: sqrt(0.1) / 16
    = 2e-2 of the attention's part, rms.  Allowed: 5e-2."""
    shape, heads, q_rank = SHAPES["tiny"]
    layer = HeadsLayer(shape, heads, q_rank, 40, 16, DEV, seed=1)
    lens, parts = [70, 33, 5], [[64, 30, 3], [5, 0, 1], [1, 3, 1]]
    x = [torch.randn((n, shape.d), device=DEV).bfloat16() for n in lens]
    tokens = lambda new: torch.tensor(new, dtype=torch.int32, device=DEV)  # noqa: E731
    whole = Pages(3, 20, 16, 80, DEV)
    at_once = layer.attention(torch.cat(x), whole.step(tokens(lens), sum(lens)), whole.table, max(lens), sum(lens)).split(lens)
    pages, ctx, got = Pages(3, 20, 16, 80, DEV), [0, 0, 0], [[], [], []]
    for new in parts:
        rows = torch.cat([x[b][ctx[b]:ctx[b] + n] for b, n in enumerate(new)])
        plan = pages.step(tokens(new), sum(new))
        y = layer.attention(rows, plan, pages.table, max(new), sum(ctx) + sum(new)).split(new)
        for b, n in enumerate(new):
            ctx[b] += n
            got[b].append(y[b])
    torch.cuda.synchronize()
    for b in range(3):
        a, c = at_once[b].float() - x[b].float(), torch.cat(got[b]).float() - x[b].float()
        assert torch.isfinite(c).all() and (a - c).norm() <= 5e-2 * a.norm()


def test_decoder_layer_runs_whole_steps():
    shape, heads, q_rank = SHAPES["tiny"]
    layer = HeadsLayer(shape, heads, q_rank, 40, 16, DEV, seed=2)
    pages = Pages(2, 40, 16, 64, DEV)
    x = torch.randn((12, shape.d), device=DEV).bfloat16()
    plan = pages.step(torch.tensor([9, 3], dtype=torch.int32, device=DEV), 12)
    y = layer(x, plan, pages.table, 9, 12)
    torch.cuda.synchronize()
    assert y.shape == x.shape and torch.isfinite(y.float()).all()
