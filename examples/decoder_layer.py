"""A decoder layer that serves a batch from a paged cache.

One step, for requests with any number of new tokens each (a prompt, or the
one token of a decode step):

    plan      pages, slots and positions of the new tokens       caee.paged_plan
    queries   x -> rank -> heads, 8-bit weights                  caee.block_matmul
    cache     x -> [latent | rotary key] rows into their slots   caee.block_matmul, caee.latent_store
    attention over the cached rows, output projection            caee.latent_attention, caee.block_matmul
    experts   router, cost-aware selection and the expert FFN    caee.moe_layer

With --attention heads the layer keeps keys and values of grouped heads in its
pages instead of latent rows:

    queries, keys, values   x -> heads, 8-bit weights            caee.block_matmul
    cache     norms, rotation, keys and values into their slots  caee.head_store
    attention over the cached heads, output projection           caee.head_attention, caee.block_matmul

Other norms, the latent rows' rotary embedding and the router's scores are torch operations.  The
plan, the cache's pages and all sums of lengths stay on the device; the host
knows only bounds.  Weights are random; a step's output is the next input.

    python examples/decoder_layer.py                             # small shape
    python examples/decoder_layer.py --attention heads
    python examples/decoder_layer.py --shape deepseek-r1-fp8     # 128 heads, 256 experts
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2606_29982_amd import caee                                           # noqa: E402
from synth_inputs import R1_FP8, TINY_F32, make_expert_weights_torch, make_routing_inputs   # noqa: E402

NOPE, ROPE, LATENT, V = 128, 64, 512, 128
SHAPES = {   # MoE shape, heads, rank of the queries
    "tiny": (TINY_F32.with_(name="tiny", w_dtype="bf16", x_dtype="bf16", y_dtype="bf16"), 4, 256),
    "deepseek-r1-fp8": (R1_FP8, 128, 1536),
}


def rms_norm(x, eps=1e-6):
    x = x.float()
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + eps)


def rotate(x, position, base=10000.0):
    """Rotary embedding of [T][...][ROPE], the two halves of the last dimension as pairs."""
    freq = base ** (-torch.arange(0, ROPE, 2, device=x.device, dtype=torch.float32) / ROPE)
    angle = position.float()[:, None] * freq
    angle = angle.view(angle.shape[0], *([1] * (x.dim() - 2)), ROPE // 2)
    a, b = x.float().chunk(2, -1)
    return torch.cat((a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()), -1)


class Linear8:
    """y = x W^T with e4m3 codes and one scale per 128 x 128 block of W."""

    def __init__(self, rows, cols, gen):
        w = torch.randn((rows, cols), generator=gen, device=gen.device) * cols ** -0.5
        rb = -(-rows // 128)
        blocks = torch.nn.functional.pad(w, (0, 0, 0, rb * 128 - rows)).view(rb, 128, cols // 128, 128)
        self.scale = (blocks.abs().amax((1, 3)) / 448.0).clamp_min(1e-12)
        codes = (blocks / self.scale[:, None, :, None]).view(rb * 128, cols)[:rows].to(torch.float8_e4m3fn)
        self.codes, self.layout = codes.contiguous(), caee.LAYOUT_ROWMAJOR
        if rows % 16 == 0:
            tiled = torch.empty_like(self.codes)
            caee.pack_matrix("fp8", self.codes, tiled, rows, cols, 1)
            self.codes, self.layout = tiled, caee.LAYOUT_TILED

    def __call__(self, x, dtype=torch.bfloat16):
        y = torch.empty((x.shape[0], self.codes.shape[0]), dtype=dtype, device=x.device)
        ws = caee.alloc_block_matmul_workspace(x, self.codes.shape[0], x.device)
        return caee.block_matmul(x, self.codes, self.scale, y, ws, layout=self.layout)


class Pages:
    """The cache's pages and the requests' block tables, on the device."""

    def __init__(self, n_requests, n_pages, block, max_len, device):
        i32 = dict(dtype=torch.int32, device=device)
        self.block = block
        self.table = torch.full((n_requests, -(-max_len // block)), -1, **i32)
        self.free = torch.randperm(n_pages, device=device).to(torch.int32)
        self.ctx = torch.zeros(n_requests, **i32)
        self.head = torch.zeros(1, **i32)

    def step(self, new, T):
        """The plan of a step in which request b receives new[b] tokens, T in all."""
        plan = caee.alloc_paged_plan(self.ctx.shape[0], T, self.ctx.device)
        caee.paged_plan(self.block, self.ctx, new, self.table, self.free, self.head, plan)
        self.ctx, self.head = plan["seq_len"], plan["free_head"]
        return plan


class DecoderLayer:
    def __init__(self, shape, heads, q_rank, n_pages, block, device, seed=0, tau=None):
        gen = torch.Generator(device=device).manual_seed(seed)
        d = shape.d
        self.shape, self.heads, self.device = shape, heads, device
        self.make_attention(heads, q_rank, n_pages, block, gen)
        self.router = torch.randn((shape.E, d), generator=gen, device=device) * d ** -0.5
        inp = make_routing_inputs(shape, seed=seed)
        to = lambda a: None if a is None else torch.from_numpy(a).to(device)  # noqa: E731
        self.bias, self.cost, self.bins = to(inp.bias), to(inp.cost), to(inp.bins)
        self.experts = make_expert_weights_torch(shape, seed, device)
        self.over = {} if tau is None else {"tau": tau}

    def make_attention(self, heads, q_rank, n_pages, block, gen):
        d, device = self.shape.d, self.device
        self.q_down, self.q_up = Linear8(q_rank, d, gen), Linear8(heads * (NOPE + ROPE), q_rank, gen)
        self.kv_down, self.out = Linear8(LATENT + ROPE, d, gen), Linear8(d, heads * V, gen)
        rand = lambda *s: (torch.randn(s, generator=gen, device=device) * LATENT ** -0.5).bfloat16()  # noqa: E731
        self.heads_kv = caee.pack_latent_weights(rand(heads, NOPE, LATENT), rand(heads, V, LATENT))
        self.att = caee.Latent(heads=heads, nope=NOPE, rope=ROPE, latent=LATENT, v=V, scale=(NOPE + ROPE) ** -0.5)
        self.cache = torch.zeros((n_pages, block, LATENT + ROPE), dtype=torch.bfloat16, device=device)

    def attention(self, x, plan, table, max_new, max_kv):
        """x + attention(norm(x)); the new tokens' rows go into the cache on the way."""
        T, h = x.shape[0], rms_norm(x).bfloat16()
        q = self.q_up(rms_norm(self.q_down(h, torch.float32)).bfloat16()).view(T, self.heads, NOPE + ROPE)
        q[..., NOPE:] = rotate(q[..., NOPE:], plan["position"]).bfloat16()
        row = self.kv_down(h, torch.float32)
        caee.latent_store(rms_norm(row[:, :LATENT]), rotate(row[:, LATENT:], plan["position"]), plan["slots"], self.cache)
        y = torch.empty((T, self.heads, V), dtype=torch.bfloat16, device=x.device)
        ws = caee.alloc_latent_workspace(self.att, T, table.shape[0], max_new, max_kv, x.device)
        caee.latent_attention(self.att, q, self.heads_kv, self.cache, table, plan, y, ws, max_new, max_kv)
        return x + self.out(y.view(T, self.heads * V))

    def ffn(self, x):
        h = rms_norm(x).bfloat16()
        layer = caee.Layer.from_shape(self.shape, T=x.shape[0], **self.over)
        y = torch.empty_like(h)
        caee.moe_layer(layer, h, h.float() @ self.router.t(), self.bias, self.cost, self.bins, self.experts, y,
                       caee.alloc_workspace(layer, x.device))
        return x + y

    def __call__(self, x, plan, table, max_new, max_kv):
        return self.ffn(self.attention(x, plan, table, max_new, max_kv))


class HeadsLayer(DecoderLayer):
    """The same with grouped heads: four query heads share a head's keys and values."""

    def make_attention(self, heads, q_rank, n_pages, block, gen):
        d, device, kv = self.shape.d, self.device, max(heads // 4, 1)
        self.split = [heads, kv, kv]
        self.qkv, self.out = Linear8(sum(self.split) * V, d, gen), Linear8(d, heads * V, gen)
        self.q_norm, self.k_norm = 1 + 0.1 * torch.randn((2, V), generator=gen, device=device)
        self.freq = 10000.0 ** (-torch.arange(0, V, 2, device=device, dtype=torch.float64) / V)
        self.att = caee.Heads(heads=heads, kv_heads=kv, dim=V, scale=V ** -0.5)
        self.k_cache, self.v_cache = torch.zeros((2, n_pages, block, kv, V), dtype=torch.bfloat16, device=device)

    def attention(self, x, plan, table, max_new, max_kv):
        T = x.shape[0]
        q, k, v = self.qkv(rms_norm(x).bfloat16()).view(T, sum(self.split), V).split(self.split, 1)
        caee.head_store(q, k, v, plan["slots"], q, self.k_cache, self.v_cache, q_norm=self.q_norm, k_norm=self.k_norm,
                        position=plan["position"], freq=self.freq)
        y = torch.empty((T, self.heads, V), dtype=torch.bfloat16, device=x.device)
        ws = caee.alloc_head_workspace(self.att, T, table.shape[0], max_new, max_kv, x.device)
        caee.head_attention(self.att, q, self.k_cache, self.v_cache, table, plan, y, ws, max_new, max_kv)
        return x + self.out(y.view(T, self.heads * V))


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--shape", choices=SHAPES, default="tiny")
    ap.add_argument("--attention", choices=("latent", "heads"), default="latent")
    ap.add_argument("--prompts", type=int, nargs="+", default=[300, 17, 1, 129])
    ap.add_argument("--steps", type=int, default=16)
    ap.add_argument("--block", type=int, default=64)
    args = ap.parse_args()
    device = torch.device("cuda:0")
    shape, heads, q_rank = SHAPES[args.shape]
    B, longest = len(args.prompts), max(args.prompts) + args.steps
    n_pages = sum(-(-(n + args.steps) // args.block) for n in args.prompts)
    layer = (HeadsLayer if args.attention == "heads" else DecoderLayer)(shape, heads, q_rank, n_pages, args.block, device)
    pages = Pages(B, n_pages, args.block, longest, device)
    x = torch.randn((sum(args.prompts), shape.d), device=device).bfloat16()
    new, cached = torch.tensor(args.prompts, dtype=torch.int32, device=device), 0
    for s in range(args.steps + 1):
        torch.cuda.synchronize()
        t0, T = time.perf_counter(), x.shape[0]
        max_new = max(args.prompts) if s == 0 else 1
        plan = pages.step(new, T)
        cached += T
        y = layer(x, plan, pages.table, max_new, cached)
        x = y[(plan["cu_new"][1:] - 1).long()]            # each request's last token
        new = torch.ones_like(new)
        torch.cuda.synchronize()
        if s in (0, 1, args.steps):
            print(f"step {s}: {T} new tokens, {cached} cached, {(time.perf_counter() - t0) * 1e3:.2f} ms", flush=True)
    lacking, used = int(plan["lacking"][0]), int(plan["free_head"][0])
    print(f"{used} of {n_pages} pages used, {lacking} lacking; output rms {float(x.float().square().mean().sqrt()):.3f}")


if __name__ == "__main__":
    main()
