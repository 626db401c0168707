"""Inputs and 64-bit definitions of attention with grouped heads over a paged
cache, written from the formulas in float64 on the CPU."""
import numpy as np
import torch

from attention_cases import bf16

HALF_BF16, HALF_F32 = 2.0 ** -8, 2.0 ** -24        # half a step, relative to the value


def make_cache(n, block, G, D, layout, device="cpu", fill=float("nan")):
    """Keys and values [n][block][G][D] by token, by head, as halves of one array, or with gaps between all of them."""
    bf = dict(dtype=torch.bfloat16, device=device)
    if layout == "token":
        return tuple(torch.full((n, block, G, D), fill, **bf) for _ in range(2))
    if layout == "head":
        return tuple(torch.full((n, G, block, D), fill, **bf).transpose(1, 2) for _ in range(2))
    if layout == "joint":
        kv = torch.full((n, 2, block, G, D), fill, **bf)
        return kv[:, 0], kv[:, 1]
    assert layout == "gaps"
    return tuple(torch.full((n, block + 1, G, D + 8), fill, **bf)[:, :block, :, :D] for _ in range(2))


def chain_tree(new, words):
    """Masks under which every new token sees those up to itself: the causal order as a tree."""
    m = np.zeros((int(np.sum(new)), words), np.uint32)
    at = 0
    for n in new:
        for i in range(int(n)):
            for j in range(i + 1):
                m[at + i, j // 32] |= np.uint32(1 << (j % 32))
        at += int(n)
    return m


def random_tree(new, words, rng, empty=0.1):
    """Ancestor masks of random trees, some tokens without their own bit, some masks empty, bits past the request's tokens set."""
    m = np.zeros((int(np.sum(new)), words), np.uint32)
    at = 0
    for n in new:
        for i in range(int(n)):
            if i and rng.random() < 0.9:
                m[at + i] = m[at + rng.integers(0, i)]
            if rng.random() < 0.9:
                m[at + i, i // 32] |= np.uint32(1 << (i % 32))
        for i in range(int(n)):
            if rng.random() < empty:
                m[at + i] = 0
        for j in range(int(n), 32 * words):
            m[at:at + int(n), j // 32] |= np.uint32(1 << (j % 32))
        at += int(n)
    return m


class HeadCase:
    """Random queries and a paged cache of requests with `seq` tokens, the last `new` of them new."""

    def __init__(self, seq, new, H=8, G=2, D=128, block=16, layout="token", seed=0, pad=0, scale=None, wide=0, q_std=1.0,
                 tree=None, cut=0):
        rng = np.random.default_rng(seed)
        self.seq, self.new = np.array(seq, np.int64), np.array(new, np.int64)
        self.H, self.G, self.D, self.block = H, G, D, block
        self.scale = D ** -0.5 if scale is None else scale
        B = len(seq)
        self.T = int(self.new.sum()) + pad - cut
        self.q = bf16(rng, self.T, H, D, std=q_std)
        self.wide, self.tree = wide, None
        if tree is not None:
            self.tree = np.zeros((self.T, tree.shape[1]), np.uint32)
            n = min(self.T, len(tree))
            self.tree[:n] = tree[:n]
        need = -(-self.seq // block)
        n = int(need.sum()) + 2
        width = max(1, int(need.max()) if B else 1) + 1
        ids = rng.permutation(n)
        self.table = np.full((B, width), -1, np.int32)
        at = 0
        for b in range(B):
            self.table[b, :need[b]] = ids[at:at + need[b]]
            at += int(need[b])
        self.layout = layout
        self.k_cache, self.v_cache = make_cache(n, block, G, D, layout)       # what no token owns is NaN
        self.k, self.v = [], []
        for b in range(B):
            S = int(self.seq[b])
            k, v = bf16(rng, S, G, D), bf16(rng, S, G, D)
            pos = np.arange(S)
            self.k_cache[self.table[b, pos // block], pos % block] = k
            self.v_cache[self.table[b, pos // block], pos % block] = v
            self.k.append(k)
            self.v.append(v)
        self.cu_new = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int32)

    def put(self, b, pos, k=None, v=None):
        at = int(self.table[b, pos // self.block]), pos % self.block
        if k is not None:
            self.k[b][pos] = k
            self.k_cache[at] = k
        if v is not None:
            self.v[b][pos] = v
            self.v_cache[at] = v

    def device_caches(self, dev):
        """The caches on the device with their strides."""
        n, block, G, D = self.k_cache.shape
        k, v = make_cache(n, block, G, D, self.layout, dev)
        k.copy_(self.k_cache)
        v.copy_(self.v_cache)
        return k, v

    def arguments(self, dev, form="auto", causal=True, y_dtype=torch.bfloat16):
        """Everything a call needs, on the device."""
        from paper_2606_29982_amd import caee
        att = caee.Heads(heads=self.H, kv_heads=self.G, dim=self.D, scale=self.scale, causal=causal, form=form)
        to = lambda a, dt=None: torch.as_tensor(a).to(dev, dt)  # noqa: E731
        q = to(self.q)
        if self.wide:
            big = torch.full((self.T, self.H * self.D + self.wide), 7.0, dtype=q.dtype, device=dev)
            big[:, :self.H * self.D] = q.reshape(self.T, -1)
            q = big[:, :self.H * self.D].view(self.T, self.H, self.D)
        k, v = self.device_caches(dev)
        plan = dict(cu_new=to(self.cu_new, torch.int32), seq_len=to(self.seq, torch.int32))
        tree = None if self.tree is None else to(self.tree.view(np.int32))
        max_new, max_kv = int(self.new.max()) if len(self.new) else 0, int(self.seq.sum())
        ws = caee.alloc_head_workspace(att, self.T, len(self.seq), max_new, max_kv, dev, tree=tree is not None)
        ws.fill_(0xFF)
        return dict(att=att, q=q, k_cache=k, v_cache=v, block_table=to(self.table), plan=plan, ws=ws, max_new=max_new,
                    max_kv=max_kv, tree=tree)

    def run(self, dev, form="auto", causal=True, y_dtype=torch.bfloat16, lse=True):
        from paper_2606_29982_amd import caee
        a = self.arguments(dev, form, causal, y_dtype)
        # Outputs begin 16-byte aligned a row into a larger buffer, which must stay as it is around them.
        y = torch.full((self.T + 2, self.H, self.D), 7.0, dtype=y_dtype, device=dev)
        lbuf = torch.full((self.T + 8, self.H), 7.0, dtype=torch.float32, device=dev)
        caee.head_attention(y=y[1:self.T + 1], lse=lbuf[4:self.T + 4] if lse else None, **a)
        torch.cuda.synchronize()
        assert torch.all(y[0] == 7.0) and torch.all(y[self.T + 1] == 7.0), "write outside y"
        assert torch.all(lbuf[:4] == 7.0) and torch.all(lbuf[self.T + 4:] == 7.0), "write outside lse"
        return y[1:self.T + 1].float().cpu().numpy().astype(np.float64), lbuf[4:self.T + 4].cpu().numpy()

    def sees(self, b, i, causal=True):
        """Which of request b's tokens new token i sees."""
        S, n = int(self.seq[b]), int(self.new[b])
        pos = np.arange(S)
        if self.tree is not None:
            m, bit = self.tree[self.cu_new[b] + i], pos - (S - n)
            inside = (bit >= 0) & (bit < 32 * m.size)
            word = m[np.where(inside, bit, 0) // 32] >> (np.where(inside, bit, 0) % 32).astype(np.uint32) & 1
            return (bit < 0) | (inside & (word == 1))
        return pos < S - n + i + 1 if causal else pos < S

    def ref(self, causal=True):
        """y, lse, sum of weights times |v|, and the largest scale * sum |q| |k| of a row's scores."""
        f8 = torch.float64
        y = torch.zeros(self.T, self.H, self.D, dtype=f8)
        ya, sa = torch.zeros_like(y), torch.zeros(self.T, self.H, dtype=f8)
        lse = torch.full((self.T, self.H), -float("inf"), dtype=f8)
        r = self.H // self.G
        for b in range(len(self.seq)):
            k, v = self.k[b].to(f8), self.v[b].to(f8)
            for i in range(int(self.new[b])):
                t = int(self.cu_new[b]) + i
                if t >= self.T:
                    break
                seen = torch.from_numpy(self.sees(b, i, causal))
                if not seen.any():
                    continue
                for g in range(self.G):
                    q, kk, vv = self.q[t, g * r:(g + 1) * r].to(f8), k[seen, g], v[seen, g]
                    s = self.scale * (q @ kk.t())
                    p = torch.softmax(s, 1)
                    h = slice(g * r, (g + 1) * r)
                    lse[t, h], y[t, h], ya[t, h] = torch.logsumexp(s, 1), p @ vv, p @ vv.abs()
                    sa[t, h] = self.scale * (q.abs() @ kk.abs().t()).amax(1)
        return y.numpy(), lse.numpy(), ya.numpy(), sa.numpy()


def check_heads(got, ref, y_dtype=torch.bfloat16, rows=None):
    """Every value within what the roundings can do.

    A score sums `dim` exact products in 32 bits, in any order: it is off by at most 128 half steps of scale * sum |q|
    |k| =: sa, and a few of its own, taken as 2^-16 sa + 2^-20 in all; the weight by as much, relatively.  Weights are
    rounded to bf16 (half a step), for a 32-bit result to two bf16 parts (half a step squared), and so may be their
    sum's addends; a value is then off by twice the weights' error times sum p |v|, and by its own rounding."""
    (y, lse), (ry, rl, ya, sa) = got, ref
    if rows is not None:
        y, lse, ry, rl, ya, sa = (a[rows] for a in (y, lse, ry, rl, ya, sa))
    none = np.isneginf(rl)
    assert np.array_equal(np.isneginf(lse), none)
    assert np.all(y[none] == 0.0)
    if none.all():
        return
    assert np.all(np.isfinite(y))
    weight = (HALF_BF16 if y_dtype == torch.bfloat16 else HALF_BF16 ** 2) + 2.0 ** -16 * sa + 2.0 ** -20
    out = HALF_BF16 if y_dtype == torch.bfloat16 else HALF_F32
    tol = 2 * weight[:, :, None] * ya + out * (1 + 2 * HALF_BF16) * (np.abs(ry) + 2 * weight[:, :, None] * ya) + 1e-30
    over = np.abs(y - ry) / tol
    assert over.max() <= 1.0, (over.max(), np.unravel_index(over.argmax(), over.shape))
    tol = weight + 2.0 ** -22 * np.abs(np.where(none, 0.0, rl))
    off = np.abs(np.where(none, 0.0, lse) - np.where(none, 0.0, rl))
    assert np.all(off <= tol), (off / tol).max()


def store_ref(x, w, freq, position, adjacent, eps, rotate=True):
    """Norm and rotation of [T][heads][D] float64 heads."""
    x = x.to(torch.float64).clone()
    if w is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w.to(torch.float64)
    size = x.abs().clone()      # what a value's error goes by: both of its pair's
    if freq is not None and rotate:
        r = 2 * len(freq)
        a, b = (x[..., 0:r:2], x[..., 1:r:2]) if adjacent else (x[..., :r // 2], x[..., r // 2:r])
        angle = position.to(torch.float64)[:, None, None] * freq
        u, v = a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()
        n = a.abs() + b.abs()
        out, big = x.clone(), size
        if adjacent:
            out[..., 0:r:2], out[..., 1:r:2], big[..., 0:r:2], big[..., 1:r:2] = u, v, n, n
        else:
            out[..., :r // 2], out[..., r // 2:r], big[..., :r // 2], big[..., r // 2:r] = u, v, n, n
        x = out
    return x, size
