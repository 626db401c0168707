"""GPU parity of the paging plan and the latent cache store: every integer
and every stored bit must match the definitions."""
import numpy as np
import pytest
import torch

from attention_cases import plan_ref
from paper_2606_29982_amd import caee

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def _plan(block, T, ctx, new, width, n_free, head, seed=0):
    rng = np.random.default_rng(seed)
    ctx, new = np.asarray(ctx, np.int32), np.asarray(new, np.int32)
    B = len(ctx)
    table = np.full((B, width), -1, np.int32)
    for b in range(B):
        have = min(width, -(-max(int(ctx[b]), 0) // block))
        table[b, :have] = rng.integers(0, 5000, have)
    free = rng.permutation(np.arange(6000, 6000 + n_free)).astype(np.int32)
    ref = plan_ref(block, T, ctx, new, table, free, head)
    to = lambda a: torch.from_numpy(a).to(DEV)  # noqa: E731
    tab = to(table)
    out = caee.alloc_paged_plan(B, T, DEV)
    for v in out.values():
        v.fill_(-77)
    args = (to(ctx), to(new), tab, to(free), torch.tensor([head], dtype=torch.int32, device=DEV))
    for _ in range(2):      # the same inputs again: the same outputs
        caee.paged_plan(block, *args, out)
        torch.cuda.synchronize()
        for k, v in dict(out, table=tab).items():
            assert np.array_equal(v.cpu().numpy(), ref[k]), k
    return ref


@pytest.mark.parametrize("block", [1, 7, 16, 64])
@pytest.mark.parametrize("B", [1, 3, 64, 1000])
def test_plan(B, block):
    rng = np.random.default_rng(B + block)
    ctx, new = rng.integers(0, 200, B), rng.integers(0, 40, B)
    total = int(new.sum())
    _plan(block, total + 5, ctx, new, 300 // block + 2, total + B + 3, 3)


def test_plan_more_requests_than_threads():
    rng = np.random.default_rng(0)
    B = 2500
    _plan(16, 3000, rng.integers(0, 50, B), rng.integers(0, 2, B), 5, 4000, 0)


def test_plan_edges():
    _plan(16, 4, [0], [0], 1, 1, 0)                            # nothing new, nothing cached
    _plan(16, 0, [5, 9], [3, 1], 2, 4, 0)                      # no token list
    _plan(16, 3, [15, 16, 17], [1, 1, 1], 3, 4, 1)             # a page filled exactly, a page begun
    _plan(16, 8, [-3, 4], [2, -1], 2, 4, 0)                    # negative lengths count as none
    _plan(4, 6, [0, 0], [9, 9], 8, 8, 0)                       # fewer token entries than tokens
    _plan(128, 70000, [0], [70000], 600, 600, 0)               # one long prompt
    ref = _plan(4, 40, [2, 0, 7], [10, 12, 3], 6, 4, 1)        # the free list ends
    assert ref["lacking"][0] > 0 and (ref["slots"] < 0).any()
    ref = _plan(4, 40, [2, 0, 7], [10, 12, 3], 2, 20, 0)       # a table row ends
    assert ref["lacking"][0] > 0
    ref = _plan(4, 10, [2], [6], 6, 3, 9)                      # the head is past the list already
    assert ref["free_head"][0] == 9


def test_plan_no_requests():
    i32 = dict(dtype=torch.int32, device=DEV)
    out = caee.alloc_paged_plan(0, 5, DEV)
    caee.paged_plan(16, torch.empty(0, **i32), torch.empty(0, **i32), torch.empty((0, 4), **i32),
                    torch.arange(3, **i32), torch.tensor([2], **i32), out)
    torch.cuda.synchronize()
    assert out["slots"].tolist() == [-1] * 5 and out["cu_new"].tolist() == [0] and out["free_head"].tolist() == [2]


def test_plan_feeds_the_next_step():
    """Two decode steps in a row, the free head handed on."""
    i32 = dict(dtype=torch.int32, device=DEV)
    table = torch.full((2, 4), -1, **i32)
    free = torch.tensor([9, 4, 7, 5], **i32)
    a, b = caee.alloc_paged_plan(2, 20, DEV), caee.alloc_paged_plan(2, 2, DEV)
    caee.paged_plan(8, torch.zeros(2, **i32), torch.tensor([8, 3], **i32), table, free, torch.zeros(1, **i32), a)
    caee.paged_plan(8, a["seq_len"], torch.ones(2, **i32), table, free, a["free_head"], b)
    torch.cuda.synchronize()
    assert table.tolist() == [[9, 7, -1, -1], [4, -1, -1, -1]]
    assert b["slots"].tolist() == [7 * 8, 4 * 8 + 3] and b["free_head"].tolist() == [3]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,latent,rope,block", [(1, 512, 64, 64), (33, 512, 64, 16), (1000, 128, 64, 7), (5, 8, 8, 1)])
def test_store(T, latent, rope, block, dtype):
    rng = np.random.default_rng(T)
    blocks = -(-T // block) + 3
    slots = rng.permutation(blocks * block)[:T]
    slots[rng.random(T) < 0.2] = -1
    if T > 4:
        slots[2] = blocks * block            # past the cache: not written
    wide = torch.randn(T, latent + rope + 16, generator=torch.Generator().manual_seed(T)).to(dtype)
    wide[0, 0], wide[0, 1] = float("nan"), float("inf")
    cache = torch.randn(blocks + 2, block, latent + rope).to(torch.bfloat16)
    got = cache.to(DEV)
    w = wide.to(DEV)
    caee.latent_store(w[:, :latent], w[:, latent:latent + rope], torch.from_numpy(slots).to(DEV), got[:blocks])
    torch.cuda.synchronize()
    flat = cache.view(-1, latent + rope)
    for t, s in enumerate(slots):
        if 0 <= s < blocks * block:
            flat[s] = wide[t, :latent + rope].to(torch.bfloat16)
    a, b = got.cpu().view(torch.int16), cache.view(torch.int16)
    nan = torch.isnan(cache)
    assert torch.equal(torch.isnan(got.cpu()), nan) and torch.equal(a[~nan], b[~nan])


def test_store_keeps_slots_past_2_31_bytes():
    """A slot whose byte offset does not fit 32 bits."""
    rows = (5 << 30) // (576 * 2)
    cache = torch.zeros((rows + 1, 1, 576), dtype=torch.bfloat16, device=DEV)
    c = torch.full((2, 576), 3.0, dtype=torch.bfloat16, device=DEV)
    caee.latent_store(c[:, :512], c[:, 512:], torch.tensor([rows, 1], dtype=torch.int64, device=DEV), cache)
    torch.cuda.synchronize()
    assert torch.all(cache[rows] == 3.0) and torch.all(cache[1] == 3.0)
    assert float(cache[:1].float().abs().sum() + cache[2:1000].float().abs().sum()) == 0.0
    wrapped = rows - (1 << 32) // (576 * 2)
    assert torch.all(cache[wrapped - 2:wrapped + 3] == 0.0)


def test_plan_and_store_on_another_stream():
    s = torch.cuda.Stream()
    i32 = dict(dtype=torch.int32, device=DEV)
    with torch.cuda.stream(s):
        table = torch.full((1, 4), -1, **i32)
        out = caee.alloc_paged_plan(1, 9, DEV)
        caee.paged_plan(4, torch.zeros(1, **i32), torch.full((1,), 9, **i32), table, torch.arange(4, **i32),
                        torch.zeros(1, **i32), out)
        rows = torch.randn(9, 192, device=DEV)
        cache = torch.zeros((4, 4, 192), dtype=torch.bfloat16, device=DEV)
        caee.latent_store(rows[:, :128], rows[:, 128:], out["slots"], cache)
    s.synchronize()
    assert torch.equal(cache.view(16, 192)[:9], rows.to(torch.bfloat16))


def test_plan_and_store_in_a_graph():
    """Captured once, replayed on new lengths with the program's own work between the replays."""
    i32 = dict(dtype=torch.int32, device=DEV)
    B, T = 5, 64
    ctx, new = torch.zeros(B, **i32), torch.zeros(B, **i32)
    table, free, head = torch.full((B, 8), -1, **i32), torch.arange(40, **i32), torch.zeros(1, **i32)
    out = caee.alloc_paged_plan(B, T, DEV)
    rows = torch.zeros(T, 192, device=DEV)
    cache = torch.zeros((40, 8, 192), dtype=torch.bfloat16, device=DEV)

    def call():
        caee.paged_plan(8, ctx, new, table, free, head, out)
        caee.latent_store(rows[:, :128], rows[:, 128:], out["slots"], cache)

    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    rng = np.random.default_rng(1)
    for _ in range(4):
        n = rng.integers(0, 12, B).astype(np.int32)
        new.copy_(torch.from_numpy(n))
        rows.copy_(torch.randn(T, 192, device=DEV))
        table.fill_(-1)
        cache.zero_()
        g.replay()
        torch.cuda.synchronize()
        ref = plan_ref(8, T, np.zeros(B, np.int32), n, np.full((B, 8), -1, np.int32), np.arange(40), 0)
        assert np.array_equal(out["slots"].cpu().numpy(), ref["slots"])
        live = ref["slots"] >= 0
        want = torch.zeros(320, 192, dtype=torch.bfloat16)
        want[ref["slots"][live]] = rows.cpu()[torch.from_numpy(live)].to(torch.bfloat16)
        assert torch.equal(cache.cpu().view(320, 192), want)


def test_store_one_row_of_an_array_of_any_width():
    wide = torch.randn(2, 133 + 72, device=DEV).to(torch.bfloat16)
    cache = torch.zeros((2, 4, 192), dtype=torch.bfloat16, device=DEV)
    caee.latent_store(wide[:1, :128], wide[:1, 128:192], torch.tensor([5], dtype=torch.int64, device=DEV), cache)
    torch.cuda.synchronize()
    assert torch.equal(cache[1, 1], wide[0, :192]) and float(cache.float().abs().sum(2).count_nonzero()) == 1


def test_store_of_two_tokens_with_one_slot():
    """Each value of the row is of either token (the row's pieces are written apart); other rows are as ever."""
    T, rows = 4096, 64
    x = torch.arange(T, device=DEV, dtype=torch.float32)[:, None].expand(T, 192).contiguous() % 256     # a token's values: its number
    slots = torch.arange(T, device=DEV) % rows + 2
    cache = torch.full((2, 64, 192), -5.0, dtype=torch.bfloat16, device=DEV)
    caee.latent_store(x[:, :128], x[:, 128:], slots, cache)
    torch.cuda.synchronize()
    flat = cache.view(128, 192).float()
    assert torch.all(flat[:2] == -5.0) and torch.all(flat[2 + rows:] == -5.0)
    assert torch.all(flat[2:2 + rows] % rows == torch.arange(rows, device=DEV)[:, None]) and torch.all(flat[2:2 + rows] >= 0)
