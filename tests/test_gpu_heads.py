"""GPU parity of attention with grouped heads over a paged cache, both forms,
against the formula in float64."""
import numpy as np
import pytest
import torch

from head_cases import HeadCase, chain_tree, check_heads, random_tree
from paper_2606_29982_amd import caee

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
FORMS = ["split", "whole"]
BF, F32 = torch.bfloat16, torch.float32


def _check(form, causal=True, y_dtype=BF, **kw):
    c = HeadCase(**kw)
    print("case", form, causal, y_dtype, {k: v for k, v in kw.items() if k != "tree"}, flush=True)
    check_heads(c.run(DEV, form, causal, y_dtype), c.ref(causal), y_dtype)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("S", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300, 1025])
def test_one_new_token(S, form):
    _check(form, seq=[S], new=[1], seed=S)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,G", [(1, 1), (4, 4), (8, 1), (12, 4), (24, 1), (40, 8), (64, 8), (33, 1), (65, 1), (80, 1), (5, 5)])
def test_head_groups(H, G, D, form):
    _check(form, seq=[70, 5, 129], new=[1, 2, 1], H=H, G=G, D=D, seed=H)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("layout", ["token", "head", "joint", "gaps"])
@pytest.mark.parametrize("block", [1, 3, 16, 64, 100])
def test_pages(block, layout, form):
    _check(form, seq=[1, 64, 150], new=[1, 2, 30], H=6, G=3, block=block, layout=layout, seed=block)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("y_dtype", [BF, F32])
def test_prompts_ragged(y_dtype, causal, form):
    _check(form, causal, y_dtype, seq=[1, 17, 64, 127, 255, 256, 257, 400], new=[1, 17, 64, 100, 255, 256, 257, 300], H=4, G=2,
           seed=7)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("D", [64, 128])
def test_prompts_behind_a_prefix(D, form):
    _check(form, seq=[700, 333, 1100], new=[290, 1, 64], H=6, G=2, D=D, seed=8)


@pytest.mark.parametrize("form", FORMS)
def test_requests_without_new_tokens_and_padding(form):
    _check(form, seq=[40, 0, 9, 100, 5], new=[2, 0, 0, 1, 5], pad=11, seed=9)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("y_dtype", [BF, F32])
def test_nothing_but_padding(y_dtype, form):
    _check(form, y_dtype=y_dtype, seq=[0, 9], new=[0, 0], pad=5, seed=9)


@pytest.mark.parametrize("form", FORMS)
def test_more_new_tokens_than_cached_leaves_rows_empty(form):
    _check(form, seq=[3, 20], new=[7, 2], seed=10)


@pytest.mark.parametrize("form", FORMS)
def test_rows_end_inside_a_request(form):
    """Fewer rows than new tokens: they see what they see among all of them."""
    _check(form, seq=[30, 200], new=[3, 90], cut=41, seed=10)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("B", [63, 64, 65, 300])
def test_many_requests(B, form):
    rng = np.random.default_rng(11)
    seq = rng.integers(0, 90, B)
    _check(form, seq=seq, new=np.minimum(seq, rng.integers(0, 3, B)), H=4, G=2, D=64, pad=3, seed=11)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("y_dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 128])
def test_every_number_of_rows(D, y_dtype, form):
    """Requests of 1 to 128 rows, so that the last row tile of one has each of its numbers of rows."""
    new = list(range(1, 129))
    _check(form, y_dtype=y_dtype, seq=[n + 3 for n in new], new=new, H=1, G=1, D=D, seed=11)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("D", [64, 128])
def test_every_length(D, form):
    """Requests of 0 to 263 tokens, the last 0 to 4 of them new."""
    seq = list(range(264))
    _check(form, seq=seq, new=[min(n, n % 5) for n in seq], H=4, G=2, D=D, seed=11)


@pytest.mark.parametrize("ratio", [3, 8])
@pytest.mark.parametrize("B", [2, 7, 40, 64])
def test_row_tiles_of_several_requests_by_place(B, ratio):
    """More row tiles than run at a time, few enough to be taken by place: some requests without new tokens, prefixes of
    any length, one far behind the others."""
    rng = np.random.default_rng(B)
    new = rng.integers(0, 2 * (9600 // (ratio * B)), B)
    seq = new + rng.integers(0, 150, B)
    new[B // 2], seq[B // 2] = (0, 5) if B > 2 else (new[1], seq[1])
    seq[0] += 900
    _check("whole", seq=seq, new=new, H=8 * ratio, G=8, D=64, seed=11)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("D", [64, 128])
def test_float32_output_and_strided_queries(D, form):
    _check(form, y_dtype=F32, seq=[50, 130, 700], new=[2, 9, 1], D=D, wide=40, seed=12)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("y_dtype", [BF, F32])
def test_sharp_scores(y_dtype, form):
    """Scores of spread 8: single tokens dominate, maxima move late."""
    _check(form, y_dtype=y_dtype, seq=[500, 77], new=[1, 40], seed=13, q_std=8.0)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("way", [1, -1])
def test_growing_and_falling_scores(way, form):
    """Every later (or earlier) tile's scores exceed the others by far: each tile moves the running maximum, or none."""
    c = HeadCase(seq=[400], new=[20], seed=14)
    for j in range(400):
        c.put(0, j, k=c.k[0][j] * (0.05 + (j if way > 0 else 399 - j) / 40.0))
    check_heads(c.run(DEV, form), c.ref())


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("size", [1e4, 1e17])
def test_scores_of_any_size(size, form):
    """One token's score is far above or below all others': its value alone, or the rest without it."""
    c = HeadCase(seq=[150, 90], new=[3, 40], H=4, G=2, seed=14)
    for b, j in ((0, 70), (1, 3)):
        c.put(b, j, k=c.k[b][j] * size)
    (y, lse), (ry, rl, ya, sa) = c.run(DEV, form), c.ref()
    # sa is as large as the score here: rows that the token wins or loses outright are checked by value
    assert np.all(np.isfinite(y)) and np.all(np.isfinite(lse))
    assert np.all(np.abs(y - ry) <= 4 * 2.0 ** -8 * (ya + np.abs(ry)) + 1e-30)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("which", ["k", "v", "kv"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf"), 3.3e38])
def test_unseen_tokens_may_hold_anything(bad, which, form):
    """The last of five new tokens is garbage: the four before it do not see it (the cache's unowned rows are NaN always)."""
    c = HeadCase(seq=[70, 130], new=[5, 2], seed=15)
    row = torch.full((c.G, c.D), bad, dtype=BF)
    c.put(0, 69, k=row if "k" in which else None, v=row if "v" in which else None)
    got, ref = c.run(DEV, form), c.ref()
    check_heads(got, ref, rows=[0, 1, 2, 3, 5, 6])
    if bad != bad:
        assert np.all(np.isnan(got[0][4]))


@pytest.mark.parametrize("form", FORMS + ["split tree", "whole tree"])
@pytest.mark.parametrize("at", [3, 64, 66])
def test_values_without_a_number_reach_who_sees_them(at, form):
    """Infinities and NaNs in single places of a seen value (before the new tokens or among them) are in those places
    of the results that see it, and in no others."""
    new = 6
    tree = chain_tree([new], 1) if "tree" in form else None
    c = HeadCase(seq=[70], new=[new], seed=16, tree=tree)
    v = c.v[0][at].clone()
    v[:, 5], v[:, 17], v[:, 100] = float("inf"), float("nan"), -float("inf")
    c.put(0, at, v=v)
    got = c.run(DEV, form.split()[0])
    clean = c.v[0][at].clone()
    clean[:, [5, 17, 100]] = 0.0
    c.put(0, at, v=clean)
    ref = c.ref()
    y = got[0]
    for t in range(new):
        sees = at < 64 + t + 1
        assert np.all(y[t, :, 5] == np.inf) == sees and np.all(np.isnan(y[t, :, 17])) == sees
        assert np.all(y[t, :, 100] == -np.inf) == sees
    keep = [d for d in range(128) if d not in (5, 17, 100)]
    check_heads((y[:, :, keep], got[1]), (ref[0][:, :, keep], ref[1], ref[2][:, :, keep], ref[3]))


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("y_dtype", [BF, F32])
def test_several_values_without_a_number_in_one_place(y_dtype, D, form):
    """Infinities of one sign add up to one, of both signs to NaN, over tiles and pieces."""
    c = HeadCase(seq=[3000], new=[9], H=16, G=2, D=D, seed=16)
    for at, signs in ((3, (1, 1)), (70, (0, -1)), (2995, (1, 0))):
        v = c.v[0][at].clone()
        for d, sign in zip((2, D - 1), signs):
            if sign:
                v[:, d] = sign * float("inf")
        c.put(0, at, v=v)
    y, _ = c.run(DEV, form, y_dtype=y_dtype)
    assert np.all(y[:, :, 2] == np.inf) and np.all(np.isnan(y[:, :, D - 1]))
    keep = [d for d in range(D) if d not in (2, D - 1)]
    for at in (3, 70, 2995):
        v = c.v[0][at].clone()
        v[:, [2, D - 1]] = 0.0
        c.put(0, at, v=v)
    got, ref = c.run(DEV, form, y_dtype=y_dtype), c.ref()
    check_heads(got, ref, y_dtype)
    # (weights of 2^-9 and less of the values' own make no difference to the other places)
    assert np.array_equal(got[0][:, :, keep], y[:, :, keep])


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("H,G", [(64, 8), (32, 2), (48, 3)])
def test_many_row_tiles_of_several_requests(H, G, form):
    """More row tiles than run at a time: the latest in their requests go first."""
    c = HeadCase(seq=[300, 17, 700, 130, 64], new=[280, 17, 200, 130, 1], H=H, G=G, D=64, pad=2, seed=17)
    check_heads(c.run(DEV, form), c.ref())


@pytest.mark.parametrize("G", [1, 2])
def test_many_requests_whose_row_tiles_are_cut(G):
    rng = np.random.default_rng(5)
    seq, new = rng.integers(1, 80, 70), np.ones(70, np.int64)
    seq[33], new[33], seq[50], new[50] = 9000, 40, 5000, 3
    _check("split", seq=seq, new=new, H=4 * G, G=G, D=64, seed=18, block=64)


@pytest.mark.parametrize("H,G,new,D", [(64, 8, 1, 128), (16, 2, 3, 64), (32, 1, 4, 128), (8, 8, 1, 128), (16, 1, 20, 64)])
def test_long_context_is_split_and_joined(H, G, new, D):
    _check("split", seq=[20000, 3], new=[new, 1], H=H, G=G, D=D, block=64, seed=16)


@pytest.mark.parametrize("form", FORMS)
def test_long_prompt(form):
    _check(form, seq=[1500], new=[1400], H=4, G=2, block=64, seed=17)


@pytest.mark.parametrize("y_dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,G,new,ctx,words", [
    (8, 2, [1], [40], 1), (8, 2, [5, 0, 13], [100, 7, 0], 1), (32, 4, [33, 64, 2], [500, 31, 1000], 2),
    (16, 2, [61, 61], [2000, 0], 3), (64, 1, [9, 30], [33, 64], 1), (4, 4, [130], [90], 5), (4, 1, [32, 31], [64, 1], 1)])
@pytest.mark.parametrize("form", FORMS)
def test_trees(form, H, G, new, ctx, words, D, y_dtype):
    rng = np.random.default_rng(sum(new) + H)
    seq = np.array(ctx) + np.array(new)
    _check(form, y_dtype=y_dtype, seq=seq, new=new, H=H, G=G, D=D, pad=3, seed=18, tree=random_tree(new, words, rng))


def test_tree_with_more_tokens_than_bits():
    """New tokens past the mask's words are seen by nobody."""
    rng = np.random.default_rng(1)
    _check("auto", seq=[100, 41], new=[40, 41], H=4, G=2, seed=19, tree=random_tree([40, 41], 2, rng)[:, :1].copy())


@pytest.mark.parametrize("form", FORMS)
def test_tree_with_empty_masks_and_an_empty_cache(form):
    _check(form, seq=[5, 3], new=[5, 3], seed=20, tree=np.zeros((8, 1), np.uint32))


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("new", [[7, 20], [61, 3]])
def test_a_chain_is_the_causal_order(new, form):
    seq = [300, 90]
    c, t = HeadCase(seq=seq, new=new, seed=21), HeadCase(seq=seq, new=new, seed=21, tree=chain_tree(new, 2))
    a, b = c.run(DEV, form), t.run(DEV, form)
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), 3.3e38])
def test_tree_tokens_off_the_path_may_hold_anything(bad, form):
    """Token 2 of five is on nobody's path."""
    tree = chain_tree([5], 1)
    tree[2] = 0
    tree &= np.uint32(~(1 << 2) & 0xFFFFFFFF)
    c = HeadCase(seq=[75], new=[5], seed=22, tree=tree)
    c.put(0, 72, k=torch.full((c.G, c.D), bad, dtype=BF), v=torch.full((c.G, c.D), bad, dtype=BF))
    check_heads(c.run(DEV, form), c.ref())


def test_auto_takes_every_call():
    for kw in (dict(seq=[200], new=[1]), dict(seq=[300], new=[200]), dict(seq=[5000, 4000], new=[64, 70], block=64),
               dict(seq=[200], new=[40], tree=chain_tree([40], 2))):
        _check("auto", seed=23, **kw)


@pytest.mark.parametrize("B,new,S", [(1, 13, 213), (1, 13, 1413), (4, 30, 463), (4, 30, 830), (16, 1, 300), (16, 1, 900), (3, 60, 1600)])
def test_auto_by_rows_and_length(B, new, S):
    _check("auto", seq=[S - 7 * b for b in range(B)], new=[new] * B, H=8, G=2, seed=23)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("new", [[2, 1, 30], [200, 40, 300]])
def test_results_repeat_bit_for_bit(new, form):
    c = HeadCase(seq=[3000, 40, 999], new=new, H=16, G=4, seed=24)
    a, b = c.run(DEV, form), c.run(DEV, form)
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("layout", ["token", "head"])
def test_cache_past_4_gib(layout, form):
    """Pages whose byte offset does not fit 32 bits."""
    c = HeadCase(seq=[100], new=[3], H=4, G=2, block=64, seed=25)
    n = (5 << 30) // (64 * 2 * 128 * 2)
    shape = (n, 64, 2, 128) if layout == "token" else (n, 2, 64, 128)
    k, v = (torch.zeros(shape, dtype=BF, device=DEV) for _ in range(2))
    if layout == "head":
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    a = c.arguments(DEV, form)
    last = torch.arange(n - 3, n)
    used = torch.as_tensor(c.table[0, :2].astype(np.int64))
    for i in range(2):
        k[int(last[i])], v[int(last[i])] = a["k_cache"][int(used[i])], a["v_cache"][int(used[i])]
    a["block_table"] = torch.tensor([[int(last[0]), int(last[1]), -1]], dtype=torch.int32, device=DEV)
    y, lse = torch.empty(3, 4, 128, dtype=BF, device=DEV), torch.empty(3, 4, device=DEV)
    caee.head_attention(**dict(a, k_cache=k, v_cache=v), y=y, lse=lse)
    check_heads((y.float().cpu().numpy().astype(np.float64), lse.cpu().numpy()), c.ref())


@pytest.mark.parametrize("form", FORMS)
def test_on_another_stream_and_captured(form):
    """A captured call, replayed with eager calls of other sizes in the same workspace between, gives the eager result."""
    c = HeadCase(seq=[900, 64, 333], new=[2, 60, 1], H=16, G=2, seed=26)
    a = c.arguments(DEV, form)
    want = torch.empty(c.T, 16, 128, dtype=BF, device=DEV)
    caee.head_attention(y=want, **a)
    y = torch.zeros_like(want)
    other = HeadCase(seq=[70], new=[5], H=16, G=2, seed=27)
    b = dict(other.arguments(DEV, form), ws=a["ws"])
    yb = torch.empty(other.T, 16, 128, dtype=BF, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        caee.head_attention(y=y, **a)
    side.synchronize()
    assert torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        caee.head_attention(y=y, **a)
    for _ in range(4):
        y.zero_()
        caee.head_attention(y=yb, **b)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)


@pytest.mark.parametrize("form", FORMS)
def test_lengths_past_the_bounds_are_left_out(form):
    """More new tokens than max_new, page numbers that are none: nothing outside the outputs is written, rows within the
    bounds of other requests are right."""
    c = HeadCase(seq=[200, 90], new=[9, 3], seed=28)
    a = c.arguments(DEV, form)
    a["block_table"][0] = 1 << 30
    a["max_new"] = 4
    a["ws"] = caee.alloc_head_workspace(a["att"], c.T, 2, 4, a["max_kv"], DEV)
    y = torch.full((c.T + 2, c.H, c.D), 7.0, dtype=BF, device=DEV)
    lse = torch.empty(c.T, c.H, device=DEV)
    caee.head_attention(y=y[1:c.T + 1], lse=lse, **a)
    torch.cuda.synchronize()
    assert torch.all(y[0] == 7.0) and torch.all(y[c.T + 1] == 7.0)
    got = y[1:c.T + 1].float().cpu().numpy().astype(np.float64), lse.cpu().numpy()
    check_heads(got, c.ref(), rows=[9, 10, 11])


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("B", [3, 70])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("junk", [(2 ** 31 - 1, 2 ** 31 - 1), (-2 ** 31, 2 ** 31 - 1), (2 ** 31 - 1, -2 ** 31), (-7, -9)])
def test_lengths_that_are_none(junk, D, B, form):
    """A request whose length and count of new tokens are junk: nothing outside the outputs is written; the lists before
    it, whose new tokens are right, have theirs."""
    new = [520] * (B - 2) + [1, 1] if B < 64 else [20] * (B - 2) + [1, 1]
    c = HeadCase(seq=[n + 30 for n in new], new=new, H=128, G=8, D=D, seed=28)
    a = c.arguments(DEV, form)
    a["plan"]["seq_len"][B - 1], a["plan"]["cu_new"][B] = junk
    y = torch.full((c.T + 2, c.H, c.D), 7.0, dtype=BF, device=DEV)
    lse = torch.empty(c.T, c.H, device=DEV)
    caee.head_attention(y=y[1:c.T + 1], lse=lse, **a)
    torch.cuda.synchronize()
    assert torch.all(y[0] == 7.0) and torch.all(y[c.T + 1] == 7.0)
    got = y[1:c.T + 1].float().cpu().numpy().astype(np.float64), lse.cpu().numpy()
    if junk[1] > 0:
        check_heads(got, c.ref(), rows=range(c.T - 1))


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("new", [2, 60])
def test_infinite_keys_count_by_their_scores(new, form):
    """One infinity in a key of one group: +inf where the query is positive there, which is NaN, -inf where it is
    negative, which leaves the token out."""
    c = HeadCase(seq=[150], new=[new], H=4, G=2, seed=31)
    k = c.k[0][40].clone()
    k[1, 9] = float("inf")
    c.put(0, 40, k=k)
    y, lse = c.run(DEV, form)
    up = (c.q[:, :, 9] > 0).numpy() & (np.arange(4) // 2 == 1)
    assert np.all(np.isnan(y[up])) and np.all(np.isnan(lse[up]))
    k[1, 9] = 0.0
    c.put(0, 40, k=k)
    ry, rl, ya, sa = c.ref()
    # the token left out of the others of the group
    q64, k64, v64 = c.q.double().numpy(), c.k[0].double().numpy(), c.v[0].double().numpy()
    for t in range(new):
        for h in range(2, 4):
            if up[t, h]:
                y[t, h], lse[t, h] = ry[t, h], rl[t, h]
                continue
            seen = [j for j in range(150 - new + t + 1) if j != 40]
            s = c.scale * k64[seen, 1] @ q64[t, h]
            w = np.exp(s - s.max())
            rl[t, h] = s.max() + np.log(w.sum())
            w /= w.sum()
            ry[t, h], ya[t, h] = w @ v64[seen, 1], w @ np.abs(v64[seen, 1])
    check_heads((y, lse), (ry, rl, ya, sa))


@pytest.mark.parametrize("form", FORMS)
def test_lengths_past_the_table_are_cut(form):
    c = HeadCase(seq=[200, 90], new=[2, 3], seed=29)
    a = c.arguments(DEV, form)
    a["plan"]["seq_len"][0] = 5000
    a["max_kv"] = 1 << 20
    y = torch.full((c.T + 2, c.H, c.D), 7.0, dtype=BF, device=DEV)
    lse = torch.empty(4, c.H * c.T // 4, device=DEV).view(-1)[:c.T * c.H].view(c.T, c.H)
    caee.head_attention(y=y[1:c.T + 1], lse=lse, **a)
    torch.cuda.synchronize()
    assert torch.all(y[0] == 7.0) and torch.all(y[c.T + 1] == 7.0)
    got = y[1:c.T + 1].float().cpu().numpy().astype(np.float64), lse.cpu().numpy()
    check_heads(got, c.ref(), rows=[2, 3, 4])


@pytest.mark.parametrize("form", FORMS + ["auto"])
def test_no_requests(form):
    i32 = dict(dtype=torch.int32, device=DEV)
    att = caee.Heads(heads=4, kv_heads=2, dim=64, scale=0.1, form=form)
    k, v = (torch.zeros(2, 16, 2, 64, dtype=BF, device=DEV) for _ in range(2))
    y, lse = torch.full((5, 4, 64), 7.0, device=DEV), torch.full((5, 4), 7.0, device=DEV)
    caee.head_attention(att, torch.zeros(5, 4, 64, dtype=BF, device=DEV), k, v, torch.zeros(0, 3, **i32),
                        dict(cu_new=torch.zeros(1, **i32), seq_len=torch.zeros(0, **i32)), y,
                        caee.alloc_head_workspace(att, 5, 0, 0, 0, DEV), 0, 0, lse=lse)
    torch.cuda.synchronize()
    assert torch.all(y == 0) and torch.all(torch.isneginf(lse))


@pytest.mark.parametrize("form", FORMS)
def test_queries_without_a_number_stay_in_their_rows(form):
    c = HeadCase(seq=[300, 90], new=[4, 30], seed=30)
    c.q[1, 3, 7] = float("nan")
    c.q[20, 0, 0] = float("inf")
    y, lse = c.run(DEV, form)
    assert np.all(np.isnan(y[1, 3])) and np.all(np.isnan(y[20, 0]))
    c.q[1, 3], c.q[20, 0] = 0.0, 0.0
    ry, rl, ya, sa = c.ref()
    for t, h in ((1, 3), (20, 0)):
        y[t, h], lse[t, h] = ry[t, h], rl[t, h]
    check_heads((y, lse), (ry, rl, ya, sa))
