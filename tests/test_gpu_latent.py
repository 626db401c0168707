"""GPU parity of latent attention, both forms, against the formula in
float64."""
import numpy as np
import pytest
import torch

from attention_cases import LatentCase, TOL_ALL, check_attention
from paper_2606_29982_amd import caee

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
FORMS = ["absorbed", "expanded"]


def _check(form, causal=True, y_dtype=torch.bfloat16, **kw):
    c = LatentCase(**kw)
    print("case", form, causal, {k: v for k, v in kw.items()}, flush=True)
    check_attention(c.run(DEV, form, causal, y_dtype), c.ref(causal))


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("S", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300, 1025])
def test_one_new_token(S, form):
    _check(form, seq=[S], new=[1], H=4, seed=S)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("H", [1, 3, 16, 33, 64, 65, 128])
def test_heads(H, form):
    _check(form, seq=[70, 5, 129], new=[1, 1, 1], H=H, seed=H)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("nope,latent,v", [(128, 512, 128), (64, 512, 128), (128, 512, 64), (128, 256, 128),
                                           (64, 256, 64), (128, 128, 128), (64, 128, 64)])
def test_head_layouts(nope, latent, v, form):
    _check(form, seq=[90, 200], new=[3, 40], H=5 if nope + v == 256 else 6, nope=nope, latent=latent, v=v, seed=latent + v)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("block", [1, 3, 16, 64, 100])
def test_page_sizes(block, form):
    _check(form, seq=[1, 64, 150], new=[1, 2, 30], H=8, block=block, seed=block)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("causal", [True, False])
def test_prompts_ragged(form, causal):
    _check(form, causal=causal, seq=[1, 17, 64, 255, 256, 257, 400], new=[1, 17, 64, 255, 256, 257, 300], H=2, seed=7)


@pytest.mark.parametrize("form", FORMS)
def test_prompt_behind_a_prefix(form):
    _check(form, seq=[700, 333], new=[290, 1], H=3, seed=8)


@pytest.mark.parametrize("form", FORMS)
def test_requests_without_new_tokens_and_padding(form):
    _check(form, seq=[40, 0, 9, 100, 5], new=[2, 0, 0, 1, 5], H=4, pad=11, seed=9)


@pytest.mark.parametrize("form", FORMS)
def test_more_new_tokens_than_cached_leaves_rows_empty(form):
    """seq_len below the new tokens: the first of them see nothing."""
    _check(form, seq=[3, 20], new=[7, 2], H=4, seed=10)


@pytest.mark.parametrize("form", FORMS)
def test_many_requests(form):
    rng = np.random.default_rng(11)
    seq = rng.integers(1, 90, 300)
    _check(form, seq=seq, new=np.minimum(seq, rng.integers(1, 3, 300)), H=2, latent=128, seed=11)


@pytest.mark.parametrize("form", FORMS)
def test_float32_output_and_strided_queries(form):
    _check(form, y_dtype=torch.float32, seq=[50, 130], new=[2, 9], H=4, wide=40, seed=12)


@pytest.mark.parametrize("form", FORMS)
def test_sharp_scores(form):
    """Scores of spread 6: single tokens dominate, maxima move late.  The score's rounding weighs six times as much."""
    c = LatentCase(seq=[500, 77], new=[1, 40], H=4, seed=13, q_std=6.0)
    f = 1 + 6 * 3
    check_attention(c.run(DEV, form), c.ref(), tol_all=f * TOL_ALL / 4, tol_row=f * TOL_ALL, tol_lse=6 * TOL_ALL * 2)


@pytest.mark.parametrize("form", FORMS)
def test_growing_scores(form):
    """Every later tile's scores exceed the ones before by far: each tile moves the running maximum."""
    c = LatentCase(seq=[400], new=[2], H=4, seed=14)
    for j in range(400):
        c.set_row(0, j, c.rows[0][j] * (0.05 + j / 60.0))
    got, ref = c.run(DEV, form), c.ref()
    spread = 7.0
    check_attention(got, ref, tol_all=(1 + 3 * spread) * TOL_ALL / 4, tol_row=(1 + 3 * spread) * TOL_ALL,
                    tol_lse=4 * spread * TOL_ALL)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf"), 3.3e38])
def test_unseen_tokens_may_hold_anything(bad, form):
    """The last of five new tokens is garbage: the four before it do not see it (the cache's unowned rows are NaN always)."""
    c = LatentCase(seq=[70, 130], new=[5, 2], H=4, seed=15)
    c.set_row(0, 69, torch.full((576,), bad, dtype=torch.bfloat16))
    (y, lse), (ry, rl) = c.run(DEV, form), c.ref()
    keep = [0, 1, 2, 3, 5, 6]
    check_attention((y[keep], lse[keep]), (ry[keep], rl[keep]))
    if bad != bad:
        assert np.all(np.isnan(y[4]))


@pytest.mark.parametrize("heads,new", [(128, 1), (16, 1), (32, 2), (64, 1)])
def test_long_context_is_split_and_joined(heads, new):
    _check("absorbed", seq=[20000, 3], new=[new, 1], H=heads, block=64, seed=16)


def test_long_prompt():
    _check("expanded", seq=[1500], new=[1400], H=2, block=64, seed=17)


def test_auto_takes_both_forms():
    few, many = LatentCase(seq=[200], new=[1], H=4, seed=18), LatentCase(seq=[300], new=[200], H=4, seed=18)
    for c, form in ((few, "absorbed"), (many, "expanded")):
        a, f = c.run(DEV, "auto"), c.run(DEV, form)
        assert np.array_equal(a[0], f[0]) and np.array_equal(a[1], f[1])


@pytest.mark.parametrize("form", FORMS)
def test_results_repeat_bit_for_bit(form):
    c = LatentCase(seq=[3000, 40, 999], new=[2, 1, 30], H=16, seed=19)
    a, b = c.run(DEV, form), c.run(DEV, form)
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])


def test_cache_past_4_gib():
    """Pages whose byte offset does not fit 32 bits."""
    c = LatentCase(seq=[100], new=[1], H=4, block=64, seed=20)
    n = (5 << 30) // (64 * 576 * 2)
    cache = torch.zeros((n + 2, 64, 576), dtype=torch.bfloat16, device=DEV)
    for j, page in enumerate((n, n + 1)):
        cache[page] = c.cache[int(c.table[0, j])].to(DEV)
    c.table[0, :2] = (n, n + 1)
    c.cache = cache
    for form in FORMS:
        check_attention(c.run(DEV, form), c.ref())


@pytest.mark.parametrize("form", FORMS)
def test_in_a_graph(form):
    c = LatentCase(seq=[130, 64], new=[3, 2], H=4, seed=21)
    att = caee.Latent(heads=4, nope=128, rope=64, latent=512, v=128, scale=c.scale, form=form)
    to = lambda a, dt=None: torch.as_tensor(a).to(DEV, dt)  # noqa: E731
    plan = dict(cu_new=to(c.cu_new, torch.int32), cu_kv=to(c.cu_kv, torch.int32), seq_len=to(c.seq, torch.int32))
    q, cache, table, w = to(c.q), to(c.cache), to(c.table), caee.pack_latent_weights(to(c.w_uk), to(c.w_uv))
    y = torch.empty((c.T, 4, 128), dtype=torch.bfloat16, device=DEV)
    ws = caee.alloc_latent_workspace(att, c.T, 2, 8, 400, DEV)
    call = lambda: caee.latent_attention(att, q, w, cache, table, plan, y, ws, max_new=8, max_kv=400)  # noqa: E731
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for k in range(4):
        q.copy_(torch.randn(q.shape, device=DEV).to(q.dtype))
        plan["seq_len"].copy_(to(np.array([130 - 7 * k, 64 - k]), torch.int32))
        plan["cu_kv"].copy_(to(np.array([0, 130 - 7 * k, 194 - 8 * k]), torch.int32))
        y.zero_()
        g.replay()
        torch.cuda.synchronize()
        got = y.clone()
        y.zero_()
        call()
        torch.cuda.synchronize()
        assert torch.equal(got, y) and float(y.float().abs().sum()) > 0


def test_forms_agree_on_another_stream():
    c = LatentCase(seq=[600, 31], new=[150, 31], H=4, seed=22)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        a, e = c.run(DEV, "absorbed"), c.run(DEV, "expanded")
    d = np.linalg.norm(a[0] - e[0]) / np.linalg.norm(e[0])
    assert d <= 2 * TOL_ALL


@pytest.mark.parametrize("heads,seq,block", [(128, 20000, 100), (8, 60000, 3), (64, 40000, 12)])
def test_long_context_in_pages_that_end_inside_eight_rows(heads, seq, block):
    """Several tiles a workgroup, whose rows come page by page."""
    _check("absorbed", seq=[seq, 70], new=[1, 1], H=heads, block=block, seed=block)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("B", [63, 64, 65, 200])
def test_numbers_of_requests(B, form):
    rng = np.random.default_rng(B)
    seq = rng.integers(0, 90, B)
    new = np.minimum(rng.integers(0, 4, B), seq)
    _check(form, seq=list(seq), new=list(new), H=5, block=16, seed=B)


def test_few_and_many_rows_of_split_requests():
    """Partial results of a request joined by one wave a row and by four."""
    for heads, new, seq in ((128, 20, 3000), (16, 4, 9000)):
        _check("absorbed", seq=[seq, 500], new=[new, 1], H=heads, block=32, seed=new)


@pytest.mark.parametrize("form", FORMS)
def test_lengths_past_the_hosts_bound_are_cut(form):
    """Device lengths above max_kv: with max_kv = 0 no row sees a token, with one request's length it alone counts."""
    c = LatentCase(seq=[90, 40], new=[2, 3], H=4, seed=23)
    att = caee.Latent(heads=4, nope=128, rope=64, latent=512, v=128, scale=c.scale, form=form)
    to = lambda a, dt=None: torch.as_tensor(a).to(DEV, dt)  # noqa: E731
    plan = dict(cu_new=to(c.cu_new, torch.int32), cu_kv=to(c.cu_kv, torch.int32), seq_len=to(c.seq, torch.int32))
    w = caee.pack_latent_weights(to(c.w_uk), to(c.w_uv))
    for kv in (0, 90):
        y = torch.full((c.T + 2, 4, 128), 7.0, dtype=torch.bfloat16, device=DEV)
        lse = torch.full((c.T + 2, 4), 7.0, device=DEV)
        ws = caee.alloc_latent_workspace(att, c.T, 2, 3, kv, DEV)
        caee.latent_attention(att, to(c.q), w, to(c.cache), to(c.table), plan, y[1:-1], ws, max_new=3, max_kv=kv,
                              lse=lse[1:-1])
        torch.cuda.synchronize()
        assert torch.all(y[0] == 7.0) and torch.all(y[-1] == 7.0) and torch.all(lse[0] == 7.0) and torch.all(lse[-1] == 7.0)
        if kv == 0:
            assert torch.all(y[1:-1] == 0.0) and torch.all(torch.isneginf(lse[1:-1]))
        else:
            ry, rl = c.ref()
            check_attention((y[1:3].double().cpu().numpy(), lse[1:3].cpu().numpy()), (ry[:2], rl[:2]))


@pytest.mark.parametrize("heads,new", [(16, 1), (128, 1), (64, 2)])
def test_one_request_of_forty_thousand_tokens(heads, new):
    """Weights rounded to bf16 only, whole pages, one row tile and pairs of them."""
    _check("absorbed", seq=[40000], new=[new], H=heads, block=64, seed=heads)


def test_weights_of_short_contexts_keep_their_remainders():
    """Without a cached query's rounding (no nope part) and in float32 the result's error is the weights' alone: the
    remainder's 8 bits leave at most 2^-3 of a rounding to bf16, whose 2^-9 the plain weights would show."""
    c = LatentCase(seq=[700, 90], new=[1, 2], H=8, seed=24)
    c.q[..., :128] = 0
    (y, _), (ry, _) = c.run(DEV, "absorbed", y_dtype=torch.float32), c.ref()
    assert np.linalg.norm(y - ry) <= 2.0 ** -12 * np.linalg.norm(ry)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("T", [1, 10, 23, 300])
def test_rows_that_end_inside_a_request(T, causal, form):
    """Fewer query rows than the plan has new tokens: the rows there are see what they would see among all of them."""
    c = LatentCase(seq=[40, 90, 400, 7], new=[3, 20, 290, 5], H=4, seed=25)
    y, lse = c.ref(causal)
    c.T, c.q = T, c.q[:T]
    check_attention(c.run(DEV, form, causal), (y[:T], lse[:T]))


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("size", [2.0 ** 24, 2.0 ** 32, 2.0 ** 40, 2.0 ** 66, 2.0 ** 106, 2.0 ** 120])
@pytest.mark.parametrize("sign", ["below", "above", "both"])
def test_scores_of_any_size(size, sign, form):
    """Finite scores however large, all below zero among them: the largest takes the whole weight, a row's own value.

    The rotary parts alone make the scores, by one product each, so a row's largest score is at least a 256th of its
    size (the spacing of the rows' bf16 factors) above the next; the result is a value with the roundings of a weight
    of one, exact, and of the value and the result (two of 2^-9 for a row, allowed: TOL_ROW's eight)."""
    c = LatentCase(seq=[3, 100, 300], new=[1, 2, 4], H=4, seed=26)
    c.q[..., :129] = 0
    c.q[..., 129:] = 0
    c.q[..., 128] = size ** 0.5
    rng = np.random.default_rng(27)
    for b, n in enumerate(c.seq):
        factor = 1.0 + rng.permutation(int(n)) / 128.0              # n different bf16 factors, the largest anywhere
        factor = np.exp2(np.floor(factor - 1.0)) * (1.0 + (factor - 1.0) % 1.0)
        factor *= {"below": -1.0, "above": 1.0, "both": np.where(rng.random(int(n)) < 0.5, -1.0, 1.0)}[sign]
        for j in range(int(n)):
            row = c.rows[b][j].clone()
            row[c.latent:] = 0
            row[c.latent] = float(factor[j]) * size ** 0.5
            c.set_row(b, j, row)
    (y, lse), (ry, rl) = c.run(DEV, form), c.ref()
    assert np.all(np.isfinite(y)) and np.all(np.isfinite(lse))
    assert np.all(np.linalg.norm(y - ry, axis=2) <= 8 * 2.0 ** -9 * np.linalg.norm(ry, axis=2))
    assert np.all(np.abs(lse - rl) <= 1e-6 * np.abs(rl))


def _needs_memory(gib):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info(DEV)[0] < gib << 30:
        pytest.skip(f"{gib} GiB of device memory")


def test_requests_times_heads_past_a_launchs_threads():
    """65536 requests of one token, 128 heads: 2^23 query tiles of 512 threads.  A row's result is its own value."""
    _needs_memory(24)
    B, H, R, V = 65536, 128, 128, 64
    g = torch.Generator(device=DEV).manual_seed(28)
    rand = lambda *s: torch.randn(s, generator=g, device=DEV).to(torch.bfloat16)  # noqa: E731
    w = caee.pack_latent_weights(rand(H, 64, R) * R ** -0.5, rand(H, V, R) * R ** -0.5)
    cache, q = rand(B, 1, R + 64), rand(B, H, 128)
    i32 = dict(dtype=torch.int32, device=DEV)
    table = torch.randperm(B, generator=g, device=DEV).to(torch.int32)[:, None]
    plan = dict(cu_new=torch.arange(B + 1, **i32), cu_kv=torch.arange(B + 1, **i32), seq_len=torch.ones(B, **i32))
    att = caee.Latent(heads=H, nope=64, rope=64, latent=R, v=V, scale=0.1, form="expanded")
    y = torch.full((B, H, V), 7.0, dtype=torch.bfloat16, device=DEV)
    ws = caee.alloc_latent_workspace(att, B, B, 1, B, DEV)
    caee.latent_attention(att, q, w, cache, table, plan, y, ws, max_new=1, max_kv=B)
    torch.cuda.synchronize()
    for h in (0, 1, 63, 127):
        want = cache[table[:, 0].long(), 0, :R].double() @ w["w_uv"][h].double().t()
        d = (y[:, h].double() - want).norm(dim=1) / want.norm(dim=1)
        assert float(d.max()) <= 8 * 2.0 ** -9       # a value's and a result's rounding, of a row


def test_rows_past_a_launchs_threads():
    """2^26 query rows, a wave each where partial results are joined.  A sample of them against the formula."""
    _needs_memory(130)
    T, H, R, V, S = 1 << 20, 64, 128, 64, 64
    g = torch.Generator(device=DEV).manual_seed(29)
    rand = lambda *s: torch.randn(s, generator=g, device=DEV, dtype=torch.bfloat16)  # noqa: E731
    w = caee.pack_latent_weights(rand(H, 64, R) * R ** -0.5, rand(H, V, R) * R ** -0.5)
    cache, q = rand(1, S, R + 64), rand(T, H, 128)
    i32 = dict(dtype=torch.int32, device=DEV)
    plan = dict(cu_new=torch.tensor([0, T - 3], **i32), cu_kv=torch.tensor([0, S], **i32), seq_len=torch.tensor([S], **i32))
    att = caee.Latent(heads=H, nope=64, rope=64, latent=R, v=V, scale=128 ** -0.5, causal=False, form="absorbed")
    y = torch.full((T, H, V), 7.0, dtype=torch.bfloat16, device=DEV)
    ws = caee.alloc_latent_workspace(att, T, 1, T, S, DEV)
    caee.latent_attention(att, q, w, cache, torch.zeros((1, 1), **i32), plan, y, ws, max_new=T, max_kv=S)
    torch.cuda.synchronize()
    assert torch.all(y[T - 3:] == 0)
    c, r = cache[0, :, :R].double(), cache[0, :, R:].double()
    for t in (0, 1, 12345, T // 2, T - 5, T - 4):
        ql = torch.matmul(q[t, :, None, :64].double(), w["w_uk"].double())[:, 0]
        p = torch.softmax(128 ** -0.5 * (ql @ c.t() + q[t, :, 64:].double() @ r.t()), 1)
        want = torch.matmul(w["w_uv"].double(), (p @ c)[:, :, None])[:, :, 0]
        assert float(((y[t].double() - want).norm(dim=1) / want.norm(dim=1)).max()) <= 8 * 2.0 ** -9
    del q, y, ws
    torch.cuda.empty_cache()


def test_remainders_are_kept_by_each_requests_own_length():
    """A short request beside one of 40000 tokens, as test_weights_of_short_contexts_keep_their_remainders: by its own
    length, not the batch's."""
    c = LatentCase(seq=[700, 40000], new=[2, 1], H=8, seed=30, block=64)
    c.q[..., :128] = 0
    (y, _), (ry, _) = c.run(DEV, "absorbed", y_dtype=torch.float32), c.ref()
    assert np.linalg.norm(y[:2] - ry[:2]) <= 2.0 ** -12 * np.linalg.norm(ry[:2])


def test_results_do_not_depend_on_the_hosts_bounds():
    """Bounds that a captured graph sets generously: max_kv at any size, max_new while it asks for one row tile."""
    c = LatentCase(seq=[700, 90], new=[1, 2], H=8, seed=31)
    att = caee.Latent(heads=8, nope=128, rope=64, latent=512, v=128, scale=c.scale, form="absorbed")
    to = lambda a, dt=None: torch.as_tensor(a).to(DEV, dt)  # noqa: E731
    plan = dict(cu_new=to(c.cu_new, torch.int32), cu_kv=to(c.cu_kv, torch.int32), seq_len=to(c.seq, torch.int32))
    w, got = caee.pack_latent_weights(to(c.w_uk), to(c.w_uv)), []
    for max_new, max_kv in ((2, 790), (8, 790), (2, 1 << 20), (5, 1 << 30)):
        y = torch.empty((c.T, 8, 128), device=DEV)
        ws = caee.alloc_latent_workspace(att, c.T, 2, max_new, max_kv, DEV)
        caee.latent_attention(att, to(c.q), w, to(c.cache), to(c.table), plan, y, ws, max_new=max_new, max_kv=max_kv)
        torch.cuda.synchronize()
        got.append(y)
    assert all(torch.equal(y, got[0]) for y in got)
