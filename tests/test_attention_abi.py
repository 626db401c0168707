"""Host checks of the attention block's entry points, without a GPU: every
call here is refused before anything is launched, or has nothing to do."""
import ctypes

import pytest
import torch

from paper_2606_29982_amd import caee

FAKE = 0x10000   # aligned, never dereferenced
OK, BAD, LIMIT, WS = caee.CAEE_OK, caee.CAEE_ERR_INVALID_ARG, caee.CAEE_ERR_UNSUPPORTED, caee.CAEE_ERR_WORKSPACE


def _plan(B=4, T=8, block=16, width=4, ctx=FAKE, new=FAKE, table=FAKE, free=FAKE, n_free=4, head=FAKE, out=True, **o):
    fields = dict(cu_new=FAKE, cu_kv=FAKE, seq_len=FAKE, slots=FAKE, position=None, request=None,
                  free_head=FAKE + 256, lacking=FAKE)
    fields.update(o)
    po = caee.PagedPlanOut(**fields)
    return caee.lib.caee_paged_plan(B, T, block, width, ctx, new, table, free, n_free, head,
                                    ctypes.byref(po) if out else None, None)


@pytest.mark.parametrize("kw,status", [
    (dict(B=-1), BAD), (dict(T=-1), BAD), (dict(block=0), BAD), (dict(block=65537), BAD), (dict(width=0), BAD),
    (dict(n_free=-1), BAD), (dict(out=False), BAD), (dict(ctx=None), BAD), (dict(new=FAKE + 4), BAD),
    (dict(table=None), BAD), (dict(free=None), BAD), (dict(head=None), BAD), (dict(cu_new=None), BAD),
    (dict(slots=None), BAD), (dict(position=FAKE + 8), BAD), (dict(lacking=None), BAD),
    (dict(free_head=FAKE), BAD),            # the input head may not be the output head
    (dict(B=65537), LIMIT),
])
def test_plan_refusals(kw, status):
    assert _plan(**kw) == status
    assert caee.lib.caee_last_error().decode()


def _store(T=4, latent=512, rope=64, dt=caee.CAEE_BF16, c=FAKE, cs=576, r=FAKE, rs=576, slots=FAKE, cache=FAKE, n=64):
    return caee.lib.caee_latent_store(T, latent, rope, dt, c, cs, r, rs, slots, cache, n, None)


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), BAD), (dict(latent=500), BAD), (dict(rope=0), BAD), (dict(dt=caee.CAEE_FP8_E4M3), BAD),
    (dict(cs=511), BAD), (dict(cs=577), BAD), (dict(rs=60), BAD), (dict(n=-1), BAD), (dict(c=None), BAD),
    (dict(r=FAKE + 2), BAD), (dict(slots=None), BAD), (dict(cache=None), BAD),
    (dict(T=0, c=None, r=None, slots=None, cache=None), OK),
])
def test_store_refusals(kw, status):
    assert _store(**kw) == status


def _latent_desc(**kw):
    f = dict(T=4, B=2, heads=16, nope=128, rope=64, latent=512, v=128, block_size=64, n_blocks=100, max_blocks=8,
             max_new=2, causal=1, form=0, y_dtype=caee.CAEE_BF16, max_kv=1000, q_stride=16 * 192, scale=0.1)
    f.update(kw)
    return caee.LatentDesc(**f)


def _latent_ws(d):
    n = ctypes.c_size_t(0)
    return caee.lib.caee_latent_workspace_size(ctypes.byref(d), ctypes.byref(n)), n.value


@pytest.mark.parametrize("kw,status", [
    (dict(), OK), (dict(T=0, B=0), OK), (dict(form=2), OK), (dict(nope=64, v=64, latent=128, q_stride=2048), OK),
    (dict(T=-1), BAD), (dict(B=-1), BAD), (dict(heads=0), BAD), (dict(nope=0), BAD), (dict(block_size=0), BAD),
    (dict(n_blocks=0), BAD), (dict(max_blocks=0), BAD), (dict(max_new=-1), BAD), (dict(max_kv=-1), BAD),
    (dict(causal=2), BAD), (dict(form=3), BAD), (dict(y_dtype=2), BAD), (dict(scale=0.0), BAD),
    (dict(scale=float("nan")), BAD), (dict(q_stride=16 * 192 - 8), BAD), (dict(q_stride=16 * 192 + 4), BAD),
    (dict(nope=96, q_stride=4096), LIMIT), (dict(rope=32), LIMIT), (dict(latent=384), LIMIT), (dict(v=256), LIMIT),
    (dict(heads=1025, q_stride=1025 * 192), LIMIT), (dict(B=65537), LIMIT), (dict(n_blocks=1 << 26), LIMIT),
    (dict(max_kv=1 << 31), LIMIT), (dict(max_new=1 << 20, max_kv=1 << 30, form=1), LIMIT),
])
def test_latent_descriptor(kw, status):
    d = _latent_desc(**kw)
    assert _latent_ws(d)[0] == status
    if status != OK:
        assert caee.lib.caee_last_error().decode()


def test_latent_tokens_in_all_are_bounded():
    for form in (1, 2):
        for kv in ((1 << 30) + 1, (1 << 31) - 1):
            assert _latent_ws(_latent_desc(max_kv=kv, form=form))[0] == LIMIT
    assert _latent_ws(_latent_desc(max_kv=1 << 30, form=1))[0] == OK


def test_latent_workspace_grows_with_the_call():
    for form in (1, 2):
        a, b = (_latent_ws(_latent_desc(form=form, T=t, max_kv=kv, max_new=t))[1] for t, kv in ((4, 1000), (8, 4000)))
        assert 0 < a < b


def test_auto_form_is_one_of_the_two():
    same = lambda **kw: _latent_ws(_latent_desc(form=0, **kw))[1]  # noqa: E731
    assert same() == _latent_ws(_latent_desc(form=1))[1]
    many = dict(T=600, B=2, max_new=300)
    assert same(**many) == _latent_ws(_latent_desc(form=2, **many))[1]


def _attend(d=None, q=FAKE, uk=FAKE, ukt=FAKE, uv=FAKE, cache=FAKE, table=FAKE, cu_new=FAKE, cu_kv=FAKE, seq=FAKE,
            y=FAKE, lse=None, ws=FAKE, n=None, weights=True):
    d = _latent_desc() if d is None else d
    w = caee.LatentWeights(uk, ukt, uv)
    n = _latent_ws(d)[1] if n is None else n
    return caee.lib.caee_latent_attention(ctypes.byref(d), q, ctypes.byref(w) if weights else None, cache, table,
                                          cu_new, cu_kv, seq, y, lse, ws, n, None)


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), BAD), (dict(ukt=None), BAD), (dict(uv=None), BAD), (dict(cache=FAKE + 8), BAD),
    (dict(table=None), BAD), (dict(cu_new=None), BAD), (dict(seq=None), BAD), (dict(y=None), BAD),
    (dict(lse=FAKE + 4), BAD), (dict(weights=False), BAD), (dict(ws=None), WS), (dict(ws=FAKE + 16), WS),
    (dict(n=100), WS), (dict(d=_latent_desc(form=2), uk=None), BAD), (dict(d=_latent_desc(form=2), cu_kv=None), BAD),
    (dict(d=_latent_desc(T=0), q=None, y=None, ws=None), OK),
])
def test_attention_refusals(kw, status):
    assert _attend(**kw) == status


def _bm_desc(**kw):
    f = dict(M=4, N=64, K=256, x_dtype=caee.CAEE_BF16, y_dtype=caee.CAEE_BF16, layout=0, x_stride=256, y_stride=64)
    f.update(kw)
    return caee.BlockMatmulDesc(**f)


def _bm(d, x=FAKE, xs=None, w=FAKE, ws=FAKE, y=FAKE, wsp=FAKE, n=1 << 20):
    return caee.lib.caee_block_matmul(ctypes.byref(d), x, xs, w, ws, y, wsp, n, None)


@pytest.mark.parametrize("kw,status", [
    (dict(M=-1), BAD), (dict(N=0), BAD), (dict(K=200, x_stride=256), BAD), (dict(K=0), BAD), (dict(x_dtype=7), BAD),
    (dict(y_dtype=caee.CAEE_FP8_E4M3), BAD), (dict(layout=2), BAD), (dict(layout=1, N=40), BAD),
    (dict(x_stride=255), BAD), (dict(x_stride=260), BAD), (dict(y_stride=63), BAD),
    (dict(K=65536 + 128, x_stride=65536 + 128), LIMIT),
])
def test_block_matmul_descriptor(kw, status):
    d = _bm_desc(**kw)
    n = ctypes.c_size_t(0)
    assert caee.lib.caee_block_matmul_workspace_size(ctypes.byref(d), ctypes.byref(n)) == status
    assert _bm(d) == status


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), BAD), (dict(xs=FAKE), BAD), (dict(w=FAKE + 8), BAD), (dict(ws=None), BAD), (dict(y=None), BAD),
    (dict(wsp=None), WS), (dict(wsp=FAKE + 64), WS), (dict(n=64), WS),
])
def test_block_matmul_refusals(kw, status):
    assert _bm(_bm_desc(), **kw) == status


def test_block_matmul_of_codes_needs_their_scales_and_no_workspace():
    d = _bm_desc(x_dtype=caee.CAEE_FP8_E4M3)
    assert _bm(d) == BAD
    n = ctypes.c_size_t(1)
    assert caee.lib.caee_block_matmul_workspace_size(ctypes.byref(d), ctypes.byref(n)) == OK and n.value == 0
    assert _bm(_bm_desc(M=0), x=None, y=None, wsp=None, n=0) == OK


def test_binding_refuses_tensors_that_do_not_fit():
    """What the C entry cannot see: devices, dtypes and shapes."""
    cpu = torch.zeros(4, 256)
    with pytest.raises(ValueError):
        caee.block_matmul(cpu, torch.zeros(64, 256, dtype=torch.uint8), torch.zeros(1, 2), torch.zeros(4, 64))
    with pytest.raises(ValueError):
        caee.latent_store(cpu[:, :64], cpu[:, 64:], torch.zeros(4, dtype=torch.int64), torch.zeros(4, 1, 256))
    with pytest.raises(TypeError):
        caee._code(torch.zeros(2, dtype=torch.int32))
    z = torch.zeros(2, dtype=torch.int32)
    out = caee.alloc_paged_plan(2, 4, "cpu")
    with pytest.raises(ValueError):
        caee.paged_plan(16, z, z, torch.zeros(2, 3, dtype=torch.int32), z, z[:1], out)


def test_pack_latent_weights_transposes():
    w = caee.pack_latent_weights(torch.arange(24.0).view(2, 3, 4), torch.zeros(2, 5, 4))
    assert w["w_uk_t"].shape == (2, 4, 3) and w["w_uk_t"].is_contiguous()
    assert torch.equal(w["w_uk_t"][1].t(), w["w_uk"][1])


def test_auto_form_by_new_tokens_and_prefix():
    size = lambda form, **kw: _latent_ws(_latent_desc(form=form, **kw))[1]  # noqa: E731
    for T, kv, form in ((256, 9000, 2), (255, 9000, 1), (32, 64, 2), (32, 65, 1), (31, 62, 1)):
        kw = dict(T=T, B=2, max_new=T, max_kv=kv)
        assert size(0, **kw) == size(form, **kw) != size(3 - form, **kw), (T, kv)


PLAN_READS = dict(ctx=4 * 4, new=4 * 4, free=4 * 4, head=4)
PLAN_WRITES = dict(table=4 * 4 * 4, cu_new=5 * 4, cu_kv=5 * 4, seq_len=4 * 4, slots=8 * 8, position=8 * 4, request=8 * 4,
                   free_head=4, lacking=4)


@pytest.mark.parametrize("written,other", [(w, o) for w in PLAN_WRITES for o in [*PLAN_READS, *PLAN_WRITES] if o != w])
def test_plan_refuses_what_it_writes_over_another_array(written, other):
    """The next step's ctx_len is this step's seq_len: handed in as both, the lengths change while they are read.
    The same address, and an array that begins in the last 16 bytes of the other one."""
    sizes = dict(PLAN_READS, **PLAN_WRITES)
    apart = {name: FAKE + 4096 * i for i, name in enumerate(sizes)}
    for a, b in ((written, other), (other, written)):
        for into in (0, (sizes[b] - 1) // 16 * 16):
            assert _plan(**dict(apart, **{a: apart[b] + into})) == BAD, (a, b, into)
            assert "overlaps" in caee.lib.caee_last_error().decode()


def test_binding_refuses_a_workspace_in_host_memory():
    att = caee.Latent(heads=1, nope=64, rope=64, latent=128, v=64, scale=1.0)
    ws, f = torch.zeros(1 << 10, dtype=torch.uint8), torch.zeros(1, 1, 128)
    with pytest.raises(ValueError, match="ws must be a device tensor"):
        caee.latent_attention(att, f, {}, f, f[0].int(), {}, f, ws, max_new=1, max_kv=1)
    with pytest.raises(ValueError, match="ws must be a device tensor"):
        caee.block_matmul(f[0], f[0].byte(), f[0], f[0], ws)


def test_workspaces_are_counted_in_bytes():
    class Buffer:
        is_cuda, dtype = True, torch.int64
        is_contiguous, data_ptr = (lambda self: True), (lambda self: FAKE)
        numel, element_size = (lambda self: 40), (lambda self: 8)

    assert caee._workspace(Buffer()) == (FAKE, 320) and caee._workspace(None) == (None, 0)


@pytest.mark.parametrize("rows,stride,want", [(1, 577, 576), (1, 0, 576), (1, 600, 576), (2, 600, 600), (2, 577, 577),
                                              (0, 576, 576)])
def test_a_single_row_has_no_stride(rows, stride, want):
    """A row cut out of an array of any width: nothing lies a stride away from it, so no stride is refused."""
    class Rows:
        is_cuda, shape = True, (rows, 576)
        stride = lambda self: (stride, 1)  # noqa: E731

    assert caee._rows(Rows(), "x") == want


GIB = 1 << 30


@pytest.mark.parametrize("kw,form", [
    # tokens in all past what the expanded form takes
    (dict(T=25600, B=200, max_new=200, max_kv=65534 * 256 + 1), 1), (dict(T=25600, B=200, max_new=200, max_kv=1 << 30), 1),
    (dict(T=25600, B=200, max_new=200, max_kv=65534 * 256, heads=1, q_stride=192), 2),
    # more pairs than the absorbed form counts
    (dict(T=16000, B=200, max_new=15801, max_kv=15000000, heads=32, q_stride=32 * 192), 2),
    # keys and values of more than 16 GiB: absorbed up to 256 new tokens per request where it needs less
    (dict(T=1024, B=8, max_new=128, max_kv=1000000, heads=128, q_stride=128 * 192), 1),
    (dict(T=2047, B=8, max_new=256, max_kv=1000000, heads=128, q_stride=128 * 192), 1),
    (dict(T=2048, B=8, max_new=256, max_kv=1000000, heads=128, q_stride=128 * 192), 2),
    (dict(T=1024, B=8, max_new=128, max_kv=261600, heads=128, q_stride=128 * 192), 2),
    (dict(T=1024, B=8, max_new=128, max_kv=261700, heads=128, q_stride=128 * 192), 1),
    (dict(T=100000, B=500, max_new=200, max_kv=262400, heads=128, q_stride=128 * 192), 2),
])
def test_auto_form_takes_what_either_form_takes(kw, form):
    (st, size), got = _latent_ws(_latent_desc(form=form, **kw)), _latent_ws(_latent_desc(**kw))
    assert (st, got) == (OK, (OK, size)) and _latent_ws(_latent_desc(form=3 - form, **kw)) != (OK, size)
    if form == 2 and kw["T"] < 256 * kw["B"] and size > 16 * GIB:
        assert _latent_ws(_latent_desc(form=1, **kw)) >= (LIMIT, 0) or _latent_ws(_latent_desc(form=1, **kw))[1] >= size


def test_workspace_of_either_form_is_as_the_header_says():
    d = dict(T=100, B=8, heads=128, q_stride=128 * 192, max_kv=50000, max_new=64)
    for form, most in ((1, 100 * 128 * (6 * 512 + 2 * 64) + 131072 * (512 + 2)), (2, 2 * 50000 * (128 * 256 + 64))):
        size = _latent_ws(_latent_desc(form=form, **d))[1]
        assert most <= size <= most + 8 * 256
