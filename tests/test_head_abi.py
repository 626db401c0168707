"""Host checks of the grouped-head entry points, without a GPU: every call
here is refused before anything is launched, or has nothing to do."""
import ctypes

import pytest
import torch

from paper_2606_29982_amd import caee

FAKE = 0x10000000   # aligned, never dereferenced
OK, BAD, LIMIT, WS = caee.CAEE_OK, caee.CAEE_ERR_INVALID_ARG, caee.CAEE_ERR_UNSUPPORTED, caee.CAEE_ERR_WORKSPACE
MB = 1 << 20


def _store(q=FAKE, k=FAKE + MB, v=FAKE + 2 * MB, qn=None, kn=None, freq=FAKE, pos=FAKE, slots=FAKE, out=FAKE + 3 * MB,
           kc=FAKE + 4 * MB, vc=FAKE + 5 * MB, desc=True, **kw):
    f = dict(T=0, heads=8, kv_heads=2, dim=128, rope=128, adjacent=0, x_dtype=caee.CAEE_BF16, block_size=16, n_blocks=10,
             eps=1e-6, q_stride=1024, k_stride=256, v_stride=256, q_out_stride=1024, page_stride=4096, row_stride=256,
             head_stride=128)
    f.update(kw)
    return caee.lib.caee_head_store(ctypes.byref(caee.HeadStoreDesc(**f)) if desc else None, q, k, v, qn, kn, freq, pos,
                                    slots, out, kc, vc, None)


@pytest.mark.parametrize("kw,status", [
    (dict(), OK), (dict(desc=False), BAD), (dict(T=-1), BAD), (dict(heads=0), BAD), (dict(kv_heads=0), BAD),
    (dict(dim=96), LIMIT), (dict(dim=256), LIMIT), (dict(rope=-16), BAD), (dict(rope=144), BAD), (dict(rope=24), BAD),
    (dict(adjacent=2), BAD), (dict(x_dtype=caee.CAEE_FP8_E4M3), BAD), (dict(eps=-1.0), BAD), (dict(eps=float("nan")), BAD),
    (dict(eps=float("inf")), BAD), (dict(heads=1025, q_stride=1025 * 128, q_out_stride=1025 * 128), LIMIT),
    (dict(T=(1 << 20) + 1), LIMIT), (dict(q_stride=1016), BAD), (dict(q_stride=1028), BAD), (dict(k_stride=255), BAD),
    (dict(v_stride=248), BAD), (dict(q_out_stride=1020), BAD), (dict(q_out_stride=1028), BAD), (dict(block_size=0), BAD),
    (dict(block_size=65537, page_stride=1 << 25), BAD), (dict(n_blocks=0), BAD), (dict(page_stride=4088), BAD),
    (dict(page_stride=4100), BAD), (dict(row_stride=0), BAD), (dict(row_stride=248), BAD), (dict(row_stride=260), BAD),
    (dict(head_stride=120), BAD), (dict(head_stride=0), BAD), (dict(head_stride=-128), BAD), (dict(page_stride=-4096), BAD),
    (dict(row_stride=128, head_stride=2048), OK), (dict(row_stride=128, head_stride=2040), BAD),
    (dict(kv_heads=1, head_stride=0), OK), (dict(n_blocks=1, page_stride=0), OK),
    (dict(block_size=1, row_stride=-3, page_stride=256), OK), (dict(n_blocks=1 << 30), LIMIT),
    (dict(page_stride=1 << 41), LIMIT), (dict(row_stride=1 << 27, page_stride=1 << 32), LIMIT),
    (dict(n_blocks=1 << 26, page_stride=1 << 39), LIMIT), (dict(q_stride=1 << 41), LIMIT),
    (dict(q=None, k=None, v=None, freq=None, pos=None, slots=None, out=None, kc=None, vc=None), OK),
])
def test_store_descriptor(kw, status):
    assert _store(**kw) == status
    if status != OK:
        assert caee.lib.caee_last_error().decode()


@pytest.mark.parametrize("kw", [
    dict(q=None), dict(k=FAKE + MB + 2), dict(v=None), dict(qn=FAKE + 8), dict(kn=FAKE + 4), dict(freq=None), dict(pos=None),
    dict(slots=None), dict(out=None), dict(kc=None), dict(vc=FAKE + 8), dict(kc=FAKE + 5 * MB), dict(vc=FAKE + 4 * MB + 240),
    dict(vc=FAKE + 4 * MB - 16),
    dict(out=FAKE, x_dtype=caee.CAEE_F32),                                 # over itself only in bf16,
    dict(out=FAKE, q_out_stride=1032),                                     # and of the same stride
    dict(out=FAKE + 16), dict(out=FAKE + 2048), dict(out=FAKE + MB), dict(out=FAKE + 2 * MB - 512),
    # beside the projection's keys, but reaching into them
    dict(q=FAKE, k=FAKE + 2048, v=FAKE + 2560, q_stride=1536, k_stride=1536, v_stride=1536, out=FAKE + 1024, q_out_stride=1536),
])
def test_store_refusals(kw):
    assert _store(**{"T": 4, **kw}) == BAD
    assert caee.lib.caee_last_error().decode()


def _desc(**kw):
    f = dict(T=4, B=2, heads=16, kv_heads=2, dim=128, block_size=16, n_blocks=100, max_blocks=8, max_new=2, causal=1,
             tree_words=0, form=0, y_dtype=caee.CAEE_BF16, max_kv=200, q_stride=2048, page_stride=4096, row_stride=256,
             head_stride=128, scale=0.1)
    f.update(kw)
    return caee.HeadDesc(**f)


def _ws(d):
    n = ctypes.c_size_t(0)
    return caee.lib.caee_head_workspace_size(ctypes.byref(d), ctypes.byref(n)), n.value


@pytest.mark.parametrize("kw,status", [
    (dict(), OK), (dict(T=0, B=0), OK), (dict(form=1), OK), (dict(form=2), OK), (dict(tree_words=32), OK),
    (dict(T=-1), BAD), (dict(B=-1), BAD), (dict(heads=0), BAD), (dict(kv_heads=0), BAD), (dict(kv_heads=3), BAD),
    (dict(kv_heads=32), BAD), (dict(dim=80), LIMIT), (dict(dim=0), LIMIT), (dict(block_size=0), BAD), (dict(n_blocks=0), BAD),
    (dict(max_blocks=0), BAD), (dict(max_new=-1), BAD), (dict(max_kv=-1), BAD), (dict(causal=2), BAD),
    (dict(tree_words=-1), BAD), (dict(tree_words=1, causal=0), BAD), (dict(tree_words=33), LIMIT),
    (dict(tree_words=1, form=2), OK), (dict(form=3), BAD), (dict(y_dtype=2), BAD), (dict(scale=0.0), BAD),
    (dict(scale=float("inf")), BAD), (dict(scale=3e38), BAD), (dict(q_stride=2040), BAD), (dict(q_stride=2052), BAD), (dict(q_stride=1 << 41), LIMIT),
    (dict(heads=1026, q_stride=1026 * 128), LIMIT), (dict(B=65537), LIMIT), (dict(T=(1 << 20) + 1), LIMIT),
    (dict(max_kv=(1 << 30) + 1), LIMIT), (dict(row_stride=128), BAD), (dict(page_stride=256), BAD),
    (dict(n_blocks=1 << 28), LIMIT),
])
def test_descriptor(kw, status):
    d = _desc(**kw)
    assert _ws(d)[0] == status
    if status != OK:
        assert caee.lib.caee_last_error().decode()
    assert caee.lib.caee_head_workspace_size(None, ctypes.byref(ctypes.c_size_t(0))) == BAD
    assert caee.lib.caee_head_workspace_size(ctypes.byref(d), None) == BAD


def _attend(d=None, q=FAKE, k=FAKE, v=FAKE, table=FAKE, cu=FAKE, seq=FAKE, tree=None, y=FAKE, lse=None, ws=FAKE, n=None):
    d = _desc() if d is None else d
    n = _ws(d)[1] if n is None else n
    return caee.lib.caee_head_attention(ctypes.byref(d), q, k, v, table, cu, seq, tree, y, lse, ws, n, None)


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), BAD), (dict(k=None), BAD), (dict(v=FAKE + 8), BAD), (dict(table=None), BAD), (dict(cu=None), BAD),
    (dict(seq=None), BAD), (dict(y=None), BAD), (dict(lse=FAKE + 4), BAD), (dict(d=_desc(tree_words=1)), BAD),
    (dict(d=_desc(T=0), q=None, k=None, v=None, table=None, cu=None, seq=None, y=None, ws=None), OK),
])
def test_attention_refusals(kw, status):
    assert _attend(**kw) == status


def _cpu_call(**kw):
    bf = dict(dtype=torch.bfloat16)
    a = dict(att=caee.Heads(heads=4, kv_heads=2, dim=64, scale=0.1), q=torch.zeros(2, 4, 64, **bf),
             k_cache=torch.zeros(3, 16, 2, 64, **bf), v_cache=torch.zeros(3, 16, 2, 64, **bf),
             block_table=torch.zeros(1, 2, dtype=torch.int32),
             plan=dict(cu_new=torch.zeros(2, dtype=torch.int32), seq_len=torch.zeros(1, dtype=torch.int32)),
             y=torch.zeros(2, 4, 64, **bf), ws=None, max_new=2, max_kv=2)
    a.update(kw)
    return caee.head_attention(**a)


def test_host_tensors_are_refused_before_the_library_sees_them():
    with pytest.raises(ValueError, match="device"):
        _cpu_call()
    z = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device"):
        caee.head_store(z, z, z, torch.zeros(2, dtype=torch.int64), z, z, z)


class _At(torch.Tensor):
    """A host tensor that says it is on a device."""

    def get_device(self):
        return self.index


def _said_on(index, *shape, dtype=torch.bfloat16):
    t = torch.zeros(*shape, dtype=dtype).as_subclass(_At)
    t.index = index
    return t


def test_tensors_of_other_devices_are_refused(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: 100 + i, raising=False)
    assert caee._stream_on(1) == 101
    with pytest.raises(ValueError, match="current device"):
        caee._stream_on(0)
    assert caee._on(_said_on(1, 4), 1, "slots", torch.bfloat16, (4,)) > 0
    assert caee._heads(_said_on(1, 2, 4, 64), "q", 1, 64) == (2, 4, 256)
    monkeypatch.setattr(caee, "_need", lambda t, *a: t)
    with pytest.raises(ValueError, match="slots must be on the other"):
        caee._on(_said_on(0, 4), 1, "slots", torch.bfloat16, (4,))
    with pytest.raises(ValueError, match="device"):
        caee._heads(_said_on(0, 2, 4, 64), "q", 1, 64)
    with pytest.raises(ValueError, match="device"):
        caee._head_caches(_said_on(1, 3, 16, 2, 64), _said_on(0, 3, 16, 2, 64), 1, 2, 64)
