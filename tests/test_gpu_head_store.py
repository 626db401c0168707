"""GPU parity of the head store: norms, rotation, rounding and the paged
writes, against the formula in float64."""
import numpy as np
import pytest
import torch

from head_cases import HALF_BF16, make_cache, store_ref
from paper_2606_29982_amd import caee

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
BF, F32 = torch.bfloat16, torch.float32


def _freq(rope, base=10000.0):
    return torch.from_numpy(base ** (-np.arange(0, rope, 2) / max(rope, 1)))


def _close(got, want, size):
    """Half a step of bf16 for the result, and for the norm, the rotation and their inputs some sixteen roundings of 32
    bits of both values of a pair."""
    tol = HALF_BF16 * want.abs() + 2.0 ** -20 * size + 1e-30
    over = ((got.double() - want).abs() / tol).max().item()
    assert over <= 1.0, over


def _run(T=37, H=8, G=2, D=128, rope=None, adjacent=False, norm=True, dtype=BF, block=16, layout="token", seed=0, far=1000,
         sliced=True, in_place=False, lost=3, eps=1e-6, size=1.0):
    rng = np.random.default_rng(seed)
    rope = D if rope is None else rope
    x = torch.from_numpy(rng.standard_normal((T, (H + 2 * G) * D)).astype(np.float32) * size).to(dtype)
    n = -(-T // block) + 2
    slots = torch.from_numpy(rng.permutation(n * block)[:T].astype(np.int64))
    bad = torch.from_numpy(rng.permutation(T)[:lost])
    slots[bad] = torch.tensor([-1, n * block, 1 << 40])[:len(bad)]
    pos = torch.from_numpy(rng.integers(-1, far, T).astype(np.int32))
    wq, wk = (torch.from_numpy((1 + 0.3 * rng.standard_normal(D)).astype(np.float32)) for _ in range(2))
    if not norm:
        wq = wk = None
    freq = _freq(rope) if rope else None
    split = lambda a: [w.view(T, -1, D) for w in a.split([H * D, G * D, G * D], 1)]  # noqa: E731
    to = lambda a: None if a is None else a.to(DEV)  # noqa: E731
    xd = to(x)
    q, k, v = split(xd) if sliced else (w.contiguous() for w in split(xd))
    kc, vc = make_cache(n, block, G, D, layout, DEV, fill=7.0)
    out = q if in_place else torch.full((T, H, D), 9.0, dtype=BF, device=DEV)
    print("store", T, H, G, D, rope, adjacent, norm, dtype, block, layout, flush=True)
    caee.head_store(q, k, v, to(slots), out, kc, vc, q_norm=to(wq), k_norm=to(wk), eps=eps, position=to(pos), freq=to(freq),
                    adjacent=adjacent)
    torch.cuda.synchronize()
    rq, rk, rv = split(x)
    _close(out.cpu(), *store_ref(rq, wq, freq, pos, adjacent, eps))
    live = (slots >= 0) & (slots < n * block)
    at = slots[live] // block, slots[live] % block
    _close(kc.cpu()[at], *(a[live] for a in store_ref(rk, wk, freq, pos, adjacent, eps)))
    assert torch.equal(vc.cpu()[at], rv[live].to(BF))
    rest = torch.ones(n, block, dtype=torch.bool)
    rest[at] = False
    assert torch.all(kc.cpu()[rest] == 7.0) and torch.all(vc.cpu()[rest] == 7.0), "a row that is nobody's was written"
    return xd, x


@pytest.mark.parametrize("T", [1, 2, 16, 33, 130, 1000])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_tokens(T, dtype):
    _run(T=T, dtype=dtype, seed=T, lost=min(3, T - 1))


@pytest.mark.parametrize("H,G", [(1, 1), (3, 1), (5, 5), (32, 8), (64, 8), (17, 17), (128, 1), (1, 64)])
@pytest.mark.parametrize("D", [64, 128])
def test_heads(H, G, D):
    _run(H=H, G=G, D=D, seed=H)


@pytest.mark.parametrize("D,rope", [(128, 0), (128, 16), (128, 48), (128, 64), (128, 96), (128, 112), (64, 0), (64, 16),
                                    (64, 32), (64, 48), (64, 64)])
@pytest.mark.parametrize("adjacent", [False, True])
def test_rotations(D, rope, adjacent):
    _run(D=D, rope=rope, adjacent=adjacent, seed=rope)


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("layout", ["token", "head", "joint", "gaps"])
@pytest.mark.parametrize("block", [1, 7, 16, 128])
def test_pages(block, layout, norm):
    _run(block=block, layout=layout, norm=norm, seed=block)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_far_positions(dtype):
    """Angles of up to 2^31 radians: reduced in 32 bits they would be off by a turn."""
    _run(T=200, far=2 ** 31 - 1, dtype=dtype, seed=5)


def test_dense_inputs_and_queries_in_place():
    _run(sliced=False, seed=6)
    _run(sliced=False, in_place=True, seed=7)
    xd, x = _run(sliced=True, in_place=True, seed=8)      # only the queries of the projection change
    assert torch.equal(xd.cpu()[:, 8 * 128:], x[:, 8 * 128:])


def test_queries_between_keys_and_values():
    """q_out in rows of the same stride as the projection's, beside its keys and values."""
    T, D = 9, 64
    wide = torch.randn(T, 6, D, device=DEV).to(BF)
    out = wide[:, 2:4]
    want = torch.empty(T, 2, D, dtype=BF, device=DEV)
    kc, vc = make_cache(1, 16, 1, D, "token", DEV)
    slots = torch.arange(T, device=DEV)
    a = dict(q_norm=torch.ones(D, device=DEV), position=torch.arange(T, device=DEV, dtype=torch.int32), freq=_freq(D).to(DEV))
    keep = wide.clone()
    caee.head_store(keep[:, 0:2], keep[:, 4:5], keep[:, 5:6], slots, want, kc, vc, **a)
    caee.head_store(wide[:, 0:2], wide[:, 4:5], wide[:, 5:6], slots, out, kc, vc, **a)
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(wide[:, [0, 1, 4, 5]], keep[:, [0, 1, 4, 5]])


def test_small_and_large_values():
    _run(size=1e-12, eps=1e-30, seed=9)
    _run(size=1e15, seed=10)


def test_zero_heads_stay_zero():
    z = torch.zeros(3, 4, 64, dtype=BF, device=DEV)
    kc, vc = make_cache(1, 16, 2, 64, "token", DEV)
    out = torch.full_like(z, 5.0)
    caee.head_store(z, z[:, :2], z[:, 2:], torch.arange(3, device=DEV), out, kc, vc, q_norm=torch.ones(64, device=DEV),
                    k_norm=torch.ones(64, device=DEV), position=torch.arange(3, device=DEV, dtype=torch.int32),
                    freq=_freq(64).to(DEV))
    torch.cuda.synchronize()
    assert torch.all(out == 0) and torch.all(kc[0, :3] == 0) and torch.all(vc[0, :3] == 0)


def test_cache_past_4_gib():
    n, D = (5 << 30) // (64 * 2 * 128 * 2), 128
    kc, vc = (torch.zeros(n, 64, 2, D, dtype=BF, device=DEV) for _ in range(2))
    x = torch.randn(2, 4, D, device=DEV).to(BF)
    slots = torch.tensor([n * 64 - 1, 5], device=DEV)
    out = torch.empty(2, 2, D, dtype=BF, device=DEV)
    caee.head_store(x[:, :2], x[:, 2:], x[:, :2], slots, out, kc, vc)
    torch.cuda.synchronize()
    assert torch.equal(kc[n - 1, 63], x[0, 2:]) and torch.equal(vc[n - 1, 63], x[0, :2]) and torch.equal(kc[0, 5], x[1, 2:])
    assert torch.count_nonzero(kc[1:n - 1]) == 0 and torch.equal(out, x[:, :2])
