"""GPU parity of the block-scaled 8-bit product against the same codes and
scales in float64."""
import numpy as np
import pytest
import torch

from attention_cases import e4m3_codes, e4m3_values, quantise_rows, tile_weights
from paper_2606_29982_amd import caee

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def _weights(N, K, rng):
    w = torch.from_numpy(rng.standard_normal((N, K)).astype(np.float32) * 0.05)
    nb, kb = -(-N // 128), K // 128
    codes, sc = torch.empty(N, K, dtype=torch.uint8), torch.empty(nb, kb)
    for i in range(nb):
        for j in range(kb):
            b = w[128 * i:128 * i + 128, 128 * j:128 * j + 128]
            sc[i, j] = float(b.abs().max()) / 448.0 * (1 + i + 2 * j)     # every block's scale differs
            codes[128 * i:128 * i + 128, 128 * j:128 * j + 128] = e4m3_codes(b / (float(b.abs().max()) / 448.0))
    return codes, sc


def _run(M, N, K, x_dtype="bf16", y_dtype="bf16", tiled=False, x_pad=0, y_pad=0, seed=0, mutate=None):
    print(f"case M={M} N={N} K={K} {x_dtype}->{y_dtype} tiled={tiled} pads {x_pad}, {y_pad}", flush=True)
    rng = np.random.default_rng(seed + M + N + K)
    codes, ws = _weights(N, K, rng)
    x = torch.from_numpy(rng.standard_normal((M, K)).astype(np.float32))
    x *= torch.exp(torch.from_numpy(rng.standard_normal((M, 1)).astype(np.float32)))
    if x_dtype == "bf16":
        x = x.to(torch.bfloat16)
    if mutate:
        mutate(x)
    xq, xs = quantise_rows(x)
    given = x_dtype == "e4m3"
    src = xq if given else x
    wide = torch.zeros((M, K + x_pad), dtype=src.dtype)
    wide[:, :K] = src
    xd = wide.to(DEV)[:, :K]
    ydt = torch.bfloat16 if y_dtype == "bf16" else torch.float32
    buf = torch.full((M + 2, N + y_pad), 7.0, dtype=ydt, device=DEV)
    row0 = 16 if (buf.shape[1] * buf.element_size()) % 16 else 1       # keeps y 16-byte aligned
    buf = torch.full((M + 2 * row0, N + y_pad), 7.0, dtype=ydt, device=DEV)
    y = buf[row0:M + row0, :N]
    wsp = caee.alloc_block_matmul_workspace(xd, N, DEV)
    wsp.fill_(0xFF)
    caee.block_matmul(xd, (tile_weights(codes) if tiled else codes).to(DEV), ws.to(DEV), y, wsp,
                      x_scale=xs.to(DEV) if given else None,
                      layout=caee.LAYOUT_TILED if tiled else caee.LAYOUT_ROWMAJOR)
    torch.cuda.synchronize()
    out = torch.ones_like(buf, dtype=torch.bool)
    out[row0:M + row0, :N] = False
    assert torch.all(buf[out] == 7.0), "write outside y"
    X = e4m3_values(xq) * np.repeat(xs.numpy().astype(np.float64), 128, 1)
    W = e4m3_values(codes) * np.repeat(np.repeat(ws.numpy().astype(np.float64), 128, 0)[:N], 128, 1)
    ref, mass = X @ W.T, np.abs(X) @ np.abs(W).T
    got = y.float().cpu().numpy().astype(np.float64)
    # A fp32 sum of K products in any order is within K 2^-24 of the sum of
    # magnitudes (products of codes are exact), the scales add two roundings
    # per block; a bf16 result is rounded once more.
    tol = (K + 4) * 2.0 ** -24 * mass + (2.0 ** -8 * np.abs(ref) if y_dtype == "bf16" else 0.0)
    assert np.all(np.abs(got - ref) <= tol), np.max(np.abs(got - ref) / np.maximum(tol, 1e-30))
    return got, ref


@pytest.mark.parametrize("tiled", [False, True])
@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 32, 33, 64, 65, 130, 300])
def test_rows(M, tiled):
    _run(M, 272, 640, tiled=tiled)


@pytest.mark.parametrize("N", [1, 5, 16, 100, 127, 128, 129, 255, 576])
def test_columns_rowmajor(N):
    _run(7, N, 384)
    _run(70, N, 384, y_dtype="f32")


@pytest.mark.parametrize("K", [128, 256, 384, 1024, 1152, 4096, 7168])
@pytest.mark.parametrize("M", [3, 100])
def test_contraction(M, K):
    _run(M, 48, K, tiled=True, y_dtype="f32")


@pytest.mark.parametrize("x_dtype", ["bf16", "f32", "e4m3"])
@pytest.mark.parametrize("y_dtype", ["bf16", "f32"])
def test_types(x_dtype, y_dtype):
    _run(20, 144, 512, x_dtype, y_dtype, tiled=True)
    _run(90, 130, 512, x_dtype, y_dtype)


@pytest.mark.parametrize("M,N,K,tiled", [(1100, 528, 256, True), (1025, 129, 384, False), (1500, 2100, 128, False),
                                         (4000, 2064, 512, True), (3000, 3100, 640, False)])
@pytest.mark.parametrize("x_dtype,y_dtype", [("bf16", "bf16"), ("e4m3", "f32")])
def test_large(M, N, K, tiled, x_dtype, y_dtype):
    _run(M, N, K, x_dtype, y_dtype, tiled=tiled)


@pytest.mark.parametrize("x_dtype", ["bf16", "f32", "e4m3"])
def test_strided_rows(x_dtype):
    _run(40, 100, 256, x_dtype, x_pad=64, y_pad=3)
    _run(1200, 100, 256, x_dtype, x_pad=32, y_pad=4)


def test_zero_rows_and_blocks():
    def mutate(x):
        x[1] = 0
        x[2, 128:256] = 0
    got, ref = _run(4, 64, 384, mutate=mutate)
    assert np.all(got[1] == 0)


def test_results_repeat_bit_for_bit():
    a, b = _run(64, 576, 7168, y_dtype="f32"), _run(64, 576, 7168, y_dtype="f32")
    assert np.array_equal(a[0], b[0])


def test_quantises_as_the_quantiser_does():
    """x quantised in the call gives the very result of the same codes handed in."""
    x = torch.randn(50, 512, device=DEV).to(torch.bfloat16)
    q = torch.empty((50, 512), dtype=torch.uint8, device=DEV)
    s = torch.empty((50, 4), dtype=torch.float32, device=DEV)
    caee.quantize_rows(x, q, s)
    codes, ws = _weights(192, 512, np.random.default_rng(5))
    w, ws = codes.to(DEV), ws.to(DEV)
    a, b = (torch.empty((50, 192), dtype=torch.float32, device=DEV) for _ in range(2))
    caee.block_matmul(x, w, ws, a, caee.alloc_block_matmul_workspace(x, 192, DEV))
    caee.block_matmul(q, w, ws, b, x_scale=s)
    torch.cuda.synchronize()
    assert torch.equal(a, b)


def test_in_a_graph_on_another_stream():
    x = torch.randn(9, 512, device=DEV).to(torch.bfloat16)
    codes, ws = _weights(96, 512, np.random.default_rng(6))
    w, ws = codes.to(DEV), ws.to(DEV)
    y = torch.empty((9, 96), dtype=torch.bfloat16, device=DEV)
    wsp = caee.alloc_block_matmul_workspace(x, 96, DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        caee.block_matmul(x, w, ws, y, wsp)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        caee.block_matmul(x, w, ws, y, wsp)
    for _ in range(4):
        x.copy_(torch.randn(9, 512, device=DEV).to(torch.bfloat16))
        y.zero_()
        g.replay()
        torch.cuda.synchronize()
        got = y.clone()
        caee.block_matmul(x, w, ws, y, wsp)
        torch.cuda.synchronize()
        assert torch.equal(got, y) and float(y.float().abs().sum()) > 0


@pytest.mark.parametrize("M,N,K,tiled", [(300, 3000, 384, False), (700, 1040, 1152, True), (1200, 701, 512, False),
                                         (130, 4096, 896, True), (65, 8200, 384, False)])
@pytest.mark.parametrize("x_dtype,y_dtype", [("bf16", "bf16"), ("e4m3", "f32")])
def test_middle(M, N, K, tiled, x_dtype, y_dtype):
    _run(M, N, K, x_dtype, y_dtype, tiled=tiled)


def test_past_four_rounds_of_tiles():
    _run(2100, 2064, 2048, tiled=True)


def test_one_row_of_an_array_of_any_width():
    """x and y of a single row, cut out of arrays whose widths no two rows could have."""
    rng = np.random.default_rng(7)
    codes, ws = _weights(144, 512, rng)
    wide = torch.randn(3, 517, device=DEV).to(torch.bfloat16)
    x, y = wide[:1, :512], torch.full((2, 147), 7.0, device=DEV)
    want = torch.empty((1, 144), device=DEV)
    call = lambda a, b: caee.block_matmul(a, codes.to(DEV), ws.to(DEV), b,  # noqa: E731
                                          caee.alloc_block_matmul_workspace(a, 144, DEV))
    call(x, y[:1, :144])
    call(x.contiguous(), want)
    torch.cuda.synchronize()
    assert torch.equal(y[:1, :144], want) and torch.all(y[0, 144:] == 7.0) and torch.all(y[1] == 7.0)


def _height(M, N, K):
    """The library's rule for many rows and a bf16 result: row tiles of 32 per workgroup, None below its sizes."""
    if -(-M // 64) * -(-N // 64) <= 2 * 256:
        return None
    rounds = lambda nt: -(-(-(-M // (32 * nt)) * -(-N // 256)) // 256)  # noqa: E731
    return min(range(8, 3, -1), key=lambda nt: rounds(nt) * (nt + 1))


@pytest.mark.parametrize("height,M,N", [(4, 705, 4112), (5, 6529, 1040), (6, 8167, 1040), (7, 1538, 7184),
                                        (8, 1797, 7184)])
@pytest.mark.parametrize("K,x_dtype,tiled", [(384, "bf16", True), (512, "e4m3", False), (640, "f32", True)])
def test_every_height_of_the_many_row_kernel(height, M, N, K, x_dtype, tiled):
    """Heights differ in loads a wave, their place among the tiles and the wait for them; contractions of 0, 1 and 2
    blocks modulo the ring of three; rows and columns end inside a tile (N inside 16 columns where rows are as stored)."""
    N = N if tiled else N - 5
    assert _height(M, N, K) == height and M % (32 * height) and N % 256
    _run(M, N, K, x_dtype, tiled=tiled)


@pytest.mark.parametrize("K,tiled", [(128, False), (256, True), (384, True), (512, False), (640, True)])
def test_many_rows_into_float32(K, tiled):
    _run(1153, 2832, K, "bf16", "f32", tiled=tiled)


def test_many_rows_of_a_long_contraction():
    """More blocks than the ring in each of its places, and row scales of every block."""
    for K in (2176, 2304, 4224):
        assert _height(1410, 4112, K) is not None
        _run(1410, 4112, K, tiled=True)


@pytest.mark.parametrize("M", [512, 513, 700])
@pytest.mark.parametrize("K,tiled", [(384, True), (1024, False)])
def test_about_two_rounds_of_tiles(M, K, tiled):
    """Both sides of the size where the many-row kernel takes over, for bf16 results."""
    assert (_height(M, 4096, K) is None) == (M == 512)
    _run(M, 4096, K, tiled=tiled)
