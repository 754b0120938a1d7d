"""acrl_matmul_fp8 against its definition in 64 bits: exact where the operands
are small whole numbers and the scales powers of two (every layout, tail and
split shows), within the instruction's bound for random ones."""
import numpy as np
import pytest

from cases import random_bf16
from gpu_util import down, torch_dev, up, up_bf16
from operators64 import e4m3_values, product, quantize_blocks

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1, 32), (1, 16, 128), (2, 130, 96), (7, 64, 160), (16, 256, 2080), (17, 200, 512), (33, 384, 1184),
          (64, 1000, 256), (65, 129, 288), (100, 700, 640), (129, 128, 1024), (255, 257, 416), (256, 512, 384),
          (333, 520, 2080), (513, 1025, 160), (1, 4096, 4096), (40, 2048, 5120),
          # outputs in 32-row pieces, wider tiles, tiles of 256 x 256 (whole and cut ones)
          (13, 5200, 288), (64, 20000, 1056), (300, 3000, 2336), (900, 2100, 1184), (1300, 2050, 2080),
          (1290, 6700, 96), (1100, 7937, 352), (1290, 6712, 352), (1500, 2056, 416),
          # of 128 x 128 and 256 x 128: one turn, odd and even numbers of them, more than the scales held at a time
          (650, 4101, 96), (700, 4096, 128), (641, 4104, 256), (700, 4096, 1024), (700, 4100, 1184), (760, 4100, 2336),
          (1410, 4097, 64), (1520, 4100, 288), (1500, 4096, 1184), (1410, 4104, 2080)]


def _integers(shape, seed):
    """Codes of whole numbers -4 .. 4."""
    val = e4m3_values()
    codes = np.array([int(np.flatnonzero(val == v)[0]) for v in range(-4, 5)], np.uint8)
    return codes[np.random.default_rng(seed).integers(0, 9, size=shape)]


def _powers(shape, seed):
    return np.exp2(np.random.default_rng(seed).integers(-2, 3, size=shape)).astype(np.float32)


def _exact_case(M, N, K, seed):
    kb = -(-K // 128)
    return (_integers((M, K), seed), _powers((M, kb), seed + 1), _integers((N, K), seed + 2),
            _powers((-(-N // 128), kb), seed + 3))


def _run(ops, **kw):
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    return acrl.acrl_matmul_fp8(*[up(torch, dev, a) for a in ops], **kw)


def _bf16(torch, y):
    return torch.from_numpy(np.asarray(y, np.float32)).to(torch.bfloat16).float().numpy()


@pytest.mark.parametrize("M,N,K", SHAPES)
def test_exact(M, N, K):
    # sums of whole numbers times powers of two, below 2^24 units: every fp32 step is exact
    torch, dev = torch_dev()
    ops = _exact_case(M, N, K, M + N + K)
    want = product(*ops)[0]
    assert np.array_equal(down(_run(ops, out_dtype=torch.float32)), want.astype(np.float32))
    assert np.array_equal(down(_run(ops).float()), _bf16(torch, want))


@pytest.mark.parametrize("M,N,K", [(1, 300, 4096), (5, 520, 1056), (48, 640, 2048), (130, 260, 5120), (300, 400, 928)])
def test_random(M, N, K):
    torch, dev = torch_dev()
    xq, xs = quantize_blocks(random_bf16((M, K), K), 1)
    wq, ws = quantize_blocks(random_bf16((N, K), K + 1, std=0.05), 128)
    want, slack = product(xq, xs, wq, ws)
    y = down(_run((xq, xs, wq, ws), out_dtype=torch.float32))
    assert (np.abs(y - want) <= slack + 2.0 ** -24 * np.abs(want)).all(), (np.abs(y - want) / slack).max()
    assert np.linalg.norm(y - want) <= 2e-5 * np.linalg.norm(want)
    y = down(_run((xq, xs, wq, ws)).float())
    assert (np.abs(y - want) <= slack * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want)).all()


@pytest.mark.parametrize("M,N", [(3, 150), (70, 260), (200, 300)])
def test_output_slice(M, N):
    # columns of a wider matrix at odd and even row strides, what lies around them left alone
    torch, dev = torch_dev()
    ops = _exact_case(M, N, 352, 5)
    want = product(*ops)[0]
    for wide, at in ((N + 8, 8), (N + 9, 0), (N + 11, 8)):
        for dtype in (torch.bfloat16, torch.float32):
            buf = torch.full((M + 2, wide), -7.0, dtype=dtype, device=dev)
            out = buf[:M, at:at + N]
            if out.data_ptr() % 16:
                continue
            got = _run(ops, out=out)
            assert got.data_ptr() == out.data_ptr()
            ref = np.full((M + 2, wide), -7.0, np.float32)
            ref[:M, at:at + N] = want if dtype == torch.float32 else _bf16(torch, want)
            assert np.array_equal(down(buf.float()), ref)


@pytest.mark.parametrize("M", [1, 20, 65, 140])
def test_nan_scale_and_code(M):
    ops = [a.copy() for a in _exact_case(M, 270, 320, 3)]
    ops[0][M - 1, 300] = 0x7F                  # a NaN code of the last token
    ops[2][5, 17] = 0xFF                       # and of one weight row
    ops[3][1, 2] = np.nan                      # the scale of outputs 128 .. 255, last block
    y = down(_run(ops, out_dtype=torch_dev()[0].float32))
    bad = np.zeros((M, 270), bool)
    bad[M - 1] = bad[:, 5] = bad[:, 128:256] = True
    assert np.array_equal(np.isnan(y), bad)


def test_garbage_behind_the_last_rows_and_columns():
    # operands that end inside an allocation full of NaN codes: the last row's tail and the rows behind stay out
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    for M, N, K in ((3, 77, 96), (70, 130, 160), (130, 140, 416)):
        ops = _exact_case(M, N, K, 8)
        t = []
        for a in ops:
            buf = torch.full((a.size * a.itemsize + 4096,), 0x7F, dtype=torch.uint8, device=dev)
            raw = torch.from_numpy(a.view(np.uint8).reshape(-1))
            buf[:raw.numel()] = raw.to(dev)
            v = buf[:raw.numel()]
            t.append((v if a.dtype == np.uint8 else v.view(torch.float32)).reshape(a.shape))
        y = acrl.acrl_matmul_fp8(*t, out_dtype=torch.float32)
        assert np.array_equal(down(y), product(*ops)[0].astype(np.float32))


@pytest.mark.parametrize("M", [1, 20, 200])
def test_subnormal_codes_and_large_scales(M):
    # every code against whole numbers, with scales of 2^-20 .. 2^20: exact as long as one term a sum is not 0
    torch, dev = torch_dev()
    N, K = 260, 256
    xq, wq = np.zeros((M, K), np.uint8), np.zeros((N, K), np.uint8)
    codes = np.array([c for c in range(256) if c & 127 != 127], np.uint8)
    at = (7 * np.arange(M)) % K
    xq[np.arange(M), at] = codes[np.arange(M) % codes.size]
    wq[:] = _integers((N, K), 4)
    r = np.random.default_rng(6)
    xs = np.exp2(r.integers(-20, 21, (M, 2))).astype(np.float32)
    ws = np.exp2(r.integers(-20, 21, (3, 2))).astype(np.float32)
    y = _run((xq, xs, wq, ws), out_dtype=torch.float32)
    assert np.array_equal(down(y), product(xq, xs, wq, ws)[0].astype(np.float32))


@pytest.mark.parametrize("M,N,K", [(20, 64, 1 << 22), (300, 520, 1 << 21), ((1 << 20) + 3, 40, 4128), (70000, 40000, 128)])
def test_long_rows_and_offsets_past_32_bits(M, N, K):
    # codes 0 and 1, scales 1: the sums are counts
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    r, kb = torch.Generator(device=dev).manual_seed(K + M), -(-K // 128)

    def ones(rows):
        x = torch.empty((rows, K), dtype=torch.uint8, device=dev)
        step = max(1, (1 << 27) // K)
        for a in range(0, rows, step):
            x[a:a + step] = (torch.rand(x[a:a + step].shape, device=dev, generator=r) < 1 / 16).to(torch.uint8) * 0x38
        return x

    x, w = ones(M), ones(N)
    y = acrl.acrl_matmul_fp8(x, torch.ones((M, kb), device=dev), w, torch.ones((-(-N // 128), kb), device=dev),
                             out_dtype=torch.float32)
    rows = torch.tensor([0, 1, M // 2, M - 2, M - 1], device=dev)
    want = torch.zeros((5, N), device=dev)
    for a in range(0, K, 1 << 18):
        want += (x[rows, a:a + (1 << 18)] != 0).float() @ (w[:, a:a + (1 << 18)] != 0).float().t()
    assert torch.equal(y[rows], want)


def test_refusals():
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    xq, xs, wq, ws = (up(torch, dev, a) for a in _exact_case(4, 64, 256, 1))
    wide = torch.empty((4, 130), dtype=torch.bfloat16, device=dev)
    for bad in (dict(xq=xq[:, :128]), dict(x_scales=xs[:2]), dict(w_scales=ws.double()), dict(wq=wq.t()),
                dict(x_scales=xs.cpu()), dict(out=wide), dict(out=wide.t()[:4, :4]), dict(out_dtype=torch.float16),
                dict(out=wide[:, :64].half()), dict(xq=xq.float())):
        args = dict(xq=xq, x_scales=xs, wq=wq, w_scales=ws, **{})
        with pytest.raises(ValueError):
            acrl.acrl_matmul_fp8(**{**args, **bad})
    with pytest.raises(acrl.AcrlError):  # 2 bytes off 16
        acrl.acrl_matmul_fp8(xq, xs, wq, ws, out=wide[:, 1:65])


def test_no_rows_of_x():
    torch, dev = torch_dev()
    ops = _exact_case(1, 64, 128, 1)
    y = _run((ops[0][:0], ops[1][:0], ops[2], ops[3]))
    assert y.shape == (0, 64)


@pytest.mark.parametrize("M", [1, 30, 130])
def test_other_stream_and_repeats(M):
    torch, dev = torch_dev()
    ops = [up(torch, dev, a) for a in _exact_case(M, 390, 1056, 21)]
    from paper_2607_24062_amd import acrl
    want = acrl.acrl_matmul_fp8(*ops)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = acrl.acrl_matmul_fp8(*ops, stream=side)
    with torch.cuda.stream(side):
        again = acrl.acrl_matmul_fp8(*ops)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(again, want)


@pytest.mark.parametrize("M", [1, 30, 130])
def test_captured_and_replayed(M):
    # quantization and product in one graph, replayed on new inputs, with eager calls between
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    K, N = 1056, 390
    x = torch.zeros((M, K), dtype=torch.bfloat16, device=dev)
    w = up_bf16(torch, dev, random_bf16((N, K), 2))
    wq, ws = acrl.acrl_quantize_fp8(w, acrl.SCALE_BLOCK128)

    def step():
        xq, xs = acrl.acrl_quantize_fp8(x, acrl.SCALE_ROW128)
        return acrl.acrl_matmul_fp8(xq, xs, wq, ws)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = step()
    for k in range(3):
        x.copy_(up_bf16(torch, dev, random_bf16((M, K), 30 + k)))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, step())


@pytest.mark.parametrize("M,N,K", [(9, 520, 4096), (70, 300, 5120), (300, 260, 2080)])
def test_columns_ten_times_as_large(M, N, K):
    # the header's figure for activations with outlier channels, and the instruction's bound elementwise
    torch, dev = torch_dev()
    x = (random_bf16((M, K), K).astype(np.uint32) << 16).view(np.float32)
    x[:, 7::61] *= 10
    x = torch.from_numpy(x).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)
    xq, xs = quantize_blocks(x, 1)
    wq, ws = quantize_blocks(random_bf16((N, K), K + 1, std=0.05), 128)
    want, slack = product(xq, xs, wq, ws)
    y = down(_run((xq, xs, wq, ws), out_dtype=torch.float32))
    assert (np.abs(y - want) <= slack + 2.0 ** -24 * np.abs(want)).all(), (np.abs(y - want) / slack).max()
    assert np.linalg.norm(y - want) <= 3e-5 * np.linalg.norm(want)
