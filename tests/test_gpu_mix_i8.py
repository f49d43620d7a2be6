"""The 8-bit mix on the GPU: codes and scales bit for bit against the
definition, products against the exact integers (whose few fp32 roundings give
the bar), in both layouts."""
import sys

import numpy as np
import pytest
import torch

from oracle import recurrent_oracle as R
from paper_1906_11367_amd import boxconv as bc

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


def rand(seed, *shape):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g) * torch.exp(torch.randn(shape[:-1] + (1,), generator=g))


def quantize(src, layout=bc.BC_TOKENS):
    if layout == bc.BC_TOKENS:
        K, rows = src.shape[-1], src.numel() // src.shape[-1]
    else:
        K, rows = src.shape[1], src.numel() // src.shape[1]
    q = torch.full((rows, bc.i8_pitch(K)), 77, dtype=torch.int8, device="cuda")
    s = torch.full((rows,), 77.0, device="cuda")
    return bc.quantize_i8(src, q, s, layout)


def check_codes(src_rows, q, s):
    """src_rows: [rows, K] fp32 numpy."""
    want_q, want_s = R.codes(src_rows)
    K = src_rows.shape[1]
    got = q.cpu().numpy()
    assert (got[:, K:] == 0).all()
    assert (got[:, :K] == want_q).all()
    assert np.array_equal(s.cpu().numpy(), want_s, equal_nan=True)


# reduction lengths around a lane's 16 values, the padding's 128 and a wave's 1024
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,K", [(1, 1), (3, 15), (5, 16), (2, 17), (7, 127), (4, 128), (6, 129), (9, 1000),
                                    (3, 1024), (2, 1025), (130, 72), (1, 5000)])
def test_codes_of_tokens(rows, K, dt):
    say("codes tokens", rows, K, dt)
    x = rand(rows * 7 + K, rows, K).to(DT[dt]).cuda()
    check_codes(x.float().cpu().numpy(), *quantize(x))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("N,K,P", [(1, 1, 1), (2, 15, 3), (1, 64, 64), (3, 130, 65), (2, 129, 200), (1, 1000, 63),
                                   (2, 1024, 77), (1, 40, 1021), (1, 2100, 40), (1, 600, 96)])
def test_codes_of_maps(N, K, P, dt):
    say("codes maps", N, K, P, dt)
    x = rand(N + K + P, N, K, P).to(DT[dt]).cuda()
    rows = x.float().cpu().numpy().transpose(0, 2, 1).reshape(N * P, K)
    check_codes(np.ascontiguousarray(rows), *quantize(x, bc.BC_MAPS))


def special_rows(K):
    rows = [np.zeros(K), np.full(K, -3.0), np.full(K, 2.0 ** -101), np.full(K, 2.0 ** -100), np.full(K, 3e38)]
    half = np.full(K, 1.0)
    half[0] = 2.0            # 1 / 2 of the largest: 63.5, a tie, to even
    rows.append(half)
    for bad in (np.nan, np.inf, -np.inf):
        v = np.linspace(-1, 1, K)
        v[K // 2] = bad
        rows.append(v)
    return np.array(rows, np.float32)


def test_codes_of_special_rows():
    """All zeros, the smallest rows that have codes and smaller ones, ties, and
    rows with a NaN or an infinity: zero codes and a NaN scale."""
    x = special_rows(70)
    check_codes(x, *quantize(torch.from_numpy(x).cuda()))
    maps = np.ascontiguousarray(x.T)[None]
    check_codes(x, *quantize(torch.from_numpy(maps).cuda(), bc.BC_MAPS))


def close(got, want, bound, out_dt):
    g = got.float().cpu().numpy().astype(np.float64)
    bound = bound + (R.U_BF16 * (np.abs(want) + bound) if out_dt == "bf16" else R.EPS * np.abs(want))
    assert np.isfinite(g).all()
    over = np.abs(g - want) - bound
    at = np.unravel_index(np.argmax(over), over.shape)
    assert over.max() <= 0, f"at {at} got {g[at]} want {want[at]} bound {bound[at]}"


def weights(seed, M, K):
    w = (torch.randn((M, K), generator=torch.Generator().manual_seed(seed)) / K ** 0.5).cuda()
    return quantize(w)


# token counts around the few-token kernels' and the tiles' sizes, odd weight
# rows, reductions of less than a padded row and of many
@pytest.mark.parametrize("T", [1, 2, 4, 5, 15, 16, 17, 24, 31, 33, 48, 64, 65, 100, 128, 129, 300])
@pytest.mark.parametrize("K,M", [(72, 40), (1000, 513), (128, 128)])
def test_tokens(T, K, M):
    say("mix tokens", T, K, M)
    wq, ws = weights(M, M, K)
    for dt, out_dt, use_bias, relu in (("bf16", "bf16", False, 0), ("f32", "f32", True, 1), ("bf16", "f32", True, 0)):
        x = rand(T + K, T, K).to(DT[dt]).cuda()
        bias = rand(M, 1, M)[0].cuda() if use_bias else None
        out = torch.full((T, M), float("nan"), dtype=DT[out_dt], device="cuda")
        bc.pointwise_mix_i8(wq, ws, x, out, bias=bias, relu=relu)
        q, s = R.codes(x.float().cpu().numpy())
        z, b = R.mix_codes(q, s, wq[:, :K].cpu().numpy(), ws.cpu().numpy(),
                           None if bias is None else bias.cpu().numpy(), relu)
        close(out, z, b, out_dt)


# sizes that take the large tiles, ragged on every side
@pytest.mark.parametrize("T,K,M", [(700, 1000, 1537), (1030, 4096, 2049), (4100, 300, 520), (2048, 640, 4096),
                                   (40, 8192, 3000), (3, 8000, 4100), (1, 4096, 8192), (256, 256, 256),
                                   (4090, 130, 4000), (2047, 500, 4090), (2040, 200, 2048), (1500, 260, 3000)])
def test_tokens_large(T, K, M):
    say("mix tokens", T, K, M)
    wq, ws = weights(M, M, K)
    x = rand(T + K, T, K).to(torch.bfloat16).cuda()
    out = torch.full((T, M), float("nan"), device="cuda")
    bc.pointwise_mix_i8(wq, ws, x, out)
    q, s = R.codes(x.float().cpu().numpy())
    z, b = R.mix_codes(q, s, wq[:, :K].cpu().numpy(), ws.cpu().numpy())
    close(out, z, b, "f32")


@pytest.mark.parametrize("N,K,P,M", [(1, 72, 1, 5), (3, 100, 7, 33), (2, 128, 64, 64), (1, 513, 65, 130),
                                     (4, 64, 300, 257), (2, 1024, 640, 256), (3, 300, 1023, 96), (2, 1024, 96, 70),
                                     (5, 2048, 130, 300), (1, 1100, 513, 512), (9, 200, 1900, 70),
                                     (1, 2100, 200, 90), (2, 4000, 70, 40), (1, 600, 500, 400), (4, 1500, 1100, 60),
                                     (2, 1200, 8256, 530), (16, 128, 1030, 40)])
def test_maps(N, K, P, M):
    say("mix maps", N, K, P, M)
    wq, ws = weights(M, M, K)
    for dt, out_dt, use_bias, relu in (("bf16", "f32", False, 1), ("f32", "bf16", True, 0)):
        x = rand(N + K + P, N, K, P).to(DT[dt]).cuda()
        bias = rand(M, 1, M)[0].cuda() if use_bias else None
        out = torch.full((N, M, P), float("nan"), dtype=DT[out_dt], device="cuda")
        bc.pointwise_mix_i8(wq, ws, x, out, layout=bc.BC_MAPS, bias=bias, relu=relu)
        rows = np.ascontiguousarray(x.float().cpu().numpy().transpose(0, 2, 1).reshape(N * P, K))
        z, b = R.mix_codes(*R.codes(rows), wq[:, :K].cpu().numpy(), ws.cpu().numpy(),
                           None if bias is None else bias.cpu().numpy(), relu)
        back = lambda v: v.reshape(N, P, M).transpose(0, 2, 1)
        close(out, back(z), back(b), out_dt)


# more tokens than a block of the kernel for few takes: blocks of one to three
# tiles of 16, and the last with fewer
@pytest.mark.parametrize("T,K,M", [(49, 4096, 30), (64, 1000, 200), (97, 300, 513), (170, 5000, 130), (400, 700, 250),
                                   (601, 200, 256), (1000, 128, 16), (4097, 260, 40), (33, 4200, 1024)])
def test_several_blocks_of_tokens(T, K, M):
    say("mix blocks of tokens", T, K, M)
    wq, ws = weights(M, M, K)
    x = rand(T + K, T, K).to(torch.bfloat16).cuda()
    z, b = R.mix_codes(*R.codes(x.float().cpu().numpy()), wq[:, :K].cpu().numpy(), ws.cpu().numpy(), None, 0)
    for out_dt in ("f32", "bf16"):
        out = torch.full((T, M), float("nan"), dtype=DT[out_dt], device="cuda")
        bc.pointwise_mix_i8(wq, ws, x, out)
        close(out, z, b, out_dt)


# sizes for which each of the products' tiles is the cheapest, few to the chip and
# many, from codes
@pytest.mark.parametrize("layout", ["tokens", "maps"])
@pytest.mark.parametrize("N,P,K,M", [(1, 100, 70, 60000), (4, 15000, 70, 100), (1, 65800, 40, 40), (1, 2047, 300, 2060),
                                     (3, 3000, 130, 200), (2, 4100, 257, 1100), (1, 700, 900, 300), (10, 210, 64, 4090)])
def test_tiles(N, P, K, M, layout):
    say("mix tiles", N, P, K, M, layout)
    maps = layout == "maps"
    rows = rand(N + K + P, N * P, K)
    q, s = quantize(rows.cuda())
    wq, ws = weights(M, M, K)
    out = torch.full((N, M, P) if maps else (N, P, M), float("nan"), device="cuda")
    if maps:
        bc.pointwise_mix_i8(wq, ws, q, out, layout=bc.BC_MAPS, x_scale=s)
    else:
        bc.pointwise_mix_i8(wq, ws, q, out, x_scale=s)
    z, b = R.mix_codes(*R.codes(rows.numpy()), wq[:, :K].cpu().numpy(), ws.cpu().numpy(), None, 0)
    back = lambda v: v.reshape(N, P, M).transpose(0, 2, 1) if maps else v.reshape(N, P, M)
    close(out, back(z), back(b), "f32")


# a row's last strip of 1 to 63 pixels, in strips of 64, 32 and 16, and rows of
# outputs that are whole runs of 64 or 16 bytes, or none
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("N,K,P,M", [(2, 90, 8, 33), (2, 300, 9, 40), (1, 520, 15, 70), (70, 40, 71, 20),
                                     (90, 140, 143, 300), (4, 1239, 138, 251), (3, 1909, 143, 704), (100, 33, 184, 17),
                                     (300, 50, 12, 9), (2, 70, 4104, 30)])
def test_last_strips(N, K, P, M, dt):
    say("mix last strips", N, K, P, M, dt)
    x = rand(N + K + P, N, K, P).to(DT[dt]).cuda()
    rows = np.ascontiguousarray(x.float().cpu().numpy().transpose(0, 2, 1).reshape(N * P, K))
    check_codes(rows, *quantize(x, bc.BC_MAPS))
    wq, ws = weights(M, M, K)
    out = torch.full((N, M, P), float("nan"), dtype=DT[dt], device="cuda")
    bc.pointwise_mix_i8(wq, ws, x, out, layout=bc.BC_MAPS)
    z, b = R.mix_codes(*R.codes(rows), wq[:, :K].cpu().numpy(), ws.cpu().numpy(), None, 0)
    back = lambda v: v.reshape(N, P, M).transpose(0, 2, 1)
    close(out, back(z), back(b), dt)


def test_extreme_codes():
    """Codes at both ends of the type (also -128, which quantize_i8 never makes)
    over a long reduction: the largest sums, exact."""
    T, K, M = 70, 32768, 66
    for a, b in ((-128, -128), (127, -128), (127, 127)):
        x = torch.full((T, K), a, dtype=torch.int8, device="cuda")
        w = torch.full((M, K), b, dtype=torch.int8, device="cuda")
        one = lambda n: torch.ones(n, device="cuda")
        for rows in (T, 20, 3):
            out = torch.empty((rows, M), device="cuda")
            bc.pointwise_mix_i8(w, one(M), x[:rows], out, x_scale=one(rows))
            assert (out == float(a * b * K)).all()
        out = torch.empty((2, M, T // 2), device="cuda")
        bc.pointwise_mix_i8(w, one(M), x, out, layout=bc.BC_MAPS, x_scale=one(T))
        assert (out == float(a * b * K)).all()


def test_codes_given_or_made_give_the_same():
    for T in (3, 20, 200):
        K, M = 500, 300
        wq, ws = weights(1, M, K)
        x = rand(2, T, K).cuda()
        q, s = quantize(x)
        a, b = torch.empty((T, M), device="cuda"), torch.empty((T, M), device="cuda")
        bc.pointwise_mix_i8(wq, ws, x, a)
        bc.pointwise_mix_i8(wq, ws, q, b, x_scale=s)
        assert torch.equal(a, b)


@pytest.mark.parametrize("T", [2, 20, 150])
def test_rows_in_larger_tensors(T):
    """Tokens as a slice of wider rows, and of batches."""
    K, M = 200, 96
    wq, ws = weights(3, M, K)
    big = torch.full((2, T, K + 56), float("nan"), dtype=torch.bfloat16, device="cuda")
    big[..., :K] = rand(4, 2, T, K).to(torch.bfloat16).cuda()
    view = big[..., :K]
    out, want = torch.empty((2, T, M), device="cuda"), torch.empty((2, T, M), device="cuda")
    bc.pointwise_mix_i8(wq, ws, view, out)
    bc.pointwise_mix_i8(wq, ws, view.contiguous(), want)
    assert torch.equal(out, want) and torch.isfinite(out).all()
    pick = big[1, ::2, :K]   # every other token
    one, ref = torch.empty((pick.shape[0], M), device="cuda"), torch.empty((pick.shape[0], M), device="cuda")
    bc.pointwise_mix_i8(wq, ws, pick, one)
    bc.pointwise_mix_i8(wq, ws, pick.contiguous(), ref)
    assert torch.equal(one, ref)


@pytest.mark.parametrize("T", [3, 20, 150])
def test_non_finite_tokens(T):
    """A token with a NaN or an infinity gives NaN outputs, and only it does."""
    K, M = 150, 80
    wq, ws = weights(5, M, K)
    x = rand(6, T, K).cuda()
    clean, out = torch.empty((T, M), device="cuda"), torch.empty((T, M), device="cuda")
    bc.pointwise_mix_i8(wq, ws, x, clean, relu=1)
    x[0, 7], x[T - 1, 149] = float("inf"), float("nan")
    bc.pointwise_mix_i8(wq, ws, x, out, relu=1)
    assert torch.isnan(out[[0, T - 1]]).all()
    assert torch.equal(out[1:T - 1], clean[1:T - 1])
    maps = torch.empty((1, M, T), device="cuda")
    bc.pointwise_mix_i8(wq, ws, x.t().contiguous()[None], maps, layout=bc.BC_MAPS, relu=1)
    assert torch.equal(maps[0].t().nan_to_num(7.0), out.nan_to_num(7.0))


def test_same_bits_on_another_stream():
    for T in (2, 24, 500):
        K, M = 1024, 700
        wq, ws = weights(7, M, K)
        x = rand(8, T, K).to(torch.bfloat16).cuda()
        a, b = torch.empty((T, M), device="cuda"), torch.empty((T, M), device="cuda")
        bc.pointwise_mix_i8(wq, ws, x, a)
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            bc.pointwise_mix_i8(wq, ws, x, b)
        s.synchronize()
        assert torch.equal(a, b)
