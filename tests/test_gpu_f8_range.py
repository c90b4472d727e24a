"""The e4m3 layers' and the experts' calls at the ends of their ranges: values beyond binary16 and next to the end of fp32 on the way; two streams; very many
tokens, outputs and channels."""
import numpy as np
import pytest
import torch

import paper_2511_11446_amd as ql
from oracle import f8 as of
from test_gpu_f8 import _block, _close, _codes, _dev, _experts, _rng, _rows, _weights

pytestmark = pytest.mark.gpu

# rows of (token, choice) that go without a plan, through tiles of 16, of 64 and of 128 rows
PATHS = [(3, 8, 2, 256, 144, 136), (40, 8, 2, 256, 144, 136), (300, 8, 2, 256, 272, 200), (1800, 2, 2, 256, 144, 136)]


@pytest.mark.parametrize("T, E, k, K, I, N", PATHS)
@pytest.mark.parametrize("power", [17, 40])
def test_outputs_of_experts_beyond_binary16(T, E, k, K, I, N, power):
    """|o| up to 2^power, weights that bring it back: y is finite, also where a weight is 0 and where two outputs cancel."""
    g = _rng("beyond", T, E, power)
    args, res, _ = _experts(g, T, E, k, K, I, N, True)
    x, ids, weights, up, ups, down, downs = args
    w_up, w_down = _codes(up), _codes(down)
    ids[2] = 0
    xs, i, s_up = x.cpu().numpy(), ids.cpu().numpy(), ups.cpu().numpy()
    # every expert's largest output, of all tokens that it has, is brought next to 2^power (of half of the experts: the others' stay)
    _, c, s = of.quantize(xs.astype(np.float64))
    for e in range(0, E, 2):
        t = np.nonzero(i == e)[0]
        if not t.size:
            continue
        h, _ = of.gated(*(of.product(c[t], s[t], w_up[e, j], s_up[e, j])[0] for j in (0, 1)), 0.0, 0.0)
        _, hc, hs = of.quantize(h)
        o, _ = of.product(hc, hs, w_down[e], downs[e].cpu().numpy())
        downs[e] *= 2.0 ** (power - int(np.ceil(np.log2(np.abs(o).max()))))
    weights.copy_(2.0 ** (4 - power) * _dev(g.uniform(-1, 1, (T, k)).astype(np.float32)))
    weights[0, 0] = 0.0
    weights[2, 0], weights[2, 1] = 1.0, -1.0
    ref, tol = of.experts(xs, i, weights.cpu().numpy(), w_up, s_up, w_down, downs.cpu().numpy(), res)
    y = ql.experts_f8(*args, residual=_dev(res))
    assert np.isfinite(ref).all() and bool(torch.isfinite(y).all())
    _close(y, ref, tol)


@pytest.mark.parametrize("T, E, k, K, I, N", PATHS)
def test_gated_products_next_to_the_end_of_fp32(T, E, k, K, I, N):
    """silu(g) * u between 2^119 and 2^127, where 448 of them are no finite number in fp32, and outputs of ordinary size behind them."""
    g = _rng("gated", T, E)
    args, res, _ = _experts(g, T, E, k, K, I, N, True)
    x, ids, weights, up, ups, down, downs = args
    w_up, w_down = _codes(up), _codes(down)
    xs, i = x.cpu().numpy(), ids.cpu().numpy()
    _, c, s = of.quantize(xs.astype(np.float64))
    most = 0.0
    for e in range(E):
        t = np.nonzero(i == e)[0]
        if t.size:
            most = max(most, *(np.abs(of.product(c[t], s[t], w_up[e, j], ups[e, j].cpu().numpy())[0]).max() for j in (0, 1)))
    ups *= 2.0 ** (63 - int(np.ceil(np.log2(most))))        # |g| and |u| up to 2^63
    downs *= 2.0 ** -118
    with np.errstate(over="ignore"):                        # exp(-g) of large negative g
        ref, tol = of.experts(xs, i, weights.cpu().numpy(), w_up, ups.cpu().numpy(), w_down, downs.cpu().numpy(), res)
    y = ql.experts_f8(*args, residual=_dev(res))
    assert np.isfinite(ref).all() and np.isfinite(tol).all()
    _close(y, ref, tol)


def test_two_blocks_each_on_its_stream():
    """Two blocks of a mixture, each with its workspace and its stream, one behind the other there: only the two overlap.  What they give is poisoned before."""
    blocks = [_block(200, 8, 2, 256, 256, seed=2), _block(3, 8, 2, 256, 256, seed=3)]
    for _, _, _, room in blocks:
        for name in ("logits", "gu", "shared", "y", "weights"):
            room[name].fill_(float("nan"))
        room["ids"].fill_(-1)
        room["ws"].fill_(255)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for s, (step, _, _, _) in zip(streams, blocks):
            with torch.cuda.stream(s):
                step()
    torch.cuda.synchronize()
    for _, check, _, _ in blocks:
        check()


# ---- sizes whose launches have more than 2^32 threads -------------------------------------------------------------------------------

def test_routes_of_more_than_2_26_tokens():
    T = 2 ** 26 + 5
    x = torch.randint(-3, 4, (T, 2), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").half()
    ids, w = ql.route_experts(x, 1, ids=torch.full((T, 1), 7, dtype=torch.int32, device="cuda"), weights=torch.full((T, 1), 7.0, device="cuda"))
    assert torch.equal(ids[:, 0], (x[:, 1] > x[:, 0]).int()) and bool((w == 1.0).all())


def _last(shape, rows, axis):
    """e4m3 codes that are all 0 but those of the last expert's last rows."""
    codes = torch.zeros(shape, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    at = codes[-1].narrow(axis, codes.shape[axis + 1] - rows.shape[axis], rows.shape[axis])
    at.view(torch.uint8).copy_(rows.view(torch.uint8))
    return codes


@pytest.mark.parametrize("T, E, K, I, N", [(16, 1, 16, 16, 8650752), (17, 17, 16, 16, 30000128), (17, 17, 16, 15000064, 8), (1, 1, 16, 16, 2 ** 27 - 8)])
def test_experts_of_very_many_outputs_and_channels(T, E, K, I, N):
    """Rows without a plan and tiles of 16 rows; every token goes to the last expert, whose last 64 channels or outputs alone are not 0."""
    g = _rng("very many", T, I, N)
    live_i, live_n = min(I, 64), min(N, 64)
    (u, _, w_up, _), (d, _, w_down, _) = _weights(g, 2, live_i, K), _weights(g, live_n, live_i)
    up, down = _last((E, 2, I, K), u, 1), torch.zeros((E, N, I), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    down[-1].view(torch.uint8)[N - live_n:, I - live_i:] = d.view(torch.uint8)
    ups, downs = torch.full((E, 2, of.blocks(I), of.blocks(K)), 2.0 ** -9, device="cuda"), torch.full((E, of.blocks(N), of.blocks(I)), 2.0 ** -9, device="cuda")
    x = (g.standard_normal((T, K)) * 0.3).astype(np.float16)
    y = ql.experts_f8(_dev(x), torch.full((T, 1), E - 1, dtype=torch.int32, device="cuda"), torch.ones((T, 1), device="cuda"), up, ups, down, downs)
    # the live channels' place in their block does not matter: all others of it are 0
    s_up, s_down = np.full((1, 2, 1, 1), 2.0 ** -9, np.float32), np.full((1, 1, 1), 2.0 ** -9, np.float32)
    ref, tol = of.experts(x, np.zeros((T, 1), np.int32), np.ones((T, 1), np.float32), w_up[None], s_up, w_down[None], s_down)
    _close(y[:, N - live_n:], ref, tol)
    assert not N > live_n or bool((y[:, : N - live_n] == 0).all())


# ---- what is no finite number ------------------------------------------------------------------------------------------------------

NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("glu", [False, True])
def test_codes_of_what_is_no_finite_number(glu):
    """NaN is left out of a block's scale and its code alone is NaN; an infinite value makes its block's scale infinite and all its codes NaN; other blocks and rows are as without."""
    g = _rng("nan codes")
    K = 272
    x = _rows(g, 40, K)
    x[:, K // 2] = 1.0
    gate = np.concatenate([_rows(g, 40, K), x], axis=1) if glu else x       # (of [g | u] the second half is changed)
    bad = gate.copy()
    v = bad[:, -K:]
    v[1, 5], v[2, 130], v[3, 128:256], v[4, 270], v[5, 3], v[5, 4] = NAN, INF, NAN, -INF, INF, NAN
    without = gate.copy()
    w = without[:, -K:]
    w[1, 5] = 0.0                                                           # the same block without the NaN
    q, s = (t.view(torch.uint8).cpu().numpy() if t.dtype != torch.float32 else t.cpu().numpy() for t in ql.daq_quantize_f8(_dev(bad), glu=glu))
    q0, s0 = (t.view(torch.uint8).cpu().numpy() if t.dtype != torch.float32 else t.cpu().numpy() for t in ql.daq_quantize_f8(_dev(without), glu=glu))
    none = np.zeros((40, K), bool)
    none[1, 5] = none[2, 128:256] = none[3, 128:256] = none[4, 256:] = none[5, :128] = True
    assert np.array_equal((q & 0x7f) == 0x7f, none)
    assert np.array_equal(q[~none], q0[~none])
    scales = s0.copy()
    scales[2, 1] = scales[4, 2] = scales[5, 0] = INF
    scales[3, 1] = 1.0
    assert np.array_equal(s, scales)


@pytest.mark.parametrize("M, K, N", [(8, 272, 40), (30, 272, 72), (64, 4096, 4096), (200, 272, 1000), (300, 272, 500), (1100, 272, 520), (2100, 272, 2056)])
@pytest.mark.parametrize("glu", [False, True])
def test_a_row_with_a_nan_code_is_nan_and_no_other(M, K, N, glu):
    g = _rng("nan rows", M, N)
    dw, ds, _, _ = _weights(g, N, K)
    dw.view(torch.uint8)[: N // 2] = 0                                      # (0 times NaN, too)
    x = np.concatenate([_rows(g, M, K), _rows(g, M, K)], axis=1) if glu else _rows(g, M, K)
    bad = x.copy()
    bad[1, -2], bad[M - 2, -K + 7] = NAN, INF
    y, y0 = ql.qlinear_f8(_dev(bad), dw, ds, glu=glu), ql.qlinear_f8(_dev(x), dw, ds, glu=glu)
    there = torch.ones(M, dtype=torch.bool, device="cuda")
    there[1] = there[M - 2] = False
    assert bool(torch.isnan(y[~there]).all()) and torch.equal(y[there], y0[there]) and bool(torch.isfinite(y0).all())
