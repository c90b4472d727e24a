"""The e4m3 layers' and the experts' calls at the ends of their ranges: values beyond binary16 and next to the end of fp32 on the way; two streams."""
import numpy as np
import pytest
import torch

import paper_2511_11446_amd as ql
from oracle import f8 as of
from test_gpu_f8 import _block, _close, _codes, _dev, _experts, _rng

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
