"""Rows of logits in which many reach the bound of the places asked for (masked, equal and rising ones), as log probabilities and as beams, against literal definitions
in binary64.  Rows of 128256 that are many are one part each, whose lanes have more than sixteen chunks.

Tolerances: a row's logarithm of its sum of exponentials is off by 2^-20 + 2^-23 m, m the mean distance to the largest logit (an exponential by 2^-22 + 2^-23 of its distance, a
sum of 32 by 2^-20); the result is rounded once, 2^-24 of it.
"""
import math

import numpy as np
import pytest
import torch

import paper_2604_15356_b200 as plc

pytestmark = pytest.mark.gpu

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
V, PLACES = 128256, 128


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    plc.build()
    return torch.device("cuda:0")


def kinds(dtype, V=V):
    """Rows of different kinds [kind][V]."""
    rng = np.random.default_rng(17)
    low = torch.finfo(TYPES[dtype]).min
    x = torch.from_numpy(rng.standard_normal((8, V)).astype(np.float32))
    few = torch.from_numpy(rng.permutation(V)[:100])
    values = torch.arange(100).float() / 4                # a step apart in each type
    x[0] = -math.inf                                      # a hundred tokens that are not masked, by -inf
    x[0, few] = values
    x[1] = 1.5                                            # all alike
    x[2] = low                                            # all of it at the lowest value
    x[3] = low                                            # a hundred that are not masked, by the lowest value
    x[3, few] = values
    x[4] = torch.arange(V).float() / V * 8                # rising, many alike
    x[5] = -math.inf                                      # one token
    x[5, V - 1] = -3.0
    x[6, ::2] = 6.0                                       # half of them alike on top
    return x.to(TYPES[dtype])                             # (and one ordinary row)


def best_of(row):
    """-> order of the places, largest logit, logarithm of the sum of exponentials, mean distance to the largest."""
    y = row.double().numpy()
    order = np.lexsort((np.arange(len(y)), -y))[:PLACES]
    e = np.exp(y - y.max())
    far = np.where(e > 0, y.max() - y, 0.0)
    return order, y.max(), math.log(e.sum()), float(e @ far / e.sum()), y


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_many_alternatives_where_many_reach_the_bound(dev, dtype):
    N = 1024
    x = kinds(dtype)
    kind = torch.arange(N) % len(x)
    on = x.to(dev)[kind.to(dev)]
    tokens = torch.tensor([[0, V - 1]], dtype=torch.int32, device=dev).expand(N, 2).contiguous()
    first = None
    for _ in range(3):
        got = plc.token_logprobs(on, tokens, PLACES)
        assert first is None or all(torch.equal(a, b) for a, b in zip(got, first))
        first = first or got
    logp, entropy, top, token = first
    for k in range(len(x)):
        order, most, l, m, y = best_of(x[k])
        mine = (kind == k).nonzero()[:, 0].to(dev)
        for t in first:
            assert torch.equal(t[mine], t[mine[:1]].expand_as(t[mine]))
        want = (y[order] - most) - l
        some = np.isfinite(want)
        assert token[mine[0]].tolist() == np.where(some, order, -1).tolist(), k
        gt = top[mine[0]].double().cpu().numpy()
        assert (gt[~some] == -np.inf).all()
        tol = 2.0 ** -20 + 2.0 ** -23 * m
        assert (np.abs(gt - np.where(some, want, 0))[some] <= (tol + 2.0 ** -24 * np.abs(np.where(some, want, 0)))[some]).all(), k
        for i, v in enumerate((0, V - 1)):
            w, g = (y[v] - most) - l, float(logp[mine[0], i])
            assert g == w if math.isinf(w) else abs(g - w) <= tol + 2.0 ** -24 * abs(w)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_beams_where_many_reach_the_bound(dev, dtype):
    """128 beams and 128 places: a beam's row is one part.  Scores of beams are far apart, or equal for equal rows."""
    W = 128
    x = kinds(dtype)
    tops = [best_of(r) for r in x]
    S = len(x) + 1
    kind = np.array([[s] * W if s < len(x) else [w % len(x) for w in range(W)] for s in range(S)])
    rng = np.random.default_rng(3)
    cum = -200.0 * np.stack([rng.permutation(W) for _ in range(S)]).astype(np.float32)
    cum[1:3] = -2.0                                       # rows that are alike, beams too: the lowest columns of the lowest row
    on = x.to(dev)[torch.from_numpy(kind.reshape(-1)).to(dev)].view(S, W, V)
    score = torch.from_numpy(cum).to(dev)
    first = None
    for _ in range(3):
        got = plc.beam_select(on, score, PLACES)
        assert first is None or all(torch.equal(a, b) for a, b in zip(got, first))
        first = first or got
    out, parent, token = (t.cpu().numpy() for t in first)
    for s in range(S):
        c, slack = [], 0.0
        for w in range(W):
            order, most, l, m, y = tops[kind[s, w]]
            slack = max(slack, 2.0 ** -20 + 2.0 ** -23 * m)
            c += [(-((y[v] - most) + (float(cum[s, w]) - l)), w, int(v)) for v in order if y[v] > -math.inf]
        c = sorted(c)[:PLACES]
        assert parent[s].tolist() == [s * W + w for _, w, _ in c] and token[s].tolist() == [v for _, _, v in c], s
        want = np.array([-f for f, _, _ in c])
        assert (np.abs(out[s] - want) <= slack + 2.0 ** -24 * np.abs(want)).all(), s


@pytest.mark.parametrize("dtype, bits", [("f16", 0xfe00), ("bf16", 0xffc0), ("f32", 0xffc00000), ("f16", 0x7e00), ("bf16", 0x7fc0), ("f32", 0x7fc00000)])
def test_rows_of_nan_have_every_place_written(dev, dtype, bits):
    """NaN of both signs: a row that is no distribution has alternatives -inf and -1 at every place, whatever was in the memory, also where few or no other logits are
    there to stand in it.  One part a row, a cluster a row, parts that a second launch joins."""
    from paper_2604_15356_b200 import serving
    api, word = serving._lib(), torch.int32 if dtype == "f32" else torch.int16
    wrapped = bits - (1 << 8 * TYPES[dtype].itemsize) if bits >> (8 * TYPES[dtype].itemsize - 1) else bits
    for N, width, n_top, some in ((3, 5, 5, 1), (3, 5, 9, 1), (2, 128, 128, 1), (3, 3, 3, 3), (3, 9000, 16, 9000), (2, 128256, 128, 128200), (200, 20000, 7, 19997), (200, 20000, 7, 20000)):
        x = torch.randn(N, width, generator=torch.Generator().manual_seed(width)).to(TYPES[dtype])
        x[1].view(word)[torch.randperm(width, generator=torch.Generator().manual_seed(1))[:some]] = wrapped
        assert int(x[1].isnan().sum()) == some
        on, tokens = x.to(dev), torch.zeros(N, 1, dtype=torch.int32, device=dev)
        need = serving._bytes(dev, api.plc_token_logprobs_workspace, N, width, n_top)
        logp, entropy = torch.full((N, 1), 7.0, device=dev), torch.full((N,), 7.0, device=dev)
        top, token = torch.full((N, n_top), 7.0, device=dev), torch.full((N, n_top), 7, dtype=torch.int32, device=dev)
        ws = torch.full((need,), 7, dtype=torch.uint8, device=dev)
        assert api.plc_token_logprobs(on.data_ptr(), serving._kind(on.dtype, ""), width, N, width, tokens.data_ptr(), 1, n_top, logp.data_ptr(), entropy.data_ptr(), top.data_ptr(),
                                      token.data_ptr(), ws.data_ptr(), need, None, torch.cuda.current_stream().cuda_stream) == plc.OK
        assert bool((token[1] == -1).all()) and bool((top[1] == -math.inf).all()), (N, width, n_top, some)
        assert bool(logp[1].isnan().all()) and bool(entropy[1].isnan())
        other = torch.log_softmax(x[0].double(), 0).sort(descending=True, stable=True)
        k = min(n_top, width)
        assert token[0, :k].tolist() == other.indices[:k].tolist() and bool((token[0, k:] == -1).all()) and bool((top[0, k:] == -math.inf).all())
        # standard normal logits: mean distance to the largest below 8, so 2^-20 + 2^-23 8 and the rounding
        assert bool(((top[0, :k].double().cpu() - other.values[:k]).abs() <= 2.0 ** -19 + 2.0 ** -24 * other.values[:k].abs()).all())


@pytest.mark.parametrize("dtype, mean, spread", [("f32", 1000.0, 1.0), ("f32", -1000.0, 1.0), ("f16", 50.0, 0.1), ("f16", -900.0, 4.0), ("bf16", -50.0, 1.0), ("f32", 0.0, 1e-4)])
@pytest.mark.parametrize("places", [1, 8, 64])
def test_places_of_logits_far_from_zero(dev, dtype, mean, spread, places):
    """Logits whose upper bits are alike, of both signs: the bound that the places go by is the k-th largest maximum itself."""
    N = 1024
    x = (torch.from_numpy(np.random.default_rng(places).standard_normal((4, V)).astype(np.float32)) * spread + mean).to(TYPES[dtype])
    on = x.to(dev).repeat(N // 4, 1)
    logp, entropy, top, token = plc.token_logprobs(on, torch.zeros(N, 1, dtype=torch.int32, device=dev), places)
    score, parent, best = plc.beam_select(on.view(N, 1, V), torch.zeros(N, 1, device=dev), places)
    assert torch.equal(token, best) and bool((parent == torch.arange(N, device=dev)[:, None]).all())
    for r in range(4):
        order, most, l, m, y = best_of(x[r])
        want = (y[order[:places]] - most) - l
        for t in (top, score):
            assert torch.equal(t.view(N // 4, 4, places)[:, r], t[r].expand(N // 4, -1))
            assert (np.abs(t[r].double().cpu().numpy() - want) <= 2.0 ** -20 + 2.0 ** -23 * m + 2.0 ** -24 * np.abs(want)).all()
        assert token[r].tolist() == order[:places].tolist() and bool((token.view(N // 4, 4, places)[:, r] == token[r]).all())
