"""Selection of a beam search's next beams on the GPU against its definition in 64 bits.

Bar of a score: the exponential's argument is rounded twice and its result once to 24 bits, and a logit's distance from the largest counts with its weight,
log V at most: 2^-24 (2 * 1.45 * log 2^18 + 2) < 2.3e-6; sums of at most 8 + 4 + 6 + 2 roundings on the way to 64 bits: 20 * 2^-24 = 1.2e-6.  Together 4e-6, and half
a step of fp32 of the score itself.  Beams and tokens are the definition's wherever its values lie further apart than twice that.
"""
import numpy as np
import pytest
import torch

import paper_2605_26678_amd as nkv

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BAR = 4e-6


def _select(x, scores, n_out, stream=None):
    """A call with room to spare around the outputs and none around the scratch."""
    P, B, V = x.shape
    need = nkv.beam_workspace_bytes(P, B, V, n_out)
    ws = torch.full((need + 512,), 255, dtype=torch.uint8, device=DEV)
    outs = [torch.full((P + 2, n_out), -7, dtype=t, device=DEV) for t in (torch.float32, torch.int32, torch.int32)]
    nkv.beam_select(x, scores, *[o[1:-1] for o in outs], ws[:need], stream=stream)
    torch.cuda.synchronize()
    assert bool((ws[need:] == 255).all()), "written behind the scratch"
    for o in outs:
        assert bool((o[0] == -7).all() and (o[-1] == -7).all()), "written beside the outputs"
    return tuple(o[1:-1].cpu().numpy() for o in outs)


def _values(x, scores):
    """[P, B * V] fp64, -inf where there is no candidate."""
    x, s = x.detach().cpu().double().numpy(), scores.cpu().double().numpy()
    with np.errstate(all="ignore"):
        top = x.max(-1, keepdims=True)
        lse = top + np.log(np.exp(x - top).sum(-1, keepdims=True))
        v = s[..., None] + (x - lse)
    return np.where(np.isfinite(v), v, -np.inf).reshape(x.shape[0], -1)


def _check(x, scores, n_out, what=""):
    got, beams, tokens = _select(x, scores, n_out)
    want = _values(x, scores)
    V = x.shape[2]
    for p in range(want.shape[0]):
        order = np.argsort(-want[p], kind="stable")[:n_out + 1]
        best = want[p][order]
        best = np.concatenate([best, np.full(max(0, n_out + 1 - best.size), -np.inf)])
        there = np.isfinite(best[:n_out])
        assert np.array_equal(np.isfinite(got[p]), there), f"{what} prompt {p}: {got[p]} for {best[:n_out]}"
        assert (beams[p][~there] == -1).all() and (tokens[p][~there] == -1).all() and np.isneginf(got[p][~there]).all(), what
        n = int(there.sum())
        at = beams[p][:n].astype(np.int64) * V + tokens[p][:n]
        assert len(set(at.tolist())) == n and (tokens[p][:n] >= 0).all() and (tokens[p][:n] < V).all(), f"{what} prompt {p}: {at}"
        bar = BAR + 2.0 ** -24 * np.abs(best[:n])
        for values in (got[p][:n], want[p][at]):
            assert (np.abs(values - best[:n]) <= bar).all(), f"{what} prompt {p}: {np.abs(values - best[:n]).max()}"
        gap = best[:-1] - best[1:] if n == n_out else np.append(best[:n][:-1] - best[1:n], np.inf)
        alone = (gap[:n] > 2 * BAR) & (np.concatenate([[np.inf], gap[:n - 1]]) > 2 * BAR)
        assert np.array_equal(at[alone], order[:n][alone]), f"{what} prompt {p}"


def _logits(P, B, V, dtype, seed, pad=0, spread=2.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = spread * torch.randn(P, B, V + pad, device=DEV, generator=g)
    return x.to(dtype)[..., :V], -8.0 * torch.rand(P, B, device=DEV, generator=g)


TYPES = [torch.bfloat16, torch.float16, torch.float32]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 63, 64, 65, 511, 2047, 2048, 2049, 8193, 20011])
def test_lengths(V, dtype):
    for P, B, n_out, pad in ((1, 1, 1, 0), (2, 3, 6, 1), (3, 5, 64, 3), (1, 33, 17, 0), (1, 1024 if V < 3000 else 100, 20, 1)):
        x, scores = _logits(P, B, V, dtype, V + B, pad)
        _check(x, scores, n_out, f"{P} x {B} x {V}, {n_out}")


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_long_stretches(dtype):
    # 1024 stretches of 8192 and more: the other number of logits a thread
    for P, B, V, n_out, pad in ((16, 8, 70001, 16, 5), (64, 16, 8192, 64, 0), (1, 32, 300000, 33, 1)):
        x, scores = _logits(P, B, V, dtype, V, pad)
        _check(x, scores, n_out, f"{P} x {B} x {V}, {n_out}")


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("left", [1, 7, 255, 419, 2047, 2048, 2049])
def test_short_last_stretches(left, dtype):
    # 640 stretches of 8192 and short ones; the best tokens among the latter's too
    x, scores = _logits(16, 8, 4 * 8192 + left, dtype, left)
    x[1::2, ..., 4 * 8192:] += 6.0
    for n_out in (1, 17, 64):
        _check(x, scores, n_out, f"{left}, {n_out}")


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_many_lists(dtype):
    """More lists than a workgroup's threads hold candidates of: the best ones in all beams, in one, in one stretch of it, equal everywhere, equal in one beam, fewer than asked for."""
    x, scores = _logits(6, 24, 33000, dtype, 11)
    scores[1], scores[1, 7] = -60.0, 0.0
    x[2, 5, 20000:20100] += 12.0
    x[3], x[4, 3] = 1.0, 2.0
    scores[4] = -1000.0
    scores[4, 3] = 0.0
    x[5] = -float("inf")
    x[5, 20, 32990:] = 1.0
    for n_out in (7, 8, 48, 64):
        _check(x, scores, n_out, f"{n_out}")
    got, beams, tokens = _select(x, scores, 64)
    assert (beams[1] == 7).all() and (beams[4] == 3).all() and tokens[4].tolist() == list(range(64))
    assert tokens[5, :10].tolist() == list(range(32990, 33000)) and (tokens[5, 10:] == -1).all()


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("V", [300, 2500, 9000])
def test_orders(V, dtype):
    """Rows that hold what is looked for side by side, in ascending and descending order, few values many times, one value only."""
    ramp = torch.arange(V, device=DEV, dtype=torch.float32) / V * 8.0
    rows = [ramp, ramp.flip(0), torch.zeros_like(ramp), (ramp * 2).floor(), torch.where(torch.arange(V, device=DEV) % 8 == 3, 5.0, -5.0),
            torch.where(torch.arange(V, device=DEV) < 40, 9.0 - ramp, 0.0)]
    x = torch.stack(rows)[None].to(dtype)
    for scores in (torch.zeros(1, 6, device=DEV), torch.arange(6, device=DEV, dtype=torch.float32)[None] * -0.4):
        for n_out in (1, 6, 64):
            _check(x, scores, n_out, f"{V}, {n_out}")
    # (equal beams: the lower one's tokens first, tokens ascending)
    same = torch.zeros(2, 3, V, device=DEV).to(dtype)
    got, beams, tokens = _select(same, torch.zeros(2, 3, device=DEV), 64)
    assert (beams == 0).all() and np.array_equal(tokens, np.tile(np.arange(64, dtype=np.int32), (2, 1)))
    one = torch.zeros(1, 3, V, device=DEV).to(dtype)
    one[..., 5] = 3.0
    got, beams, tokens = _select(one, torch.zeros(1, 3, device=DEV), 5)
    assert beams[0].tolist() == [0, 1, 2, 0, 0] and tokens[0].tolist() == [5, 5, 5, 0, 1]


def test_equal_rows_have_equal_sums_wherever_they_begin():
    V = 5003
    x, _ = _logits(1, 1, V, torch.bfloat16, 3)
    rows = torch.zeros(1, 4, V + 3, dtype=torch.bfloat16, device=DEV)      # rows begin at odd elements
    rows[..., :V] = x
    got, beams, tokens = _select(rows[..., :V], torch.zeros(1, 4, device=DEV), 8)
    assert beams[0].tolist() == [0, 1, 2, 3] * 2 and (got[0][:4] == got[0][0]).all()


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_what_is_no_candidate(dtype):
    for V in (5, 3000):
        x, scores = _logits(3, 6, V, dtype, V)
        x[0, 0] = -float("inf")
        x[0, 1, V // 2] = float("nan")
        x[0, 2, V - 1] = float("inf")
        x[0, 3, : V - 1] = -float("inf")
        scores[0, 4] = -float("inf")
        scores[1] = float("nan")
        scores[2, :5] = float("inf")
        x[2, 5, 1:] = -float("inf")
        _check(x, scores, 12, f"{V}")
        got, beams, tokens = _select(x, scores, 12)
        assert set(beams[0][beams[0] >= 0].tolist()) <= {3, 5} and (beams[1] == -1).all()
        assert tokens[2].tolist() == [0] + [-1] * 11 and beams[2, 0] == 5 and abs(got[2, 0] - float(scores[2, 5])) <= BAR


def test_scores_in_place():
    x, scores = _logits(40, 5, 3000, torch.bfloat16, 4)
    want = _select(x, scores, 5)
    ws = torch.empty(nkv.beam_workspace_bytes(40, 5, 3000, 5), dtype=torch.uint8, device=DEV)
    beams, tokens = (torch.empty(40, 5, dtype=torch.int32, device=DEV) for _ in range(2))
    nkv.beam_select(x, scores, scores, beams, tokens, ws)
    for g, w in zip((scores, beams, tokens), want):
        assert np.array_equal(g.cpu().numpy(), w)


def test_far_logits():
    x = torch.tensor([[[3e38, -3e38, 2.9e38, 0.0], [1e30, 1e30, 5.0, -1e30]]], device=DEV)
    got, beams, tokens = _select(x, torch.zeros(1, 2, device=DEV), 3)
    assert beams[0].tolist() == [0, 1, 1] and tokens[0].tolist() == [0, 0, 1] and got[0][0] == 0.0


def test_strides_streams_and_graphs():
    x, scores = _logits(6, 4, 3001, torch.float16, 9, 7)
    want = _select(x.contiguous(), scores, 8)
    wide = torch.zeros(4, 6, 3001, dtype=x.dtype, device=DEV)              # beams outside of prompts
    wide.copy_(x.transpose(0, 1))
    for g, w in zip(_select(wide.transpose(0, 1), scores, 8), want):
        assert np.array_equal(g, w)
    one = x[:1].expand(6, 4, 3001)                                         # every prompt the same logits
    for g, w in zip(_select(one, scores[:1].expand(6, 4).contiguous(), 8), want):
        assert all(np.array_equal(g[p], w[0]) for p in range(6))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for g, w in zip(_select(x, scores, 8, stream=side), want):
        assert np.array_equal(g, w)
    ws = torch.empty(nkv.beam_workspace_bytes(6, 4, 3001, 8), dtype=torch.uint8, device=DEV)
    outs = [torch.zeros(6, 8, dtype=t, device=DEV) for t in (torch.float32, torch.int32, torch.int32)]
    x = x.contiguous()
    graphs = []
    for _ in range(2):                                                     # two graphs on one scratch
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            nkv.beam_select(x, scores, *outs, ws)
        graphs.append(graph)
    for i in range(6):
        y, s = _logits(6, 4, 3001, torch.float16, 20 + i)
        x.copy_(y), scores.copy_(s)
        want = _select(y.contiguous(), s, 8)
        for o in outs:
            o.zero_()
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert np.array_equal(o.cpu().numpy(), w)
