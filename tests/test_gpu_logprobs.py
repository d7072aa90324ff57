"""bs_token_logprobs against its fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import accept as OA
from oracle import logprobs as O
from paper_2605_08862_amd import binding as B
from paper_2605_08862_amd.runtime import LogprobScorer

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF = float("inf")


def _i32(v):
    return torch.as_tensor(np.asarray(v), dtype=torch.int32, device=DEV)


def _check(out, z, tokens, n_tokens, draft_len, temperature, n_top):
    """y = (z - m) / T is off by 2^-23 of itself (a difference, a product with a rounded 1/T: 1.5 steps of 2^-24 each), the logarithm of the sum by
    2^-23 of itself and by the sum's relative error: 3 * 2^-24 per exponential, its argument's, and additions of at most V / 256 terms in a row and a tree."""
    z = z.double().cpu().numpy()
    V, at = z.shape[1], 0
    got = {k: v.double().cpu().numpy() if v.is_floating_point() else v.cpu().numpy() for k, v in out.items()}
    for b in range(tokens.shape[0]):
        for i in range(tokens.shape[1]):
            if i >= n_tokens[b]:
                assert got["logprob"][b, i] == 0 and got["entropy"][b, i] == 0
                if n_top:
                    assert (got["top_tokens"][b, i] == -1).all() and (got["top_logprobs"][b, i] == 0).all()
                continue
            row = z[at + i]
            lp, h, top, ltop = O.row(row, tokens[b, i], temperature, n_top)
            y = np.abs((row - row.max()) / temperature)[np.isfinite(row)] if np.isfinite(row).any() else np.zeros(1)
            near = y[y < 100.0]
            spread = near.max() if near.size else 0.0                     # terms further down are below 2^-144 of the sum
            rel = 2.0 ** -24 * (4 + V / 256 + 16)
            base = rel + 2.0 ** -22 * (1 + np.log(V))

            def close(a, w, scale=1.0):
                if np.isnan(w) or np.isinf(w):
                    return (np.isnan(a) and np.isnan(w)) or a == w
                if abs(w) > 3.4028235677973366e38:                        # beyond the largest float32 by half a step: infinite there
                    return a == np.sign(w) * INF
                return abs(a - w) <= scale * base + 2.0 ** -22 * abs(w) + 2.0 ** -22 * np.log(V)
            assert close(got["logprob"][b, i], lp), (b, i, got["logprob"][b, i], lp)
            # the weighted mean of y: an exponential's relative error times |y|, summed with weights p: at most (spread + 1) times the above
            assert close(got["entropy"][b, i], h, 2.0 * (1.0 + min(spread, 2 * np.log(V) + 4))), (b, i, got["entropy"][b, i], h)
            if n_top:
                assert np.array_equal(got["top_tokens"][b, i], top), (b, i, got["top_tokens"][b, i], top)
                assert all(close(a, w) for a, w in zip(got["top_logprobs"][b, i], ltop)), (got["top_logprobs"][b, i], ltop)
        at += draft_len[b] + 1


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,n_top,temperature", [(2, 2, 1.0), (3, 0, 1.0), (33, 32, 0.7), (1000, 5, 1.3), (4096, 20, 1.0), (4999, 1, 0.5), (40001, 20, 0.8), (151936, 20, 1.0)])
def test_ragged_rows(dtype, V, n_top, temperature):
    rng = np.random.default_rng(V + n_top)
    k_max, draft_len = 3, [3, 0, 2, 1, 3]
    n_tokens = [4, 1, 2, 0, 3]
    M = sum(k + 1 for k in draft_len)
    z = torch.from_numpy(rng.normal(0, 2.5, (M, V)).astype(np.float32)).to(dtype)
    if V >= 1000:
        z[1, rng.random(V) < 0.5] = -INF                                  # a grammar's mask
        z[2, rng.random(V) < 0.9] = torch.finfo(dtype).min
        z[5, 5] += 60.0                                                   # a law that is nearly one token
    z = z.to(DEV)
    tokens = rng.integers(0, V, (5, k_max + 1))
    s = LogprobScorer(5, k_max, V, n_top, device=DEV)
    for _ in range(2):
        out = s(z, _i32(tokens), _i32(n_tokens), _i32(draft_len), temperature)
        _check(out, z, tokens, n_tokens, draft_len, temperature, n_top)
    assert s.poll_status() == 0


def test_ties_masks_and_rows_without_a_law():
    V, n_top = 1000, 8
    z = torch.zeros(9, V)
    z[1] = -INF
    z[2] = -INF
    z[2, [7, 999]] = 3.0                                                  # two tokens left
    z[3] = torch.finfo(torch.float32).min                                 # everything at the lowest value: a uniform law
    z[4, ::3] = 1.0                                                       # more ties than alternatives
    z[5, 13] = float("nan")
    z[6, 500] = INF
    z[7] = -0.0
    z[7, 600:] = 0.0                                                      # -0 and 0 are equal
    z[8] = -INF
    z[8, 77] = -1e30                                                      # one token left, far down
    tokens = np.array([[5], [5], [7], [0], [3], [2], [500], [1], [77]])
    s = LogprobScorer(9, 0, V, n_top, device=DEV)
    for dtype in (torch.float32, torch.bfloat16):
        zd = z.to(dtype)
        if dtype == torch.bfloat16:
            zd[3] = torch.finfo(dtype).min
        _check(s(zd.to(DEV), _i32(tokens)), zd, tokens, [1] * 9, [0] * 9, 1.0, n_top)
    assert s.poll_status() == 0


@pytest.mark.parametrize("V", [1001, 5003])
def test_rows_that_start_anywhere(V):
    """Odd vocabularies, and logits that start between sixteen-byte lines."""
    rng = np.random.default_rng(V)
    for dtype in (torch.float32, torch.bfloat16):
        for skip in (0, 1, 3):
            buf = torch.from_numpy(rng.normal(0, 2, 7 * V + skip).astype(np.float32)).to(dtype).to(DEV)
            z = buf[skip:].view(7, V)
            tokens = rng.integers(0, V, (7, 1))
            tokens[0], tokens[1] = 0, V - 1
            _check(LogprobScorer(7, 0, V, 6, device=DEV)(z, _i32(tokens)), z, tokens, [1] * 7, [0] * 7, 1.0, 6)


def test_faults_and_optional_outputs():
    V, k_max = 500, 2
    rng = np.random.default_rng(5)
    z = torch.from_numpy(rng.normal(0, 2, (9, V)).astype(np.float32)).to(DEV)
    tokens = rng.integers(0, V, (5, 3))
    s = LogprobScorer(5, k_max, V, 4, device=DEV)
    bad = tokens.copy()
    bad[0, 1], bad[2, 0] = V, -1
    out = s(z, _i32(bad), _i32([3, 1, 3, 0, 0]), _i32([2, 0, 2, 0, 0]))
    assert s.poll_status() == B.BS_FAULT_TOKEN_ID
    assert out["logprob"][0, 1] == 0 and out["logprob"][2, 0] == 0 and (out["top_tokens"][0, 1] == -1).all() and out["logprob"][2, 1] != 0
    # a bad draft_len counts no rows, a bad n_tokens skips its sequence only
    dl, nt = [2, 7, 1, -1, 2], [3, 1, 3, 0, 3]
    out = s(z, _i32(tokens), _i32(nt), _i32(dl))
    assert s.poll_status() == B.BS_FAULT_DRAFT_LEN
    keep = [0, 2, 4]
    part = {k: v[keep] for k, v in out.items()}
    _check(part, z, tokens[keep], [3, 0, 3], [2, 1, 2], 1.0, 4)
    assert (out["logprob"][[1, 3]] == 0).all() and (out["top_tokens"][[1, 3]] == -1).all()
    lp = torch.empty(3, 3, device=DEV)
    B.bs_token_logprobs(3, V, z, None, 2, _i32(tokens[:3]), None, 1.0, 0, lp, None, None, None, s.workspace)   # no status, no entropy, no alternatives
    want = torch.log_softmax(z.double(), -1).view(3, 3, V).gather(2, torch.as_tensor(tokens[:3], device=DEV)[..., None])[..., 0]
    assert torch.allclose(lp.double(), want, atol=1e-5)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_largest_vocabulary(dtype):
    """Rows of 64 segments; one in which more elements of every segment are equal than its list of candidates holds, and so are more of their best."""
    V, n_top = 2 ** 20, 32
    rng = np.random.default_rng(20)
    z = torch.from_numpy(rng.normal(0, 2.5, (4, V)).astype(np.float32))
    z[1] = 1.0
    z[2] = -INF
    z[2, rng.integers(0, V, 40)] = 2.0
    z = z.to(dtype)
    tokens = np.array([[0, V - 1], [12345, 7]])
    s = LogprobScorer(2, 1, V, n_top, device=DEV)
    _check(s(z.to(DEV), _i32(tokens)), z, tokens, [2, 2], [1, 1], 1.0, n_top)
    assert s.poll_status() == 0


@pytest.mark.parametrize("temperature", [1e-38, 1e-3, 3e38])
def test_extreme_temperatures(temperature):
    t = float(np.float32(temperature))
    z = torch.from_numpy(np.random.default_rng(3).normal(0, 2.5, (3, 200)).astype(np.float32))
    tokens = np.array([[int(z[0].argmax())], [3], [4]])
    _check(LogprobScorer(3, 0, 200, 3, device=DEV)(z.to(DEV), _i32(tokens), temperature=t), z, tokens, [1] * 3, [0] * 3, t, 3)


def test_captured_and_on_another_stream():
    """A graph sees new logits, tokens and counts in the same places; eager calls on the same workspace in between."""
    V, n_top, draft_len, n_tokens = 40001, 8, [3, 0, 2], [4, 1, 2]
    rng = np.random.default_rng(11)
    s = LogprobScorer(3, 3, V, n_top, device=DEV)
    new = lambda: torch.from_numpy(rng.normal(0, 2.5, (8, V)).astype(np.float32)).to(DEV)
    z, tokens, nt, dl = new(), rng.integers(0, V, (3, 4)), _i32(n_tokens), _i32(draft_len)
    tok = _i32(tokens)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = s(z, tok, nt, dl)
    side.synchronize()
    _check(out, z, tokens, n_tokens, draft_len, 1.0, n_top)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = s(z, tok, nt, dl)
    for _ in range(3):
        z.copy_(new())
        for v in out.values():
            v.zero_()
        g.replay()
        torch.cuda.synchronize()
        _check(out, z, tokens, n_tokens, draft_len, 1.0, n_top)
        eager = s(z, tok, nt, dl)
        assert all(torch.equal(out[k], eager[k]) for k in out)
    assert s.poll_status() == 0


def test_python_checks():
    s = LogprobScorer(2, 1, 100, 3, device=DEV)
    z, tokens = torch.zeros(4, 100, device=DEV), _i32([[1, 2], [3, 4]])
    for call in (lambda: s(z[:3], tokens), lambda: s(z[:, :99], tokens), lambda: s(z.half(), tokens), lambda: s(z.cpu(), tokens), lambda: s(z, tokens.long()), lambda: s(z, tokens.cpu()),
                 lambda: s(z, tokens, n_tokens=_i32([1])), lambda: s(z, tokens, draft_len=_i32([1])), lambda: s(z, _i32([[1, 2, 3]])), lambda: s(z, _i32([[1], [2], [3]])),
                 lambda: s(z, tokens, temperature=0.0), lambda: s(z, tokens, temperature=float("nan")), lambda: s(z, tokens, temperature=INF), lambda: s(z, tokens, temperature=1e-39)):
        with pytest.raises(B.BsError):
            call()
    assert s.poll_status() == 0


def test_outputs_of_another_type_or_too_short_are_refused():
    V, n_top = 100, 3
    z, tokens = torch.zeros(4, V, device=DEV), _i32([[1, 2], [3, 4]])
    f, i = lambda *shape: torch.full(shape, 5.0, device=DEV), lambda *shape: torch.full(shape, 5, dtype=torch.int32, device=DEV)
    s = LogprobScorer(2, 1, V, n_top, device=DEV)
    good = dict(logprob=f(2, 2), entropy=f(2, 2), top_tokens=i(2, 2, 3), top_logprobs=f(2, 2, 3), status=i(1).zero_())
    call = lambda **over: B.bs_token_logprobs(2, V, z, None, 1, tokens, None, 1.0, n_top, **{**good, **over}, workspace=s.workspace)
    call()
    kept = {k: v.clone() for k, v in good.items()}
    for name, t in good.items():
        bad = [t.flatten()[:-1], t.cpu(), t.double() if t.is_floating_point() else t.long(), t.bfloat16()]
        if t.dim() > 1:
            bad.append(t.transpose(0, 1))
        for b in bad:
            with pytest.raises(B.BsError):
                call(**{name: b})
    with pytest.raises(B.BsError):
        B.bs_token_logprobs(2, V, z[:3], None, 1, tokens, None, 1.0, n_top, **good, workspace=s.workspace)
    assert all(torch.equal(good[k], kept[k]) for k in good)


@pytest.mark.parametrize("top_k,top_p", [(5, 1.0), (0, 0.7), (40, 0.9)])
def test_the_law_of_a_filtered_sampler_from_masked_logits(top_k, top_p):
    """Rows as they are give log p under the unfiltered law; with the tokens masked that the filter drops, under the law that was sampled from.  |y| < 2^5 here: y and
    the logarithm are off by less than 2^-18 in all."""
    V, T, n_top = 3000, 0.8, 6
    z = torch.from_numpy(np.random.default_rng(top_k + 1).normal(0, 3.0, (4, V)).astype(np.float32))
    masked, tokens = torch.full_like(z, -INF), np.zeros((4, 1), dtype=np.int64)
    for i in range(4):
        keep, _ = OA.kept_tokens(z[i].numpy(), T, top_k, top_p)
        masked[i, keep] = z[i, keep]
        tokens[i] = keep[-1]
    s = LogprobScorer(4, 0, V, n_top, device=DEV)
    raw, out = s(z.to(DEV), _i32(tokens), temperature=T), s(masked.to(DEV), _i32(tokens), temperature=T)
    _check(raw, z, tokens, [1] * 4, [0] * 4, T, n_top)
    _check(out, masked, tokens, [1] * 4, [0] * 4, T, n_top)
    for i in range(4):
        p = OA.filtered_probs(z[i].double().numpy(), T, top_k, top_p)
        assert abs(float(out["logprob"][i, 0]) - np.log(p[tokens[i, 0]])) < 2.0 ** -17 and abs(float(out["entropy"][i, 0]) + (p[p > 0] * np.log(p[p > 0])).sum()) < 2.0 ** -17
        assert float(raw["logprob"][i, 0]) < float(out["logprob"][i, 0])
