"""Beam search: selection and reordering of states against numpy in 64 bits.

Tokens, parents and done flags must be equal.  A score's error: the sum of
exponentials takes each as 2^(x log2 e), whose argument and result are rounded
to fp32 (|x| 1.45 u and one ulp, 2 u; u = 2^-24), and adds up to 64 of them in
fp32 (64 u); its logarithm is then off by at most (1.5 max|x| where it counts +
66) u.  Exponentials of x < -30 are below u of the sum for V < 2^20 together,
so |x| <= 30 counts: 111 u, taken as 2^-17; then the fp32 score, u |score|.
Inputs whose order 2^-16 would change are not used (asserted).
"""
import numpy as np
import pytest
import torch

from _parity import dev, log

BF, F32 = torch.bfloat16, torch.float32
NINF = -np.inf


@pytest.fixture(scope="module")
def mmf():
    import paper_2406_02528_amd as m
    return m


def reference(z, scores, done, end, n):
    """z [B][W][V] float64, scores [B][W]; the n best in the documented order."""
    B, W, V = z.shape
    z = np.where(np.isnan(z), NINF, z)
    if done is not None:
        over = done != 0
        z[over] = NINF
        z[over, end] = 0.0
    c = np.where(np.isnan(scores) | (scores == np.inf), NINF, scores.astype(np.float64))
    out = {k: [] for k in ("scores", "tokens", "parents", "done")}
    for b in range(B):
        s = np.full((W, V), NINF)
        for w in range(W):
            m = z[b, w].max()
            if m == NINF or c[b, w] == NINF:
                continue
            with np.errstate(invalid="ignore"):
                d = np.where(z[b, w] == m, 0.0, z[b, w] - m)
            s[w] = c[b, w] + (d - np.log(np.exp(d).sum()))
        beam, token = np.divmod(np.arange(W * V), V)
        order = np.lexsort((token, -z[b].reshape(-1), beam, -s.reshape(-1)))[: n + 1]
        top = s.reshape(-1)[order]
        for i in range(len(order) - 1):
            if beam[order[i]] != beam[order[i + 1]] and top[i] != top[i + 1]:
                assert top[i] - top[i + 1] > 2.0 ** -16, "inputs next to a tie"
        order = order[:n]
        out["scores"].append(s.reshape(-1)[order])
        out["tokens"].append(token[order])
        out["parents"].append(beam[order])
        out["done"].append((token[order] == end) | (False if done is None else done[b][beam[order]] != 0))
    return {k: np.stack(v) for k, v in out.items()}


def select(mmf, z, scores, done, end, n, ws=None, stream=None):
    B, W, V = z.shape
    e = lambda dt, fill: torch.full((B, n), fill, dtype=dt, device=dev())  # noqa: E731
    out = {"scores": e(F32, float("nan")), "tokens": e(torch.int32, -7), "parents": e(torch.int32, -7),
           "done": e(torch.uint8, 9)}
    mmf.mmf_beam_select(z.reshape(B * W, V).to(dev()), scores.to(dev()), None if done is None else done.to(dev()), end, B, W,
                        n, out["scores"], out["tokens"], out["parents"], out["done"], ws, stream)
    torch.cuda.synchronize()
    return {k: v.cpu().numpy() for k, v in out.items()}


def check(mmf, z, scores, done, end, n):
    want = reference(z.double().numpy().copy(), scores.numpy(), None if done is None else done.numpy(), end, n)
    got = select(mmf, z, scores, done, end, n)
    for k in ("tokens", "parents"):
        assert np.array_equal(got[k], want[k]), (k, got[k], want[k])
    assert np.array_equal(got["done"] != 0, want["done"]) and got["done"].max() <= 1
    a, b = got["scores"].astype(np.float64), want["scores"]
    assert np.array_equal(a == NINF, b == NINF)
    fine = b != NINF
    assert (np.abs(a[fine] - b[fine]) <= 2.0 ** -17 + 2.0 ** -24 * np.abs(b[fine])).all()
    return got


def draw(B, W, V, t, seed, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(B, W, V, generator=g) * spread).to(t), -20 * torch.rand(B, W, generator=g), g


CASES = [(1, 1, 1, 1), (1, 1, 2, 2), (2, 3, 1, 3), (1, 2, 5, 10), (3, 4, 7, 4), (1, 1, 64, 64), (2, 5, 63, 10),
         (1, 4, 1000, 4), (2, 8, 4095, 8), (1, 3, 4097, 6), (5, 2, 8193, 1), (1, 64, 129, 64), (1, 5, 32000, 64),
         (2, 4, 50001, 8), (1, 2, 70001, 3)]


@pytest.mark.gpu
@pytest.mark.parametrize("t", [F32, BF], ids=["f32", "bf16"])
@pytest.mark.parametrize("B,W,V,n", CASES)
def test_selection(mmf, B, W, V, n, t):
    log(f"[beam] B={B} W={W} V={V} n={n} {t}")
    z, s, _ = draw(B, W, V, t, B + W + V + n)
    check(mmf, z, s, None, -1, n)
    check(mmf, z, s, None, V - 1, n)


@pytest.mark.gpu
@pytest.mark.parametrize("t", [F32, BF], ids=["f32", "bf16"])
@pytest.mark.parametrize("B,W,V,n", [(4, 4, 17, 8), (3, 5, 1000, 5), (6, 3, 9000, 12)])
def test_done_beams_go_on_as_themselves(mmf, B, W, V, n, t):
    z, s, g = draw(B, W, V, t, 5)
    done = (torch.rand(B, W, generator=g) < 0.5).to(torch.uint8) * 3
    done[0] = 1                                  # all of a batch
    z[done != 0] = float("nan")                  # not read
    got = check(mmf, z, s, done, 2, n)
    assert (got["tokens"][0][:W] == 2).all() and np.array_equal(np.sort(got["parents"][0][:W]), np.arange(min(W, n)))


@pytest.mark.gpu
@pytest.mark.parametrize("t", [F32, BF], ids=["f32", "bf16"])
def test_masks(mmf, t):
    z, s, _ = draw(6, 3, 5000, t, 6)
    inf = float("inf")
    z[0] = -inf                                  # nothing is left: in order, all of -inf
    z[1, 0] = -inf                               # one row without a token
    z[2, :, 4:] = -inf                           # fewer tokens than are wanted
    z[3, 1, 100:4500] = float("nan")             # NaN counts as -inf
    z[4, 2, 77] = inf                            # +inf leaves no other
    z[4, 0, [5, 4999]] = inf
    z[5, 1] = torch.finfo(t).min                 # masked with the lowest value
    z[5, 1, 9] = 3.0
    check(mmf, z, s, None, 1, 16)


@pytest.mark.gpu
def test_ties_go_to_the_lowest_beam_and_token(mmf):
    z = torch.zeros(2, 4, 6000)
    z[1] = torch.randn(6000, generator=torch.Generator().manual_seed(1)).round()  # equal rows, many equal logits
    z[0, :, 17] = -0.0
    check(mmf, z, torch.zeros(2, 4), None, -1, 64)
    check(mmf, z.to(BF), torch.zeros(2, 4), None, -1, 33)


@pytest.mark.gpu
def test_scores_that_are_not_there(mmf):
    z, s, _ = draw(3, 4, 300, F32, 8)
    s[0, 1:] = float("-inf")                     # the first step
    s[1, 0], s[1, 1] = float("nan"), float("inf")
    s[2] = float("-inf")
    check(mmf, z, s, None, 0, 8)


@pytest.mark.gpu
@pytest.mark.parametrize("V", [33, 20000])
def test_sorted_logits(mmf, V):
    """Rising and falling logits: one thread's values hold many of the best."""
    up = torch.arange(V, dtype=F32) / 64
    z = torch.stack([up, up.flip(0) - 0.003, torch.roll(up, 11) + 0.001])[None]
    check(mmf, z, torch.tensor([[0.0, -0.0301, 0.02]]), None, -1, 32)


def reorder_case(B, W, rows, seed):
    g = torch.Generator().manual_seed(seed)
    states = [torch.randint(0, 2 ** 31 - 1, (B * W, *r), generator=g, dtype=torch.int32) for r in rows]
    return states, torch.randint(0, W, (B, W), generator=g, dtype=torch.int32)


def reordered(states, parents):
    B, W = parents.shape
    p = parents.long()
    p = torch.where((p < 0) | (p >= W), torch.arange(W), p)
    src = (p + W * torch.arange(B)[:, None]).reshape(-1)
    return [s[src] for s in states]


@pytest.mark.gpu
@pytest.mark.parametrize("B,W", [(1, 1), (1, 4), (3, 5), (2, 8), (5, 13), (1, 16), (2, 17), (1, 64)])
def test_reordering(mmf, B, W):
    log(f"[beam] reorder {B} {W}")
    states, parents = reorder_case(B, W, [(4,), (2, 2, 37), (0,), (1024,), (5000, 4)], B * W)
    parents[0, 0] = -1
    parents[-1, -1] = W
    want = reordered(states, parents)
    here = [s.to(dev()) for s in states]
    outs = [torch.full_like(s, -1) for s in here]
    mmf.mmf_beam_reorder(here, parents.to(dev()), B, W, outs)
    assert all(torch.equal(a.cpu(), b) for a, b in zip(here, states))       # the inputs stay
    assert all(torch.equal(a.cpu(), b) for a, b in zip(outs, want))
    mmf.mmf_beam_reorder(here, parents.to(dev()), B, W)                     # in place
    assert all(torch.equal(a.cpu(), b) for a, b in zip(here, want))


@pytest.mark.gpu
def test_reordering_many_arrays(mmf):
    states, parents = reorder_case(2, 3, [(4 * (i % 7 + 1),) for i in range(300)], 3)
    here = [s.to(dev()) for s in states]
    mmf.mmf_beam_reorder(here, parents.to(dev()), 2, 3)
    assert all(torch.equal(a.cpu(), b) for a, b in zip(here, reordered(states, parents)))
