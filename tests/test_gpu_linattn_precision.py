"""Linear attention where its terms cancel: what is left has to be that of 32-bit
arithmetic, whatever type the result is rounded to.

Each pass is sum_s l^(i-s) (q_i . k_s) v_s with the roles of q, k and v taken by
    o: q, k, v    dq: dout, v, k    (forward)
    dk: v, dout, q    dv: k, q, dout    (from the last token)
Three tokens have keys of a single 1 each and values of which the second and the
third are the rounded rest of those before, so that from the third on the terms
cancel to a rounding of the rest's rest; the queries from there on are 1 at the
three places.  The products q . k are exact, three terms reach an entry.

With u = 2^-24 and A the sum of the terms' magnitudes, the error is below
  - 4 u for a decay's power and its products with the factors;
  - 4 u for three bf16 parts of two fp32 factors, and for the products left out;
  - 18 u for the sums of 3 terms of 6 products of parts;
  - 2 u for each chunk of 32 tokens that a state is carried on, 8 u for its
    entry into a chunk or segment, 4 u for the result's factors:
64 u A in all for up to 100 tokens, u / 8 more for each further one; then the
rounding to the result's type.  Two parts would leave up to 2^-17 of each factor.
"""
import pytest
import torch

from _parity import log
from test_gpu_linattn import BF, F32, F64, U, backward, forward, run_bwd, run_fwd, within

DECAYS = [0.97, 0.9, 0.75, 0.999, 0.5, 0.99]
ROLES = {"o": ("q", "k", "v", False), "dq": ("do", "v", "k", False), "dk": ("v", "do", "q", True), "dv": ("k", "q", "do", True)}


@pytest.fixture(scope="module")
def mmf():
    import paper_2406_02528_amd as m
    return m


def cancelling(B, T, H, dk, dv, t, do_t, result, at):
    """Inputs in which the terms of `result` cancel; `at`: the three tokens."""
    g = torch.Generator().manual_seed(T + dk)
    kinds = {"q": (dk, t), "k": (dk, t), "v": (dv, t), "do": (dv, do_t)}
    x = {n: torch.zeros(B, T, H, w, dtype=F64) for n, (w, _) in kinds.items()}
    q, k, v, rev = ROLES[result]
    place = torch.randperm(kinds[k][0], generator=g)[:3]
    l = torch.tensor(DECAYS[:H]).double()[:, None]
    rest, before = torch.zeros(B, H, kinds[v][0], dtype=F64), 0
    for n, i in enumerate(at):
        rest = rest * l ** (i - before)
        row = torch.randn(rest.shape, generator=g).double() if n == 0 else -rest
        row = row.to(kinds[v][1]).double()
        rest, before = rest + row, i
        j = T - 1 - i if rev else i
        x[v][:, j], x[k][:, j, :, place[n]] = row, 1.0
    last = slice(0, T - at[2]) if rev else slice(at[2], T)
    for p in place:
        x[q][:, last, :, p] = 1.0
    rows = {n: y.reshape(B * T, -1) for n, y in x.items()}
    return {"qkv": torch.cat([rows["q"], rows["k"], rows["v"]], 1).to(t), "decay": torch.tensor(DECAYS[:H]), "s0": None,
            "dout": rows["do"].to(do_t), "ds_last": None, "scale": 0.25, "dims": (B, T, H, dk, dv)}


CASES = [((1, 12, 6, 32, 48), (0, 4, 9)), ((2, 100, 6, 128, 128), (3, 17, 20)), ((2, 100, 3, 64, 64), (1, 33, 60)),
         ((1, 90, 2, 256, 144), (5, 30, 40)), ((1, 96, 4, 48, 256), (0, 1, 31)), ((1, 1200, 2, 128, 64), (2, 200, 500)),
         ((2, 700, 6, 80, 128), (100, 110, 117))]


# the forward has no dout
TYPES = [(r, t, do_t) for r in ROLES for t in (F32, BF) for do_t in (F32, BF) if r != "o" or t == do_t]


@pytest.mark.gpu
@pytest.mark.parametrize("result,t,do_t", TYPES, ids=["-".join(str(x).replace("torch.", "") for x in c) for c in TYPES])
@pytest.mark.parametrize("dims,at", CASES, ids=[str(c[0]) for c in CASES])
def test_cancelling_terms(mmf, dims, at, result, t, do_t):
    log(f"[linattn] cancelling {result} {dims} {t} {do_t}")
    p = cancelling(*dims, t, do_t, result, at)
    if result == "o":
        got, want, A = run_fwd(mmf, p)[0], forward(p)[0], forward(p, torch.abs)[0]
    else:
        got, want, A = run_bwd(mmf, p, do_t)[0], backward(p)[0], backward(p, torch.abs)[0]
    u = (64 + max(0, dims[1] - 100) / 8) * U
    step = torch.finfo(got.dtype).eps / 2
    # where the query sees all three, they cancel
    assert float(((want.abs() <= 2.0 ** -14 * A) & (A > 0)).sum()) > 0.2 * float((A > 0).sum())
    within(got, want, u * A + step * (want.abs() + u * A) + 1e-37, result)
