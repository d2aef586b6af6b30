"""verify_drafts on rows of P that are far from adding up to one: 8 and more is reported and gives token 0, less is summed
as ever."""
import pytest
import torch

import _drafts_ref as D
from test_serve_drafts_gpu import _dev, _dists, _tree, _uniform

pytestmark = pytest.mark.gpu
F32, BF16, I32 = torch.float32, torch.bfloat16, torch.int32


def _run(parents, tokens, P, Q, u):
    from paper_2308_13137_gb300 import serve
    st = torch.zeros(1, dtype=I32, device="cuda")
    return serve.verify_drafts(_tree(parents), _dev(tokens), P, u, draft_probs=Q, status=st), int(st)


# one CTA and eight, sums that end within a lane, a warp, a CTA and between CTAs, and multiples of 16 (which 64 bits forget)
@pytest.mark.parametrize("V,ones", [(100, 8), (100, 16), (1000, 20), (4000, 4000), (4097, 9), (5000, 16), (32000, 32000), (32000, 12001),
                                    (128256, 100000)])
@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("dt", [F32, BF16])
def test_rows_of_eight_and_more(cuda_lib, V, ones, drawn, dt):
    """Such a row at the root (one node, a rejected child) and below an accepted child, each beside ordinary sequences."""
    plain = [-1, 0, 0, 1]
    parents = [plain, [-1], plain, [-1, 0, 0], [-1, 0, 1, 1], plain]
    first = [0, 4, 5, 9, 12, 16]
    n = 20
    P, Q = _dists(n, V, V + ones, dt=dt)
    # the weights stand spread over the row; token V - 1 has none
    at = torch.linspace(0, V - 2, ones, device="cuda").long() if ones < V else torch.arange(V - 1, device="cuda")
    heavy = torch.zeros(V, dtype=dt, device="cuda")
    heavy[at] = 1.0
    tokens = [0, 3, 7, 2] + [0] + [0, 1, 1, 4] + [0, V - 1, V - 1] + [0, 5, V - 1, V - 1] + [0, 8, 9, 9]
    P[4], P[9], P[13] = heavy, heavy, heavy
    P[12, 5], Q[12, 5] = 1.0, 0.5                               # accepted at any number
    for seed in range(3):
        u = _uniform(n, seed)
        got, st = _run(parents, tokens, P, Q if drawn else None, u)
        assert st == 1
        for b, path in ((1, [0]), (3, [0]), (4, [0, 1])):
            row = first[b] + path[-1]
            if b != 1 and drawn and float((P[row].double() - Q[row].double()).clamp_min(0).sum()) < 8:
                continue                                        # what a rejection leaves of 8 may be less: an ordinary draw
            assert int(got.count[b]) == len(path)
            assert got.path[b].tolist() == path + [-1] * (4 - len(path))
            assert got.tokens[b].tolist() == [tokens[first[b] + i] for i in path[1:]] + [0] + [-1] * (4 - len(path))
        for b in (0, 2, 5) + ((3, 4) if drawn and ones == 8 else ()):
            rows = slice(first[b], first[b] + len(parents[b]))
            path, out = D.verify(parents[b], tokens[rows], P[rows], Q[rows] if drawn else None, u[rows].double().tolist(), 4)
            assert got.path[b].tolist() == path + [-1] * (4 - len(path)) and got.tokens[b].tolist() == out + [-1] * (4 - len(out))


@pytest.mark.parametrize("V", [60, 4096, 32000])
def test_rows_below_eight(cuda_lib, V):
    """Sums of 7 to 7.99 are exact, and the draw is from the weights as they are."""
    P, Q = _dists(6, V, V)
    P[:, torch.linspace(1, V - 3, 7, device="cuda").long()] = 1.0
    P *= 7.99 / P.double().sum(-1, keepdim=True).clamp_min(7.99).float()
    parents = [[-1, 0, 0], [-1, 0, 1]]
    tokens = [0, V - 1, V - 2, 0, V - 1, 2]
    P[0::3, V - 1] = 0
    for seed in range(6):
        u = _uniform(6, seed)
        for q in (Q, None):
            got, st = _run(parents, tokens, P, q, u)
            assert st == 0
            for b in range(2):
                rows = slice(3 * b, 3 * b + 3)
                path, out = D.verify(parents[b], tokens[rows], P[rows], None if q is None else q[rows], u[rows].double().tolist(), 3)
                assert got.path[b].tolist() == path + [-1] * (3 - len(path)) and got.tokens[b].tolist() == out + [-1] * (3 - len(out))
