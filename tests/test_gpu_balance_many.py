"""The balance loss of a packed batch of more sequences than a call takes: a call for each so many of them, the gradient added up."""
import pytest
import torch

import fp4_plain as plain
import paper_2411_02581_amd as tuna

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def ok(rc):
    assert rc == tuna.TUNA_OK, tuna.tuna_strerror(rc)


@pytest.mark.parametrize("sequences,experts,k", [(1025, 16, 2), (1500, 70, 3), (2600, 8, 1)])
def test_more_sequences_than_a_call_takes(sequences, experts, k):
    g = torch.Generator().manual_seed(sequences)
    lengths = torch.randint(0, 7, (sequences,), generator=g)
    rows = torch.cat([torch.tensor([3]), 3 + lengths.cumsum(0)]).int()          # three tokens in front, two behind
    n = int(rows[-1]) + 2
    logits, dloss = torch.randn(n, experts, generator=g), torch.randn(sequences, generator=g)
    chosen = torch.stack([torch.randperm(experts, generator=g)[:k] for _ in range(n)]).int()
    most = tuna.TUNA_MOE_MAX_EXPERTS
    new = lambda *s, dtype=torch.float32: torch.full(s, 7, dtype=dtype, device=DEV)  # noqa: E731
    l, ex, r, d = logits.to(DEV), chosen.to(DEV), rows.to(DEV), dloss.to(DEV)
    counts, tokens, shares, loss = new(sequences, experts, dtype=torch.int32), new(sequences, dtype=torch.int32), new(sequences, experts), new(sequences)
    dlogits = torch.zeros(n, experts, device=DEV)
    rc, size = tuna.tuna_moe_balance_workspace(n, experts, most)
    ok(rc)
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)
    assert tuna.tuna_moe_balance(l, 0, experts, n, experts, ex, k, r, sequences, counts, tokens, shares, loss, ws, size) == tuna.TUNA_ERR_ARG
    for a in range(0, sequences, most):
        here = min(most, sequences - a)
        ok(tuna.tuna_moe_balance(l, 0, experts, n, experts, ex, k, r[a:], here, counts[a:], tokens[a:], shares[a:], loss[a:], ws, size))
        ok(tuna.tuna_moe_balance_grad(l, 0, experts, n, experts, r[a:], here, counts[a:], tokens[a:], d[a:], tuna.TUNA_BALANCE_ADD, dlogits, experts))
    c, t, s, want = plain.balance(logits, chosen, rows.tolist())
    assert torch.equal(counts.cpu().long(), c) and torch.equal(tokens.cpu().long(), t)
    # sums of a few positive terms in 32 bits, an exponential of two units of the last place
    assert torch.allclose(shares.cpu().double(), s, rtol=1e-5, atol=1e-9) and torch.allclose(loss.cpu().double(), want, rtol=1e-5)
    exact = plain.balance_grad(logits, c, t, rows.tolist(), dloss)
    # d = slope p (f - sum f p): the bracket is a difference of numbers up to one
    p = plain.softmax(logits)
    room = torch.zeros_like(exact)
    for i, (a, b) in enumerate(zip(rows[:-1].tolist(), rows[1:].tolist())):
        room[a:b] = 1e-5 * abs(float(dloss[i])) * experts / max(int(t[i]), 1) * p[a:b]
    assert bool(((dlogits.cpu().double() - exact).abs() <= room).all())
