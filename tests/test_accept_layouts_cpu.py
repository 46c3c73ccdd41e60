"""Tensors that do not lie as a kvb_vocab says are refused by the binding (no GPU: calls of no requests, which launch nothing)."""
import pytest
import torch

from paper_2605_19049_amd import kvb

B, T, V = 3, 2, 50
NAMES = ("n_drafts", "parent", "tokens", "target", "draft", "u", "s", "path", "accepted", "token")


def arrays(**more):
    whole = lambda *size: torch.zeros(size, dtype=torch.int32)
    a = dict(n_drafts=whole(B), parent=whole(B, T), tokens=whole(B, T), target=torch.zeros(B, T + 1, V), draft=torch.zeros(B, T, V),
             u=torch.zeros(B, T), s=torch.zeros(B), path=whole(B, T), accepted=whole(B), token=whole(B))
    return {**a, **more}


def accept(a, bound, stride=0):
    args = [kvb.vocab(0, T, V, kvb.F32, stride)] + [a[x] for x in NAMES] + [torch.zeros(64)]
    if bound:
        return kvb.bind("kvb_accept", *args, 0)()
    return kvb.kvb_accept(*args, stream=0)


@pytest.mark.parametrize("bound", [False, True])
@pytest.mark.parametrize("name, rows", [("target", T + 1), ("draft", T)])
def test_rows_of_probabilities(name, rows, bound):
    """A padded vocabulary's first V columns need the stride; every row is as far from the one before, also from request to request."""
    other = "draft" if name == "target" else "target"
    wide = {name: torch.zeros(B, rows, V + 14)[..., :V], other: torch.zeros(B, T + 1 if other == "target" else T, V + 14)}
    accept(arrays(**wide), bound, V + 14)
    for bad in (wide[name], torch.zeros(B, rows + 1, V)[:, :rows], torch.zeros(B, rows, 2 * V)[..., ::2], torch.zeros(rows, B, V).transpose(0, 1),
                torch.zeros(V).expand(B, rows, V)):
        with pytest.raises(ValueError):
            accept(arrays(**{name: bad}), bound)
    with pytest.raises(ValueError):
        accept(arrays(), bound, V + 14)
    accept(arrays(**{name: torch.zeros(B * rows, V)}), bound)     # rows one after the other
    accept(arrays(**{name: torch.zeros(B * rows * V)}), bound)
    accept(arrays(**{name: torch.zeros(1, rows, 2 * V)[..., :V] if rows == 1 else torch.zeros(1, rows, V)}), bound)


@pytest.mark.parametrize("bound", [False, True])
def test_what_has_no_stride_is_packed(bound):
    for name, x in arrays().items():
        if name not in ("target", "draft"):
            wide = torch.zeros(tuple(x.shape) + (2,), dtype=x.dtype)[..., 0]
            with pytest.raises(ValueError):
                accept(arrays(**{name: wide}), bound)
    accept(arrays(n_drafts=None, parent=None, draft=None), bound)
    accept({x: 4096 for x in NAMES}, bound, V + 14)
