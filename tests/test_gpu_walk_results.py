"""Results that a caller brings to the walk with filtered tokens: refused before anything is launched where a kernel would write past
them, written in place otherwise."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _call(out):
    import paper_2604_12989_amd as dd
    batch, T, V, B = 2, 3, 40, 4
    x = torch.randn(batch, T, V, device="cuda")
    x[:, 0, 7] = 50.0
    x[:, 1, 9] = 50.0
    tokens, parent, depth = (torch.tensor([v] * batch, dtype=torch.int32, device="cuda") for v in ([0, 7, 8], [-1, 0, 0], [0, 1, 1]))
    n_nodes = torch.full((batch,), 2, dtype=torch.int32, device="cuda")
    ws = dd.Workspace(batch, B, V, T - 1, 1, 1, 64, 0)
    return dd.accept_filtered(x, tokens, parent, depth, n_nodes, B, torch.full((batch, T), 0.5, device="cuda"), ws, top_k=1, out=out)


def _out(**other):
    def ints(*shape):
        return torch.full(shape, -7, dtype=torch.int32, device="cuda")
    return dict(dict(path=ints(2, 5), n_accepted=ints(2), bonus_token=ints(2), posterior=ints(2, 3)), **other)


@pytest.mark.parametrize("name,shape", [("path", (2, 4)), ("n_accepted", (1,)), ("bonus_token", (1,)), ("posterior", (2, 2))])
def test_a_result_of_another_size_or_type_is_refused(name, shape):
    import paper_2604_12989_amd as dd
    right = _out()[name]
    for t in (torch.zeros(shape, dtype=torch.int32, device="cuda"), right.short(), right.long(), right.cpu(),
              torch.zeros(2 * right.numel(), dtype=torch.int32, device="cuda")[::2].view_as(right)):
        with pytest.raises(dd.DDTreeError):
            _call(_out(**{name: t}))
    for name in ("path", "n_accepted", "bonus_token"):
        with pytest.raises(dd.DDTreeError):
            _call(_out(**{name: None}))


@pytest.mark.parametrize("other", [dict(), dict(posterior=None)])
def test_results_are_written_in_place(other):
    out = _out(**other)
    got = _call(out)
    assert all(got[k] is out[k] for k in out)
    assert got["path"].tolist() == [[0, 1, -1, -1, -1]] * 2 and got["n_accepted"].tolist() == [1, 1] and got["bonus_token"].tolist() == [9, 9]
