"""fe_verify_drafts without draft probabilities: what the drafted token itself holds is looked at, too."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def i32(a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("value", [float("nan"), -0.25, -float("inf")])
@pytest.mark.parametrize("V,y", [(5, 0), (5, 4), (300, 0), (300, 151), (300, 299), (9001, 4500)])
def test_a_drafted_token_without_a_probability_is_reported(V, y, value, dtype):
    from paper_2603_02565_gb300 import verify_drafts
    p = torch.full((6, V), 1 / V, device="cuda").to(dtype)
    tokens, start, accept = i32([y] * 6), i32([0, 2, 4, 6]), torch.full((6,), 0.999, device="cuda")
    sample, status = torch.full((3,), 0.5, device="cuda"), i32([0])
    want, n = verify_drafts(p, tokens, start, accept, sample, status=status)
    assert status.item() == 0 and n.tolist() == [0, 0, 0]
    p[2, y] = value  # the first row of the second sequence: its draft is not accepted
    out, accepted = verify_drafts(p, tokens, start, accept, sample, status=status)
    want = want.clone()
    want[2] = -1
    assert status.item() == 1 and accepted.tolist() == [0, 0, 0] and torch.equal(out, want)


@pytest.mark.parametrize("V,y", [(5, 2), (300, 151)])
def test_a_negative_zero_at_the_drafted_token_is_a_zero(V, y):
    from paper_2603_02565_gb300 import verify_drafts
    p = torch.full((2, V), 1 / V, device="cuda")
    args = i32([y, y]), i32([0, 2]), torch.zeros(2, device="cuda"), torch.full((1,), 0.5, device="cuda")
    got = []
    for zero in (0.0, -0.0):
        p[:, y] = zero
        status = i32([0])
        out, n = verify_drafts(p, *args, status=status)
        assert status.item() == 0 and n.tolist() == [0]
        got.append(out)
    assert torch.equal(*got)
