"""A number of 1 or more takes the last token with any mass, however the sums before it are rounded: the tokens behind the rows' bulk have
so little mass that they change no sum."""
import pytest
import torch

from paper_2607_27735_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V,bulk", [(777, 500), (3001, 2990), (50000, 20000), (131072, 131000)])
def test_the_last_token_with_mass(V, bulk):
    g = torch.Generator().manual_seed(V)
    B = 256
    p = torch.zeros(B, 1, V)
    p[:, 0, :bulk] = torch.softmax(torch.randn(B, bulk, generator=g) * 3, -1)
    last = torch.randint(bulk, V, (B,), generator=g)
    p[torch.arange(B), 0, last] = 1e-30
    p[:, 0, bulk - 1] = 1e-25
    u = torch.ones(B, 1)
    u[::3] = 1.5
    n, token = binding.spec_accept_sample(p.cuda(), torch.zeros(B, 0, dtype=torch.int32, device="cuda"), u.cuda())
    assert n.tolist() == [0] * B
    assert token.tolist() == last.tolist()
