"""128 rows of a head over page scales: a long context goes to the score-cache kernel in two halves of the rows, within its limits with the ring of
scales in shared memory; a shorter one to the kernel over the expanded copy, as with a scale for each head."""
import pytest

from paper_2607_27735_b200 import binding
from test_gpu_page_scales import compare, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ctx,ps,route", [((33000,), 64, binding.VERIFY_TCGEN05_CACHED_2PASS),
                                          ((5000, 900), 16, binding.VERIFY_TCGEN05_CACHED_EXPANDED)])
def test_the_route_of_many_rows(ctx, ps, route):
    kv, q, lens = make(ctx=ctx, n_q=32, Hq=16, H=4, seed=8, ps=ps)
    binding.spec_verify_attn(kv, q, lens, int(lens.max()))
    assert binding.last_verify_impl() == route
    compare(kv, q, lens, route)
