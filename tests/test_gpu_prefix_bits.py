"""What a row over a shared prefix does not depend on, to the last bit: the scores of the rows beside it."""
import pytest
import torch

from paper_2511_20340_amd import binding as sfb

from test_gpu_prefix_attention import call, load, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads", ["f32", "1b", "8b", "14b"])
@pytest.mark.parametrize("B,n_q", [(3, 2), (7, 5)])
def test_a_row_does_not_hang_on_its_neighbours(heads, B, n_q):
    """The other sequences' scores rise and fall by hundreds along the prefix; one sequence keeps its bits, wherever it stands."""
    P, cap = 700, 64
    eng, one, q, pk, pv, k, v = make(heads, B, n_q, P, cap, 21)
    ramp = torch.linspace(-1, 1, pk.shape[2], device="cuda")[None, None, :, None]
    pk = (pk.float() * 0.5 + ramp * torch.where(torch.arange(q.shape[-1], device="cuda") % 2 == 0, 1.0, -0.5)).to(pk.dtype)
    load(eng, one, pk, pv, k, v)
    lens = [20] * B
    for b in (0, B // 2, B - 1):
        want = call(eng, one, q, P, lens, n_q, sfb.SF_MASK_CAUSAL)[b].clone()
        for scale in (0.0, 4.0, -4.0, 50.0):
            other = q * scale
            other[b] = q[b]
            got = call(eng, one, other, P, lens, n_q, sfb.SF_MASK_CAUSAL)[b]
            assert torch.equal(got, want), (b, scale)
