"""Numbers past 32 bits in the binding of the steps: refused before anything is launched
or allocated, where a C int would hold their low half."""
import pytest

from test_gpu_steps import SCALE, device, steps, torch, trees  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("past", [2 ** 32, -2 ** 32, 2 ** 40])
def test_numbers_past_32_bits_are_refused(torch, steps, past):  # noqa: F811
    lens = torch.tensor([3, 4], dtype=torch.int32, device="cuda")
    table = torch.zeros((2, 4), dtype=torch.int32, device="cuda")
    free, state = steps.new_pool(8, "cuda")
    plan = steps.empty_plan(2, 9, "cuda")
    before = [x.clone() for x in (table, free, state)]
    with pytest.raises(ValueError, match="block_size"):
        steps.extend(lens, lens, table, free, state, 9, block_size=past + 16, plan=plan)
    with pytest.raises(ValueError, match="block_size"):
        steps.release(lens, lens, table, free, state, block_size=past + 16)
    with pytest.raises(ValueError, match="T ="):
        steps.extend(lens, lens, table, free, state, past + 9)
    args = device(torch, trees([20, 5], [3, 4], 4, 2, 40))
    with pytest.raises(ValueError, match="max_nodes"):
        steps.tree_attention(*args[:9], past + 4, SCALE)
    for bad in ((past + 4, 32, 8), (4, past + 32, 8), (4, 32, past + 8)):
        with pytest.raises(ValueError):
            steps.tree_workspace_bytes(*bad)
    assert all(torch.equal(x, y) for x, y in zip(before, (table, free, state)))
