"""batch_plan_pages where pages that requests hold already are no pages of the pool."""
import pytest

from tests.test_gpu_batch_plan import Step

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu(built_lib):
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")


@pytest.mark.parametrize("bad", [-1, 1000, 1 << 30])
def test_a_held_page_outside_the_pool_that_rows_go_to_is_flagged(bad):
    """The rows lose their slots, and the status says so; request 1's rows keep theirs."""
    s = Step(16, [20, 3], [14, 2], [2, 1], [[4, bad, -1], [6, -1, -1]], [7], 0, 16, n_pages=1000).run()
    assert s.status.item() == 64
    assert s.slot.tolist() == [-1] * 12 + [7 * 16, 7 * 16 + 1, 6 * 16 + 3, 6 * 16 + 4]
    assert s.table.tolist() == [[4, bad, 7], [6, -1, -1]] and s.row_start.tolist() == [0, 14, 16]


def test_a_held_page_of_cached_tokens_alone_is_not_looked_at():
    s = Step(16, [20, 3], [2, 2], [2, 1], [[-1, 5], [6, -1]], [7], 0, 4, n_pages=1000).run()
    assert s.status.item() == 0 and s.slot.tolist() == [5 * 16 + 4, 5 * 16 + 5, 6 * 16 + 3, 6 * 16 + 4]


def test_a_held_page_that_no_row_reaches_is_not_looked_at():
    """Held beyond what the step needs."""
    s = Step(16, [5], [2], [2], [[4, 5000]], [7], 0, 2, n_pages=1000).run()
    assert s.status.item() == 0 and s.slot.tolist() == [4 * 16 + 5, 4 * 16 + 6] and s.held_out.tolist() == [2]
