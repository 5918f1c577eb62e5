"""A new PagedPlan holds no lengths and has taken no pages: the first step may go on from it, as the usage in README.md does."""
import pytest

torch = pytest.importorskip("torch")
from paper_1712_01084_b200 import binding as pb


def test_a_new_plan_starts_at_nothing(monkeypatch):
    pb._load_torch()
    monkeypatch.setattr(torch, "empty", lambda n, **kw: torch.full((n,), 77, **kw))        # memory as an earlier tensor left it
    plan = pb.PagedPlan(3, 8, device="cpu")
    assert plan.lengths.tolist() == [0, 0, 0] and plan.taken.tolist() == [0]
    assert plan.lengths.dtype == plan.taken.dtype == torch.int32 and plan.slots.shape == plan.positions.shape == (8,) and plan.starts.shape == (4,)


@pytest.mark.gpu
def test_the_first_steps_of_a_new_plan():
    """The lines of README.md, on memory that other tensors have used."""
    for n in (1, 4, 5, 8):
        torch.full((n,), 1000, dtype=torch.int32, device="cuda")
    requests, rows, width, pages = 4, 8, 3, 20
    plan = pb.PagedPlan(requests, rows)
    table = torch.full((requests, width), -1, dtype=torch.int32, device="cuda")
    free = torch.arange(pages, dtype=torch.int32, device="cuda")
    added = torch.tensor([1, 3, 0, 2], dtype=torch.int32, device="cuda")
    for step in (1, 2):
        pb.pp_paged_plan(plan.lengths, added, table, free, plan.taken, 16, out=plan)
        assert plan.lengths.tolist() == [step * n for n in (1, 3, 0, 2)] and plan.taken.tolist() == [3]
    assert table.tolist() == [[0, -1, -1], [1, -1, -1], [-1, -1, -1], [2, -1, -1]]
    assert plan.slots.tolist() == [1, 19, 20, 21, 34, 35, -1, -1] and plan.positions.tolist() == [1, 3, 4, 5, 2, 3, 0, 0]
