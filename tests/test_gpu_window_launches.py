"""More requests than a launch takes, all of them split: each launch's partials lie in
the same workspace and are merged before the next launch writes its own."""
import pytest
import torch

from test_gpu_window import DEV, Case

pytestmark = pytest.mark.gpu


def batch(T, branched):
    """Requests of about T keys, alike to the planner: 140 of up to six rows, or 70 of up to eight with branches."""
    if branched:
        return [(T - 15 - i % 7 - (1 + i % 3), 1 + i % 3, [(1, 1, 3), (1, 0, 2)] if i % 4 else 5) for i in range(70)]
    return [(T - 10 - i % 7 - (1 + i % 3) - i % 4, 1 + i % 3, i % 4) for i in range(140)]


@pytest.mark.parametrize("branched", [False, True])
@pytest.mark.parametrize("kv8, window, T, heads", [
    (True, None, 2000, (4, 1, 64)), (True, (2500, 9), 3000, (4, 1, 64)),
    (False, (1 << 20, 0), 2000, (4, 1, 128)), (False, (1200, 9), 3000, (4, 1, 64))])
def test_split_requests_of_several_launches(kv8, window, T, heads, branched):
    c = Case(batch(T, branched), heads, kv8=kv8, window=window)
    a_launch = 64 if branched else 128
    need = c.workspace_bytes()
    # partials of 32 columns x D and two numbers a column: as many runs for every
    # request of the first launch, two at least, and so for the alike ones behind it
    runs, rest = divmod(need, a_launch * 32 * (c.b.d + 2) * 4)
    assert runs >= 2 and rest == 0
    ws = torch.full((need,), 0xff, dtype=torch.uint8, device=DEV)
    c.check(workspace=ws)
    first = c.call(workspace=ws)
    again = c.call(workspace=ws.fill_(0xff))
    assert all(torch.equal(x, y) for x, y in zip(first, again))
