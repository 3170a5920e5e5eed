"""sx_append_slots on the GPU, beside test_gpu_decode.py: the count of tokens that got no slot."""
import pytest
import torch

import kv4ref as R
import paper_2606_01751_amd as sx
from test_gpu_decode import run_slots

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    sx.lib()


def check(ctx, new, b, free, head, table, room):
    """Against the loops of kv4ref; a slot that int32 does not hold is none, and the count is that of the slots."""
    got = run_slots(ctx, new, b, free, head, table, room)
    want = list(R.append_slots(ctx, new, b, free, head, table, room))
    want[4] = [s if s < 1 << 31 else -1 for s in want[4]]
    live = sum(new)
    want[5][1] = sum(s < 0 for s in want[4][:live]) + max(live - room, 0)
    for name, g, w in zip(("table", "seq", "cu", "pos", "slot", "state"), got, want):
        assert torch.equal(g, torch.as_tensor(w, dtype=torch.int32).reshape(g.shape)), name
    return want[5][1]


BIG = 1 << 27                       # its slots pass int32 with 16 tokens a block


@pytest.mark.parametrize("free", [
    [20, -1, 21, 22, 23, 24], [20, BIG, 21, -7, 22, 23], [-1] * 6, [BIG] * 6, [20, 21, 22, 23, 24, -1], [BIG - 1] * 3 + [-1],
    [-1, 20], [20, 21, 22, 23, 24, 25, -1, BIG],      # (the last two stand behind what is taken)
])
@pytest.mark.parametrize("room", [0, 5, 30, 61, 70])
def test_bad_entries_of_the_free_list_are_counted(free, room):
    table = torch.full((4, 4), -9, dtype=torch.int32)
    table[0, 0], table[2, :2] = 5, torch.tensor([6, 7])
    ctx, new = [10, 0, 30, 0], [20, 16, 24, 1]
    check(ctx, new, 16, free, 0, table, room)
    check(ctx, new, 16, [3, -1] + free, 2, table, room)


def test_an_open_block_whose_slots_pass_int32_is_counted():
    # the block of the last token held: its first slots fit, the others do not (block size 5: 2^31 / 5 = 429496729.6)
    edge = (1 << 31) // 5
    table = torch.tensor([[edge, -9, -9], [BIG * 4, -9, -9], [-1, -9, -9], [1, -9, -9]], dtype=torch.int32)
    for c in range(1, 5):
        for room in (0, 3, 9, 40):
            assert check([c, 2, 3, 4], [7, 5, 1, 2], 5, [10, edge, 12, edge - 1], 0, table, room) > 0


def test_long_lists_with_a_few_bad_entries():
    g = torch.Generator().manual_seed(5)
    n, width = 700, 40
    ctx = torch.randint(0, 200, (n,), generator=g).tolist()
    new = torch.randint(0, 300, (n,), generator=g).tolist()
    table = torch.full((n, width), -9, dtype=torch.int32)
    for r in range(n):
        k = -(-ctx[r] // 16)
        table[r, :k] = torch.arange(k) + r * width
    free = (torch.randperm(9000, generator=g) + n * width).tolist()
    assert check(ctx, new, 16, free, 1, table, sum(new) + 3) == 0
    for at in (1, 2, 255, 256, 1500, 4001, 6000):
        free[at] = -1 if at % 2 else BIG
    taken = sum(-(-(c + m) // 16) + c // -16 for c, m in zip(ctx, new))
    assert taken > 6000
    for room in (sum(new), 50000):
        assert check(ctx, new, 16, free, 1, table, room) > 0
    free = free[:5000]
    check(ctx, new, 16, free, 1, table, sum(new))
