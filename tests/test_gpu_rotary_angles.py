"""How right pask_rotary's angles are: pairs (1, 0) come back as the cosine and the sine, nothing added."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("far", [100, 1 << 20, 2 ** 31 - 1])
def test_cosines_and_sines_in_fp32(far, transpose):
    """The table's fractions of a turn and positions are whole numbers, so that the exact angle is known.  Allowed: 2^-33 + 2^-28 of a turn (the
    upper 32 bits, and an eighth of a turn in fp32), and of sincospi a step of the result, 2^-24 below one."""
    import paper_2608_28276_b200 as P
    g = torch.Generator().manual_seed(far % 1000)
    n, pairs = 2000, 128
    pos = torch.randint(-far, far, (n,), generator=g)
    pos[:4] = torch.tensor([0, 1, -1, far - 1])
    table = torch.randint(-2 ** 63, 2 ** 63 - 1, (pairs,), generator=g)
    table[:6] = torch.tensor([1 << 61, -(1 << 61), 1 << 62, -2 ** 63, (1 << 61) - 1, 3 << 60])          # eighths and quarters: ends of what is left
    x = torch.zeros(n, 1, 2 * pairs, device="cuda")
    x[..., :pairs] = 1.0
    y = torch.empty_like(x)
    P.pask_rotary(pos.to(torch.int32).cuda(), table.cuda(), [(x, y)], transpose=transpose)
    # modulo 2^64 in signed 64-bit arithmetic, then its upper 53 bits as a part of a turn: off by 2^-54
    turn = (pos[:, None] * table[None]).cuda().double() / 2.0 ** 64
    ang = (turn - turn.round()) * (2 * math.pi) * (-1 if transpose else 1)
    off = torch.maximum((y[:, 0, :pairs].double() - ang.cos()).abs(), (y[:, 0, pairs:].double() - ang.sin()).abs())
    assert off.max().item() <= 2 * math.pi * (2.0 ** -33 + 2.0 ** -28) + 2.0 ** -24
