"""Into how many sums an 8-bit product splits k: every share has steps, and together they are all of k.  No GPU needed."""
import random
from types import SimpleNamespace

import torch

import paper_1711_00244_amd as cl

F8 = torch.float8_e4m3fn


def test_every_share_has_steps():
    rng, split = random.Random(2), 0
    for n in range(6000):
        M, K, batch = 2 * int(2 ** rng.uniform(0, 12)), int(2 ** rng.uniform(0, 15 if n % 2 else 11)), int(2 ** rng.uniform(0, 12))
        x, y, act = rng.choice([torch.float32, torch.bfloat16, F8]), rng.choice([torch.float32, torch.bfloat16, F8]), rng.choice(["none", "gated"])
        form, splits = cl.f8_fc_resolved_form(SimpleNamespace(shape=(M, K), K=K), batch, x, act, y)
        blocks = cl.f8_row_blocks(K)
        fours = (blocks + 3) // 4
        # (as the kernels divide: fours of steps, the first shares one more)
        each, more = divmod(fours, splits)
        first = [4 * (s * each + min(s, more)) for s in range(splits)]
        steps = [min(4 * (each + (s < more)), blocks - f) for s, f in enumerate(first)]
        assert min(steps) > 0 and sum(steps) == blocks, (M, K, batch, form, splits)
        split += splits > 1
    assert split > 500
