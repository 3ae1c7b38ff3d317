"""The scratch that is asked for some tokens is enough for fewer: a program that sizes its buffers once, for the most it will send, is not refused
later.  Sizes only: none of this needs a GPU."""
import ctypes as C
import random

from paper_1711_00244_amd import binding
from paper_1711_00244_amd.binding import CL_OK, MxExpertsCall, MxMatrix


def test_lists():
    L, n = binding.lib(), C.c_size_t(0)

    def need(tokens, k, experts):
        assert L.cl_expert_lists_bytes(tokens, k, experts, n) == CL_OK
        return n.value

    for k, experts in ((1, 1), (1, 1024), (3, 300), (8, 64)):
        most = 0
        # around every multiple of 2^12 pairs that begins another chunk, of 2^20 that makes chunks longer, and where counts get a launch of their own
        for pairs in sorted({p + d for p in (4096, 8192, 32768, 1 << 18, 1 << 20, 1 << 21, 3 << 20, 1 << 24) for d in range(-9, 10)}):
            now = need(pairs // k, k, experts)
            assert now >= most, (pairs, k, experts, now, most)
            most = now


def experts_need(M, K, experts, x_type, tokens, k, weighted, x_per_pair):
    L, n = binding.lib(), C.c_size_t(0)
    call = MxExpertsCall(tokens, k, 256, 256 if weighted else None, None, None, 0, x_per_pair)
    assert L.cl_mx_experts_workspace_bytes(MxMatrix(None, None, M, K), experts, call, x_type, n) == CL_OK
    return n.value


def test_experts():
    # in these, one launch is priced below several again at a few tokens more (where another tile begins)
    shapes = [(2315, 3491, 128, 1), (3658, 6767, 128, 1), (1394, 4481, 128, 6), (1987, 5873, 128, 7), (1398, 4547, 128, 6), (1306, 5327, 128, 7)]
    rng = random.Random(5)
    shapes += [(rng.randint(1, 3000), rng.randint(1, 6000), rng.choice([4, 32, 128]), rng.randint(1, 4)) for _ in range(10)]
    for M, K, experts, k in shapes:
        for x_per_pair in (0, 1):
            needs = [experts_need(M, K, experts, 0, tokens, k, True, x_per_pair) for tokens in range(0, 60)]
            assert needs == sorted(needs), (M, K, experts, k)


def test_products_that_one_launch_does():
    """0 is asked only where every smaller batch is done in one launch too; else room for X's codes."""
    L, n = binding.lib(), C.c_size_t(0)
    rng = random.Random(6)
    for _ in range(40):
        M, K = int(2 ** rng.uniform(0, 13)), int(2 ** rng.uniform(0, 14.6))
        some = False
        for batch in range(0, 400):
            assert L.cl_mx_fc_workspace_bytes(MxMatrix(None, None, M, K), batch, 0, n) == CL_OK
            some |= n.value > 0
            assert not some or n.value >= batch * binding.mx_row_blocks(K) * 17, (M, K, batch)
