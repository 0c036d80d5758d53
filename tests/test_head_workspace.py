"""What include/moe_mpmc.h says of moe_head_logprobs_backward's workspace, term by term, beside what the query asks for."""
import random

import paper_2605_11537_amd as moe

GIB = 1 << 30


def test_terms():
    L, rng = moe.lib(), random.Random(1)
    sizes = [(4194309, 520, 8), (8192, 768, 50257), (1 << 16, 1024, 1 << 17), (1, 8, 1), (777, 320, 5003), (20, 704, 45094), (16384, 768, 50257), (15009, 256, 256)]
    for _ in range(2000):
        sizes.append(tuple(int(2 ** rng.uniform(0, top)) for top in (20, 8, 18)))
    for N, d, V in sizes:
        d = (d + 7) // 8 * 8
        for dtype, z in ((moe.MOE_F32, 4), (moe.MOE_BF16, 2)):
            need = L.moe_head_logprobs_backward_workspace_bytes(N, d, V, dtype)
            few = -(-N // 16) * -(-V // 32) <= 256
            db = 4 * V * -(-N // (16 if few or N <= 16 else 128 if z == 2 and N > 128 else 32 if z == 4 and N <= 192 and (N - 1) % 64 < 32 else 64))
            # a piece is a multiple of 256 ids, a block of it 512 bytes a row
            dz = N * min(-(-V * z // 512) * 512, max(256 * z, GIB // N + 512))
            dz = max(dz, 8 * N * -(-V // (256 if z == 2 and N > 128 else 128)))
            parts = max(4 * N * d, GIB)
            most = dz + N * 512 + parts + db + 64 * V * d + N * d * z + 512 * N + 4 * N + 4096
            assert 4 * N * d + db + N * d * z + 8 * N <= need <= most, (N, d, V, z, need, most)
    assert L.moe_head_logprobs_backward_workspace_bytes(4194309, 520, 8, moe.MOE_BF16) > 8 * GIB
