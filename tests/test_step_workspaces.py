"""Sizes of the scratch buffers of norms, embedding and gradient norm, on the CPU: a buffer that is made for a program's largest call serves its smaller ones."""
import random

import paper_2603_05168_amd as sbn


def test_grad_norm_takes_no_less_for_more():
    """One more tensor, or more values in one, never needs less: next to where the kernel's blocks change their length too (32 MB in either type)."""
    need = sbn.sbn_grad_norm_workspace_bytes
    rng = random.Random(1)
    border = [(1 << 23) - 1, 1 << 23, (1 << 24) - 1, 1 << 24]   # 32 MB of fp32, of bf16
    for n in border + [1, 8191, 8192, 8193, 8_000_000, 50_000_000]:
        sizes = [n]
        for _ in range(30):
            more = sizes + [rng.choice(border + [1, 700_000, 8_388_608, rng.randint(1, 1 << 22)])]
            assert need(sizes) <= need(more), (sizes, more)
            at = rng.randrange(len(sizes))
            grown = list(sizes)
            grown[at] += rng.choice([1, 8192, 1 << 20, 1 << 23])
            assert need(sizes) <= need(grown), (sizes, grown)
            sizes = more
    # a group's workspace serves any part of it
    sizes = [2560 * 2560] * 4 + [6912 * 2560] * 3 + [2560] * 2
    for _ in range(50):
        part = rng.sample(sizes, rng.randint(1, len(sizes) - 1))
        assert need(part) <= need(sizes), part
