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


def test_norm_takes_no_less_for_more():
    """Longer rows and more of them never need less: rows of 512 values go by more blocks than those of 2560, whose shares are longer."""
    need = sbn.sbn_norm_workspace_bytes
    for tokens in (1, 2, 7, 600, 3000, 1 << 20):
        sizes = [need(tokens, d) for d in range(1, 16385)]
        assert sizes == sorted(sizes), tokens
    for d in (1, 64, 512, 1001, 2560, 8192, 16384):
        sizes = [need(tokens, d) for tokens in list(range(1, 5000)) + [1 << k for k in range(13, 25)]]
        assert sizes == sorted(sizes), d
    assert need(1, 1024) <= 3 * 1024 * 4   # one row's shares at most


def test_embedding_takes_no_less_for_more():
    need = sbn.sbn_embedding_workspace_bytes
    rng = random.Random(2)
    for _ in range(20000):
        size = [int(2 ** rng.uniform(0, 20)), int(2 ** rng.uniform(0, 9)), int(2 ** rng.uniform(0, 23))]   # tokens, d_in, vocab
        more = list(size)
        more[rng.randrange(3)] += rng.choice([1, 1, 255, 256, 4096])
        if more[1] * max(more[0], more[2]) <= 1 << 34:   # the most that a call takes
            assert need(*size) <= need(*more), (size, more)
    for vocab in (1 << 14, 1 << 22, 1 << 23):   # where the ids are dealt to more blocks
        assert need(100, 64, vocab) <= need(100, 64, vocab + 1)
