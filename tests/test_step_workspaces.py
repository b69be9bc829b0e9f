"""Workspaces of the norm's and the embedding's gradients: what is enough for the longest and widest call is enough for every smaller one."""
import itertools
import random

import pytest


@pytest.fixture(scope="module")
def rr():
    from paper_2402_12399_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def _around(*values):
    return sorted({v + d for v in values for d in (-1, 0, 1)} | {1, 2, 7, 100})


def _never_less(size, firsts, seconds):
    at = {(a, b): size(a, b) for a, b in itertools.product(firsts, seconds)}
    for a0, a1 in zip(firsts, firsts[1:]):
        for b in seconds:
            assert at[a0, b] <= at[a1, b], (a0, a1, b, at[a0, b], at[a1, b])
    for b0, b1 in zip(seconds, seconds[1:]):
        for a in firsts:
            assert at[a, b0] <= at[a, b1], (a, b0, b1, at[a, b0], at[a, b1])


def test_norm_sizes_grow_with_the_matrix(rr):
    rows = _around(4, 16, 148, 296, 592, 1184, 16384, 1 << 20, (1 << 31) - 2)
    cols = _around(8, 64, 512, 1024, 2048, 4096, 4104, 8192, 16384, 20000, 32767)
    _never_less(rr.norm_workspace_bytes, rows, cols)
    r = random.Random(1)
    for _ in range(3000):
        M, N = int(10 ** r.uniform(0, 6)), r.randint(1, 32768)
        assert rr.norm_workspace_bytes(r.randint(1, M), r.randint(1, N)) <= rr.norm_workspace_bytes(M, N), (M, N)


def test_embedding_sizes_grow_with_the_batch(rr):
    def size(n, d):
        return rr.embed_workspace_bytes(n, 1000, d)[1]
    tokens = _around(32, 128, 16384, 65535, 131072, 262144, 524288, 1 << 20, (1 << 30) - 1)
    widths = _around(8, 256, 512, 1024, 2048, 4096, 5000, 8192, 1 << 20, (1 << 26) - 1)
    _never_less(size, tokens, widths)
    r = random.Random(2)
    for _ in range(3000):
        n, d = int(2 ** r.uniform(0, 24)), int(2 ** r.uniform(0, 14))
        assert size(r.randint(1, n), r.randint(1, d)) <= size(n, d), (n, d)


def test_embedding_sizes_are_enough_for_every_piece(rr):
    """Two pieces of a row in fp32 for every chunk of 8 tokens (16 and 32 where there are enough of them to fill the SMs), and sorted ids and places."""
    for n, d in itertools.product((129, 1000, 16384, 16385, 65535, 65536, 131071, 131072, 1 << 20), (1, 100, 256, 257, 1000, 1024, 4096, 8192)):
        warps = -(-d // 256)
        chunk = 32 if n * warps >= 32 << 14 else 16 if n * warps >= 16 << 14 else 8
        need = 256 + -(-n // chunk) * 2 * d * 4 + n * 8 * (2 if n > 16384 else 1) + n // (2 * chunk) * 4
        assert need <= rr.embed_workspace_bytes(n, 1000, d)[1] <= 1.1 * need + 2 * 4 * max(n * d / 8, 1) + 4096


def test_few_tokens_need_no_pieces(rr):
    for n in (1, 37, 128):
        assert rr.embed_workspace_bytes(n, 1000, 1 << 26)[1] <= 1 << 16
