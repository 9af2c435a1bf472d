"""Workspace sizes of the vocabulary calls, on the host: what a call lays out fits what was asked for, for every batch up to
the one that the workspace was sized for."""
import pytest


def B():
    from paper_2605_16154_b200 import binding
    return binding


def layout(n, vocab, d):
    """Bytes that the gradient of n embedding rows uses: two buffers of (token, position) pairs, marks of present tokens,
    digit counts of up to 256 blocks of whole thousands of pairs, and for each tile of 32 sorted pairs (8 below 9472) a job and
    two partial rows; first tiles of the tokens."""
    tiles = -(-n // (32 if n >= 9472 else 8))
    keys = max(1, -(-(-(-n // 256)) // 1024)) * 1024
    return 16 * n + vocab + -(-n // keys) * 256 * 4 + 8 * tiles + 4 * vocab + 2 * 4 * (-(-d // 4) * 4) * tiles


EDGES = (1, 2, 7, 8, 9, 31, 33, 1000, 1024, 1025, 2047, 2049, 2368, 2369, 4504, 8191, 9000, 9465, 9471, 9472, 9473, 10496, 16384, 21248,
         33536, 37887, 37889, 131073, 200000, 262143, 262144, 262145, 263169, 400000, 524289)


@pytest.mark.parametrize("vocab,d", [(1, 1), (1003, 520), (32000, 1024), (50257, 4096), (100000, 1024), (700, 8), (131072, 65536)])
def test_a_workspace_serves_every_shorter_batch(vocab, d):
    b = B()
    for most in EDGES:
        have = b.grpo_embed_workspace_bytes(most, vocab, d)
        for n in EDGES:
            if n <= most:
                assert layout(n, vocab, d) <= have, (most, n)
                assert b.grpo_embed_workspace_bytes(n, vocab, d) <= have, (most, n)


@pytest.mark.parametrize("n,d,vocab,chunk", [(42536, 1024, 32000, 33536), (30248, 1024, 50257, 21248), (30248, 4096, 50257, 21248),
                                             (15000, 1024, 100000, 10496), (28000, 512, 50000, 21248), (25384, 1024, 32000, 16384),
                                             (12000, 64, 900, 10000), (500000, 64, 300, 300000), (9473, 256, 1000, 9472), (9471, 256, 1000, 1)])
def test_the_last_chunk_of_the_head_gradient_fits(n, d, vocab, chunk):
    """The workspace behind the rows, d z, parts and factors of a full chunk holds the sums of any shorter one."""
    b = B()
    up = lambda v: -(-v // 256) * 256
    rows = min(n, chunk)
    have = b.grpo_head_logp_bwd_workspace_bytes(n, d, vocab, chunk)
    front = up(2 * rows * d) + 2 * up(2 * rows * (-(-vocab // 32) * 32)) + up(4 * rows) * 2 + 148 * 128 * 256 * 4
    for r in {rows, n % rows or rows, *(e for e in EDGES if e <= rows)}:
        assert front + layout(r, vocab, d) <= have, r


def test_no_size_falls_as_the_rows_grow():
    b = B()
    for size in (lambda n: b.grpo_embed_workspace_bytes(n, 32000, 1024), lambda n: b.grpo_head_logp_bwd_workspace_bytes(n, 1024, 64, 1 << 20)):
        sizes = [size(n) for n in range(1, 12000)]
        assert all(p <= q for p, q in zip(sizes, sizes[1:]))
    sizes = [b.grpo_embed_workspace_bytes(n, 32000, 8) for n in range(260000, 264000)]
    assert all(p <= q for p, q in zip(sizes, sizes[1:]))


@pytest.mark.parametrize("vocab", [1, 63, 700, 9473, 32000, 40000, 50257, 130011])
def test_the_log_probabilities_of_the_longest_batch_leave_room_for_shorter_ones(vocab):
    """Up to 128 rows a tile has 64 to 256 columns and leaves two parts of 16 bytes a row; beyond, 256."""
    b = B()
    sizes = [b.grpo_head_logp_workspace_bytes(n, 1024, vocab) for n in range(1, 1200)]
    assert all(p <= q for p, q in zip(sizes, sizes[1:]))
    assert all(s >= 32 * n * -(-vocab // 256) for n, s in enumerate(sizes, 1))
