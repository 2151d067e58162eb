"""Batches behind a shared prefix, by the kernel that they take: head_dim in units of 32, tiles of 16 rows that a sequence and head has (0: many), and
wavefronts to a workgroup.  test_prefix_plan.py holds them to the plan, test_gpu_prefix_widths.py computes them."""

PAGE, SHARED = 16, 9   # 144 tokens: two tiles of 64, and a quarter of one that is read with each sequence's own keys


def batch(tiles, waves):
    """(new tokens, lengths, query heads of a head of the cache): one, two or many tiles of rows to a sequence; 1024 rows of the batch and more
    with eight wavefronts."""
    if tiles == 1:
        new, group = ([1, 1, 2], 8) if waves == 4 else ([1] * 129 + [2], 8)
    elif tiles == 2:
        new, group = ([3, 1, 4], 8) if waves == 4 else ([4, 1, 0, 3] * 17, 8)
    else:
        new, group = ([40, 1, 13], 3) if waves == 4 else ([150, 3, 120, 1, 70], 3)
    return new, [SHARED * PAGE + n + (37 * i) % 190 for i, n in enumerate(new)], group


DIMS = list(range(16, 257, 16))
CASES = [(d, tiles, waves) for d in DIMS for tiles in (1, 2, 0) for waves in (4, 8) if waves == 4 or d <= 128]
