"""Cases of the attention over a 4-bit cache that run on each of its kernels: (name, rows, lengths, heads, kv heads,
head_dim, dtype, pages that the table is wide, the plan).  The width alone says for which lengths the work is cut.  A
plan: (shared, vectors, waves, key ranges, streamed) of a workgroup (include/sd.h)."""

FEW = [1, 700, 33, 64, 129, 1000, 15, 16, 17, 500, 31, 32, 255, 256, 257, 300]

CASES = [
    ("waves of 8", [5, 1, 3], [600, 33, 1000], 8, 2, 128, "bf16", 64, (0, 16, 8, 1, 0)),
    ("waves of 8, 64 dimensions", [5, 1, 3], [600, 33, 1000], 8, 2, 64, "bf16", 64, (0, 16, 8, 1, 0)),
    ("waves of 8, fp32", [5, 1, 3], [600, 33, 1000], 8, 2, 128, "fp32", 64, (0, 16, 8, 1, 0)),
    ("waves of 8, fp32, 64 dimensions", [5, 1, 3], [600, 33, 1000], 8, 2, 64, "fp32", 64, (0, 16, 8, 1, 0)),
    ("waves of 4: many short sequences", [1] * 32, [min(n, 640) for n in FEW] * 2, 32, 32, 64, "bf16", 40, (0, 16, 4, 1, 0)),
    ("waves of 4: fp32", [2] * 16, FEW, 32, 32, 128, "fp32", 70, (0, 16, 4, 1, 0)),
    ("two tiles", [9] * 16, [n + 8 for n in FEW], 32, 8, 128, "bf16", 150, (0, 32, 4, 1, 0)),
    ("two tiles, 64 dimensions", [5, 4] * 8, [n + 8 for n in FEW], 40, 8, 64, "bf16", 400, (0, 32, 4, 4, 0)),
    ("two tiles, key ranges", [9] * 4, [1300, 20, 700, 64], 32, 8, 128, "bf16", 640, (0, 32, 4, 8, 0)),
    ("few key ranges", [1], [1500], 32, 8, 128, "bf16", 110, (0, 16, 4, 6, 0)),
    ("few key ranges, fp32", [3], [1500], 16, 4, 64, "fp32", 110, (0, 16, 4, 6, 0)),
    ("many key ranges", [2], [9000], 16, 2, 128, "bf16", 600, (0, 16, 4, 37, 0)),
    ("many key ranges, 64 dimensions", [2], [9000], 16, 2, 64, "bf16", 600, (0, 16, 4, 37, 0)),
    ("many key ranges, most empty", [2, 1], [300, 7], 4, 2, 128, "fp32", 2000, (0, 16, 4, 64, 0)),
    ("two key ranges", [1] * 16, [2 * n for n in FEW], 32, 8, 128, "bf16", 170, (0, 16, 8, 2, 0)),
    ("two key ranges, fp32", [2] * 16, [2 * n for n in FEW], 32, 8, 128, "fp32", 170, (0, 16, 8, 2, 0)),
    ("two key ranges, a little over a workgroup to a CU", [1] * 36, (FEW * 3)[:36], 32, 8, 128, "bf16", 520, (0, 16, 8, 2, 0)),
    ("longest first", [1] * 40, [1, 0] + (FEW * 3)[:38], 32, 8, 128, "bf16", 300, (0, 16, 8, 1, 0)),
    ("longest first, workgroups of a sequence apart", [3, 17, 0, 9] * 16, [n + 16 for n in FEW] * 4, 24, 3, 64, "bf16", 300, (0, 32, 4, 1, 0)),
    ("longest first, fp32", [1, 5] * 32, [n + 4 for n in FEW[::-1]] * 4, 16, 8, 128, "fp32", 140, (0, 16, 4, 1, 0)),
    ("streamed", [1] * 32, (FEW * 2)[:32], 32, 8, 128, "bf16", 1100, (0, 16, 8, 1, 1)),
    ("streamed, 64 dimensions", [1] * 32, (FEW * 2)[:32], 16, 16, 64, "bf16", 1100, (0, 16, 8, 1, 1)),
    ("streamed, two tiles", [4] * 32, [n + 3 for n in FEW] * 2, 40, 8, 128, "bf16", 1100, (0, 32, 4, 1, 1)),
    ("streamed, two tiles, 64 dimensions", [4] * 32, [n + 3 for n in FEW] * 2, 40, 8, 64, "bf16", 2100, (0, 32, 4, 1, 1)),
    ("streamed, fp32", [1] * 16, FEW, 32, 32, 128, "fp32", 600, (0, 16, 4, 1, 1)),
    ("streamed, fp32, waves of 8", [1] * 16, FEW, 16, 16, 128, "fp32", 1100, (0, 16, 8, 1, 1)),
    ("streamed, fp32, 64 dimensions", [1] * 16, FEW, 32, 32, 64, "fp32", 1100, (0, 16, 8, 1, 1)),
    ("streamed, key ranges", [2], [2000], 32, 32, 128, "bf16", 8000, (0, 16, 4, 16, 1)),
    ("streamed, key ranges, 64 dimensions", [2], [2000], 32, 32, 64, "bf16", 16000, (0, 16, 4, 16, 1)),
    ("streamed, key ranges, fp32, 64 dimensions", [2], [2000], 32, 32, 64, "fp32", 16000, (0, 16, 4, 16, 1)),
    ("shared", [1030], [1101], 32, 32, 64, "bf16", 69, (1, 128, 4, 1, 0)),
    ("shared, 128 dimensions", [550, 113, 0, 310, 1], [550, 300, 5, 1000, 77], 32, 8, 128, "bf16", 70, (1, 128, 4, 1, 0)),
]


def plan(rows, H, KV, hd, dtype, n_seqs, max_len):
    import ctypes as C
    from paper_2510_11331_amd import _lib
    p = _lib.AttentionQPlan()
    rc = _lib.lib().sd_plan_attention_q(rows, H, KV, hd, n_seqs, max_len, {"bf16": _lib.SD_DTYPE_BF16, "fp32": _lib.SD_DTYPE_F32}[dtype],
                                        C.byref(p))
    assert rc == _lib.SD_OK
    return p.shared, p.vectors, p.waves, p.key_ranges, p.streamed


def kind(plan, hd, dtype):
    """What is code of its own: the kernel, and how its ranges are joined."""
    shared, vectors, waves, ranges, streamed = plan
    return dtype, hd, shared, vectors, waves, streamed, 0 if ranges == 1 else 1 if ranges <= 8 else 2
