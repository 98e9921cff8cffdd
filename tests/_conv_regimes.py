"""Calls of the short causal convolution that run its main loops, (layout, batch, L, D, W, io, packed), and what each of them reaches."""
# rows: several steps loaded ahead inside a tile ("inside"), more tiles than a workgroup has at a time ("turns").
# time: several visits of a slot ("visits"), several slots of a workgroup ("turns"); forward, several pieces of a lane ("pieces").
CASES = [("bld", 2, 9000, 520, 4, "bf16", False, {"inside"}), ("bld", 2, 9001, 520, 3, "f32", False, {"inside"}), ("bld", 1, 3001, 6144, 4, "bf16", False, {"inside"}),
         ("bld", 2, 8003, 6144, 4, "f32", False, {"inside", "turns"}), ("bld", 4, 5003, 6144, 3, "bf16", False, {"inside", "turns"}), ("bld", 5, 9001, 1029, 2, "bf16", False, {"inside"}),
         ("bld", 6, 20011, 264, 4, "bf16", True, {"inside"}), ("bld", 60, 24000, 3074, 4, "f32", True, {"inside", "turns"}), ("bld", 9, 9001, 4100, 3, "bf16", True, {"inside"}),
         ("bdl", 8, 2048, 1536, 4, "bf16", False, {"visits", "turns", "pieces"}), ("bdl", 8, 2049, 1536, 4, "f32", False, {"visits", "turns"}), ("bdl", 3, 4099, 771, 3, "bf16", False, {"visits", "turns"}),
         ("bdl", 2, 9001, 1030, 2, "f32", False, {"visits", "turns"}), ("bdl", 2, 40001, 771, 4, "f32", False, {"visits", "turns", "pieces"}),
         ("bdl", 24, 16389, 512, 4, "bf16", True, {"visits", "turns"}), ("bdl", 5, 9001, 1030, 3, "f32", True, {"visits", "turns"}), ("bdl", 400, 16384, 2048, 2, "bf16", True, {"turns"}),
         ("bdl", 7, 40003, 2000, 4, "bf16", True, {"visits", "turns", "pieces"})]


def boundaries(S, L, seed):
    """Sequences of all lengths, some of none and one step; a few steps before the first and after the last."""
    import random
    r = random.Random(seed)
    cu = sorted(r.sample(range(3, L - 2), S + 1))
    for i in range(2, S - 1, 5):
        cu[i] = cu[i - 1] + (i & 1)
    return cu
