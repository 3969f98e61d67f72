"""Calls of the long-session operators named by the kernel and plan that they are
meant to reach (tests/test_session_plans.py checks on the CPU that they do;
tests/test_gpu_session_plans.py runs them, each at both head dims and output
types)."""

DIMS = (64, 128)
OUTPUTS = (False, True)   # f32

# class, Hq, Hkv, Lq, caches, new_lens, starts
STEPS4 = [
    ("few rows, whole", 64, 8, 1, [300, 7], None, None),
    ("few rows, in parts", 16, 4, 3, [4001, 9001, 63], [3, 1, 2], [0, 0, 2]),
    ("one split, few rows", 16, 8, 2, [40, 3, 64, 0] * 8, [1, 2, 2, 1] * 8, None),
    ("one split", 64, 32, 300, [200] * 8, None, [270] * 8),      # several busy waves and query tiles
    ("one split", 24, 24, 256, [900, 889] + [900] * 7, None, None),
    ("splits", 4, 2, 70, [300] * 40, None, [10] * 40),           # lengths from memory
    ("splits", 6, 2, 200, [2500, 2490], [200, 180], None),
    ("per stream, split", 64, 8, 70, [2000, 300, 40, 0], None, None),
    ("per stream, split", 64, 8, 70, [2000, 300, 40, 0], [70, 3, 64, 65], [60, 0, 64, 1]),
    ("per stream, whole", 64, 32, 300, [1800, 100, 100, 60, 30, 7, 0, 300], None, None),
]

# class, Hq, Hkv, Lq, caches, new_lens, starts, window, sinks
STEPS_WINDOW = [
    ("one split, few rows", 8, 2, 12, [100, 71] * 16, None, [6] * 32, 64, 5),
    ("one split", 64, 32, 300, [200] * 8, None, [270] * 8, 150, 5),
    ("one split", 48, 24, 200, [700, 690] * 8, None, None, 300, 65),
    ("splits", 6, 2, 300, [640, 90], None, [60, 300], 300, 130),
    ("per stream, split", 24, 8, 90, [20000, 300, 300, 8], [90, 33, 64, 1], [80, 33, 0, 0], 9000, 100),
    ("per stream, split", 64, 8, 70, [2000, 300, 40, 0], None, None, 1500, 5),
    ("per stream, whole", 64, 32, 300, [1800, 100, 100, 60, 30, 7, 0, 300], None, [290] * 8, 1500, 3),
    ("per stream, whole", 48, 24, 200, [700, 690] * 8, [200, 33] * 8, None, 300, 65),
]

# key groups, B, Hq, Hkv, L, blocks, text, window, sinks; contiguous and paged
PREFILLS = [
    (1, 2, 40, 8, 1600, 30, True, 300, 17),
    (1, 2, 40, 8, 1500, 12, False, 300, 130),
    (2, 2, 6, 2, 1300, 30, True, 100, 17),
]


def step_class(plan, rows):
    """The class of a recorded plan (tests/session_plan_probe.py)."""
    if plan.kernel == "few rows":
        return "few rows, in parts" if plan.splits > 1 else "few rows, whole"
    if plan.per_stream:
        return "per stream, split" if plan.splits > 1 else "per stream, whole"
    return "splits" if plan.splits > 1 else "one split" if rows > 64 else "one split, few rows"
