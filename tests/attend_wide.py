"""Shapes of many layers and heads, as models have them, on which a wave of the few-row attention
stands beside those of adjacent KV heads, and the launch form that each takes: (adjacent KV heads of
a workgroup, waves that share a head's entries and join in LDS, splits joined by a second kernel).
tests/test_attend_wide.py checks the forms against the plan on the CPU, tests/test_gpu_attend_wide.py
the results. Sessions of one case list slots of the same cache."""

# name: (form, L, Hq, Hkv, D, tokens (0: the decode), list lengths, sinks, window, [(code, io)])
ALL = [("int8", "bf16"), ("e4m3", "bf16")]
CASES = {
    "heads4_splits6": ((4, 1, 6), 16, 32, 8, 128, 0, [1500], 0, 0, ALL + [("int8", "f32"), ("e4m3", "f32")]),
    "heads4_splits3": ((4, 1, 3), 36, 32, 8, 128, 0, [900], 0, 0, ALL),
    "heads4_alone": ((4, 1, 1), 32, 32, 8, 64, 0, [700] * 8, 0, 0, ALL),
    "heads4_parts2": ((4, 2, 1), 32, 32, 8, 64, 0, [2100] * 8, 0, 0, ALL),
    "heads4_parts2_splits5": ((4, 2, 5), 36, 8, 8, 64, 0, [14500], 0, 0, ALL),
    "heads2_parts2": ((2, 2, 1), 33, 16, 8, 64, 0, [500], 0, 0, ALL),
    "heads2_parts2_splits4": ((2, 2, 4), 16, 24, 6, 128, 0, [1500], 0, 0, ALL),
    "heads2_parts4": ((2, 4, 1), 128, 4, 2, 64, 0, [2100] * 4, 0, 0, ALL + [("int8", "f32")]),
    "heads2_parts4_splits2": ((2, 4, 2), 150, 4, 2, 64, 0, [4100] * 2, 0, 0, ALL),
    "ragged": ((4, 1, 2), 20, 20, 4, 128, 0, [1900, 1300, 700, 300, 90, 1100], 0, 0, ALL),
    "ragged_window": ((2, 2, 1), 20, 20, 4, 128, 0, [1900, 1300, 700, 300, 90, 1100], 4, 300, ALL),
    "chunk_one_block": ((4, 1, 3), 36, 32, 8, 128, 3, [1300], 0, 0, ALL + [("bf16", "bf16")]),
    "chunk_two_blocks": ((4, 1, 3), 36, 32, 8, 128, 6, [1300], 0, 0, ALL),
    "chunk_two_blocks_joined": ((2, 2, 1), 33, 32, 8, 128, 8, [480], 2, 100, ALL),
    "chunk_two_blocks_splits4": ((4, 1, 4), 12, 40, 8, 128, 5, [1900, 1700], 0, 0, ALL),
    "chunk_ragged": ((4, 1, 1), 48, 20, 4, 128, 3, [1500, 1100, 700, 900], 0, 0, ALL),
    "chunk_bf16_parts2": ((4, 2, 1), 32, 32, 8, 64, 4, [2100] * 8, 3, 0, [("bf16", "bf16")]),
    "chunk_f32": ((4, 1, 6), 16, 16, 8, 128, 4, [1500], 0, 0, [("int8", "f32"), ("e4m3", "f32")]),
}
PARAMS = [(name, code, io) for name, c in CASES.items() for code, io in c[-1]]
