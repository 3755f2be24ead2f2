"""Calls of hb_attention that between them take every kernel that its choice by size takes: B, Lq, Lk, Hq, Hkv, D."""

FORMS = [(2, 150, 130, 4, 2, 24), (3, 3, 517, 2, 1, 16), (2, 3, 300, 2, 1, 24), (2, 3, 12300, 2, 2, 24),
         (2, 150, 130, 4, 2, 40), (3, 3, 517, 2, 1, 48), (2, 3, 130, 2, 1, 56), (2, 3, 4100, 2, 1, 40),
         (2, 150, 130, 4, 2, 72), (3, 3, 517, 2, 1, 80), (2, 3, 130, 2, 1, 88), (2, 3, 4100, 2, 1, 72),
         (3, 3, 130, 2, 1, 104), (3, 3, 517, 2, 1, 112), (2, 3, 300, 2, 1, 120), (2, 3, 12300, 2, 1, 104),
         # split keys, rows of more than one wave
         (1, 20, 517, 2, 1, 24), (1, 20, 12300, 2, 1, 16), (1, 20, 517, 4, 2, 40), (1, 20, 12300, 2, 1, 48),
         (1, 20, 517, 2, 1, 80), (1, 20, 12300, 2, 1, 88), (1, 20, 517, 2, 1, 112), (1, 20, 12300, 2, 1, 120)]


def instance(parts, groups, Lq, Hq, Hkv, D):
    """(channels rounded up to 32, groups of waves, whether the keys are split, and then whether rows are those of one wave): what is compiled apart."""
    return (D + 31) // 32 * 32, groups, parts > 1, parts > 1 and Lq * (Hq // Hkv) <= 32
