"""Calls of hb_linear that between them take every kernel, every way its rows can stand in memory, with the sum whole and split."""

# rows: where x and w stand.  "copied": 16-byte rows, K a multiple of 8; "even": 4-byte addresses; "odd": any.
ROWS = ("copied", "even", "odd")
FORMS = [
    # few rows
    (5, 300, 1000, "copied"), (5, 300, 1001, "odd"), (3, 70, 8200, "copied"), (3, 70, 8203, "odd"),
    (20, 333, 520, "copied"), (20, 333, 521, "odd"), (30, 100, 6000, "even"), (30, 100, 6001, "odd"),
    (50, 3000, 202, "even"), (50, 3000, 201, "odd"), (60, 96, 5000, "copied"), (60, 96, 5003, "odd"),
    # tiles of 64 x 64: one step of k, an odd number of them, tails of K, parts
    (300, 500, 56, "copied"), (300, 500, 712, "copied"), (513, 769, 4104, "copied"), (65, 130, 3000, "copied"),
    (300, 500, 41, "even"), (300, 500, 715, "even"), (513, 769, 2057, "even"), (300, 500, 43, "odd"), (513, 1500, 331, "odd"), (513, 769, 2057, "odd"),
    # 128 x 64, rows through registers
    (100003, 64, 64, "copied"), (100003, 72, 50, "even"), (50021, 130, 203, "even"), (2000, 2000, 1998, "even"), (8227, 68, 2291, "even"),
    (100003, 72, 64, "odd"), (100003, 72, 47, "odd"), (100003, 40, 100, "odd"),
    # 128 x 128, copied and through registers
    (50021, 130, 200, "copied"), (30000, 200, 56, "copied"), (9000, 100, 4000, "copied"), (4000, 4001, 2001, "even"), (9000, 100, 4001, "even"),
    (30000, 200, 139, "odd"), (4000, 4001, 2001, "odd"), (2000, 2000, 1999, "odd"),
    # 256 x 256
    (4090, 4072, 4104, "copied"), (9000, 8200, 200, "copied"), (8200, 8200, 64, "copied"),
]


def instance(kernel, rows):
    """(kernel, how it loads its rows) by the numbers of linear_plan.hpp: what is compiled apart."""
    if kernel <= 2 or kernel == 4:                        # few rows, and 128 x 64: 16-byte rows as even ones
        return kernel, "odd" if rows == "odd" else "even"
    if kernel == 5:                                       # 128 x 128: even ones as odd ones
        return kernel, "copied" if rows == "copied" else "odd"
    return kernel, rows
