"""Batches of trees that reach the forms of tree attention for many rows; which form the plan takes for each is tested apart, so that a change of its rules
does not leave a form without tests unseen."""

# before: tokens in front of each tree; n: its nodes; budget: 0 or that of a chosen prefix; rows: of a workgroup, as the plan chooses.
SHAPES = {
    # one step to a dozen, of 256 rows and a few less
    "steps": dict(H=32, G=4, before=[11 * i for i in range(33)], n=[17 + i % 16 for i in range(33)], budget=0, rows=256),
    # cut into pieces, of lengths and trees that differ
    "pieces": dict(H=32, G=8, before=[0, 31, 2500, 64, 1000, 777, 2049, 3, 1500, 640] * 2, n=[33 + (7 * i) % 32 for i in range(20)], budget=0, rows=256),
    # chosen prefixes within one piece, ones shorter than the budget among them
    "lists": dict(H=32, G=8, before=[0, 5, 300, 700, 1, 299, 31, 450, 64, 129] * 2, n=[33 + (5 * i) % 32 for i in range(20)], budget=300, rows=256),
    # long ones in several pieces
    "long lists": dict(H=32, G=8, before=[4500, 4096, 100, 5000, 4097, 3000, 6000, 33, 4200], n=[64, 33, 40, 64, 50, 63, 34, 64, 47], budget=4096, rows=256),
    # trees of more nodes than a workgroup has rows for: several share the tokens
    "wide trees": dict(H=16, G=4, before=[100, 0, 513] * 11, n=[256, 100, 65] * 11, budget=0, rows=256),
    # 65 to 128 rows
    "128 rows": dict(H=8, G=2, before=[0, 40, 500, 63], n=[17, 32, 25, 31], budget=0, rows=256),
    "128 rows of lists": dict(H=8, G=2, before=[0, 40, 500, 163], n=[17, 32, 25, 31], budget=100, rows=256),
    # 129 to 256 rows in two workgroups of 128
    "two workgroups": dict(H=8, G=2, before=[0, 40, 500], n=[64, 33, 60], budget=0, rows=128),
    "two workgroups of lists": dict(H=8, G=2, before=[0, 40, 500], n=[64, 33, 60], budget=100, rows=128),
}


def bound(s):
    """Tokens of a sequence that the plan is made for."""
    return s["budget"] + max(s["n"]) if s["budget"] else max(a + b for a, b in zip(s["before"], s["n"]))
