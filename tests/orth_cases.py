"""Calls of the orthogonalisation that between them take every kernel and every way of cutting a product, with sides
that end within a tile: (batch, rows, cols, steps)."""

CALLS = [(1, 200, 250, 5), (2, 200, 1000, 5), (1, 6100, 1500, 5), (5, 850, 1000, 5), (3, 1100, 1150, 5), (48, 500, 510, 5),
         (32, 380, 384, 5), (48, 300, 380, 5), (380, 300, 40, 5), (8, 2000, 2040, 5), (5, 1250, 5100, 5),
         (16, 2048, 768, 5), (57, 600, 760, 5), (1, 2500, 2490, 5), (1, 100, 128, 8), (3, 40, 700, 8),
         (48, 380, 250, 8), (8, 1010, 1300, 7)]


def kinds(form):
    """What a form (orth_forms.form) runs: (product, shape of its tiles, how they are cut)."""
    cut = lambda p: "whole" if p.split == 1 else "in parts" if p.whole == 0 else "the last round in parts"  # noqa: E731
    return {("two" if k == "apply" and form["two"] else k, form[k].shape, cut(form[k])) for k in ("gram", "sym", "apply")}
