"""Which kernels a call of the orthogonalisation runs on: a host copy of the rules of orthogonalise.hip (plan_product,
plan_all, the choice of the Gram form) with their constants read from the source, so that a test of one form notices
when a change of the rule moves its call to another."""
import os
import re
from collections import namedtuple

_SRC = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_05116_amd", "csrc",
                         "orthogonalise.hip")).read()

Shape = namedtuple("Shape", "rows cols waves per_cu stage square other")
SHAPES = {}
for _name, _r, _c, _wm, _wn in re.findall(r"using (Big|Mid|Small) = Shape<(\d+), (\d+), (\d+), (\d+)>;", _SRC):
    _m = re.search(rf"consider\({_name}\{{\}}, \d, (\d), ([\d.]+), square \? ([\d.]+) : ([\d.]+)\);", _SRC)
    SHAPES[_name] = Shape(int(_r), int(_c), int(_wm) * int(_wn), int(_m.group(1)), *(float(v) for v in _m.groups()[1:]))
PAD = int(re.search(r"\bkPad = (\d+);", _SRC).group(1))
GRAM_ROWS = int(re.search(r"\bkGramRows = (\d+);", _SRC).group(1))
MOST_GAIN = float(re.search(r"\bkMostGain = ([\d.]+)f;", _SRC).group(1))
MOST_SPLIT = int(re.search(r"\(square && rest \? (\d+) : 1\)", _SRC).group(1))
QUINTIC_A = float(re.search(r"kQuintic\[3\] = \{([\d.]+)f", _SRC).group(1))
K_STAGE = 64

Product = namedtuple("Product", "shape split whole rest")     # split 1: every tile whole; rest: tiles computed in parts


def _up(a, b):
    return -(-a // b)


def _tiles(s, square, np_, mp):
    r, c = _up(np_, s.rows), _up(np_ if square else mp, s.cols)
    if not square:
        return r * c
    if s.rows == s.cols:
        return r * (r + 1) // 2
    return r // 2 * (r // 2 + 1) + (r // 2 + 1 if r % 2 else 0)


def plan_product(square, np_, mp, K, batch, big=True, cus=256):
    best, best_us, KT = None, 0.0, K // K_STAGE
    for name, s in SHAPES.items():
        if name == "Big" and not big:
            continue
        fixed, slots = s.square if square else s.other, s.per_cu * cus
        total = _tiles(s, square, np_, mp) * batch
        rounds, rest = divmod(total, slots)
        for split in range(1, (MOST_SPLIT if square and rest else 1) + 1):
            if split > 1 and (split * rest > slots or split > KT // 2):
                break
            us = rounds * (KT * s.stage + fixed)
            if rest and split == 1:
                us += KT * s.stage + fixed
            if split > 1:
                us += _up(KT // 2, split) * 2 * s.stage + fixed + 5.0 + 2.0 * rest * split * (s.rows * s.cols * 4 / 4e6)
            if best is None or us < best_us:
                best, best_us = Product(name, split, total - rest if split > 1 else total, rest if split > 1 else 0), us
    return best


def gain(steps, coef=None):
    now = most = 0.0
    for i in range(steps):
        now = abs(coef[i][0] if coef else QUINTIC_A) * max(now, 1.0)
        most = max(most, now)
    return most


def form(batch, rows, cols, steps=5, coef=None, cus=256):
    """None: the Gram form; else the plans of X X^T, of the n x n product and of X's update, the last with `two`: X in
    two parts."""
    n, m = min(rows, cols), max(rows, cols)
    two = gain(steps, coef) > MOST_GAIN
    if n <= GRAM_ROWS and not two:
        return None
    np_, mp = _up(n, PAD) * PAD, _up(m, PAD) * PAD
    return dict(gram=plan_product(True, np_, mp, mp, batch, cus=cus), sym=plan_product(True, np_, mp, np_, batch, cus=cus),
                apply=plan_product(False, np_, mp, 2 * np_ if two else np_, batch, not two, cus=cus), two=two)


def workspace_bytes(batch, rows, cols, cus=256):
    """Of the general form (orth_layout)."""
    n, m = min(rows, cols), max(rows, cols)
    np_, mp = _up(n, PAD) * PAD, _up(m, PAD) * PAD
    f, g = form(batch, rows, cols, 5, cus=cus) or {}, form(batch, rows, cols, 16, cus=cus)
    sym = g["sym"]
    gram = g["gram"]
    one = f.get("apply") or plan_product(False, np_, mp, np_, batch, cus=cus)
    tiles = max(_tiles(SHAPES[p.shape], False, np_, mp) * SHAPES[p.shape].waves for p in (one, g["apply"]))
    sums = max(p.rest * p.split * SHAPES[p.shape].rows * SHAPES[p.shape].cols * 4 for p in (gram, sym))
    size = rows * cols
    per = _up(size, 256)
    per = 2048 if per < 2048 else _up(per, 4) * 4
    x, q = 2 * batch * np_ * mp, 2 * batch * np_ * np_
    parts = [q] * 2 + [x, x, 2 * x, 2 * x, PAD * np_ * 4, batch * np_ * 4, batch * _up(size, per) * 4, batch * tiles * 4,
             batch * 16, sums]
    return sum(_up(v, 256) * 256 for v in parts)
