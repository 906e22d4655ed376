"""The cross entropy's plan again in Python: which kernels a call's sizes take,
so that tests can say that they reach each of them.  Its workspace totals are
held against the library's, which the same numbers decide."""
F32, BF16, F16 = 0, 1, 2
STEP, PAD, SKEW = 64, 256, 256
PIECE = 128 << 20
FEW = 64


def up(n, to):
    return -(-n // to) * to


def tiles(a, b, side):
    return -(-a // side) * -(-b // side)


def large(a, b, split):
    return tiles(a, b, 256) * split >= 128 and a > 128 and b > 128


def few_tokens(type, n, v, pack, backward):
    parts = 3 if type == F32 else 1
    if n > FEW or 4 * parts * FEW * v > 2 * PIECE:
        return False
    return pack or -(-v // 128) < 192 or (backward and n <= 32)


def few_rows(n, v):
    own = 16 if n <= 16 else 32
    return 4 * own if -(-v // (4 * own)) >= 512 else own


class Bump:
    def __init__(self):
        self.at = 0

    def take(self, nbytes):
        self.at = up(self.at + nbytes, 256)


def forward(type, n, d, v, aligned):
    """(workspace bytes, [(kernel, tile side, summed steps of a part, tiles)])."""
    pack = type == F32 or not aligned
    parts, dk, b = 3 if type == F32 else 1, up(d, STEP), Bump()
    few = few_tokens(type, n, v, pack, False)
    b.take(8 * -(-v // (few_rows(n, v) if few else 128)) * n)
    b.take(4 * n)
    if few:
        b.take(2 * parts * dk * n if pack else 0)
        return b.at, [("few", 0, 0, 0)]
    piece = v
    if pack:
        piece = min(v, PIECE // (2 * parts * dk) // PAD * PAD)
        b.take(2 * parts * dk * n)
        b.take(2 * parts * dk * piece)
    products = 6 if type == F32 else 1
    return b.at, [product("stats", min(piece, v - v0), n, products * -(-d // STEP), 1) for v0 in range(0, v, piece)]


def product(name, ni, nj, steps, split):
    side = 256 if large(ni, nj, split) else 128
    return name, side, -(-steps // split), tiles(ni, nj, side) * split


def backward(type, n, d, v, aligned, live=None):
    """The same; ``live``: tokens with a gradient (default: all)."""
    pack = type == F32 or not aligned
    parts, products, dk, b = 3 if type == F32 else 1, 6 if type == F32 else 1, up(d, STEP), Bump()
    live = n if live is None else live
    b.take(4 * n)
    b.take(4)
    b.take(4 * n if type == F16 else 0)
    if few_tokens(type, n, v, pack, True):
        nk, piece = 32 if n <= 32 else 64, up(v, 64)
        b.take(2 * parts * dk * n if pack else 0)
        b.take(2 * parts * nk * d)
        b.take(2 * parts * piece * n)
        b.take(2 * parts * nk * v)
        split = min(-(-768 // -(-d // 128)), -(-(piece // 64) // 4))
        b.take(4 * split * n * up(d, 4))
        return b.at, [("few", 0, 0, 0)]
    for k in (n, n, n, 1):
        b.take(4 * k)
    nk, piece = up(n, 8) + SKEW, up(v, PAD)
    most = min(PIECE // (2 * parts * (dk if pack and dk > n else n)), (1 << 22) // parts - SKEW)
    most = PAD if most < PAD else most // PAD * PAD
    if piece > most:
        piece = up(-(-piece // -(-piece // most)), PAD)
    b.take(2 * parts * dk * n)
    b.take(2 * parts * dk * piece if pack else 0)
    b.take(2 * parts * (piece + SKEW) * n)
    b.take(2 * parts * nk * d)
    steps = products * (piece // STEP)
    split = min(-(-256 // tiles(d, n, 256)), max(steps // 8, 1))
    b.take(4 * split * d * up(n, 4))
    w_split = 256 // tiles(d, piece, 256) if tiles(d, piece, 256) <= 64 else 1
    w_split = min(w_split, products * -(-n // STEP) // 8)
    w_split = max(w_split, 1)
    b.take(4 * w_split * piece * up(d, 4) if w_split > 1 else 0)
    runs = []
    for v0 in range(0, v, piece):
        rows = min(piece, v - v0)
        runs.append(product("prob", rows, n, products * -(-d // STEP), 1))
        runs.append(product("dh", n, d, products * -(-rows // STEP), split))
        name, side, _, count = product("dw split" if w_split > 1 else "dw", d, rows, 0, w_split)
        runs.append((name, side, -(-products * -(-live // STEP) // w_split), count))
    return b.at, runs


# (tokens, rows of w, columns, share of tokens without a target) of the cross
# entropies held against 64 bits for the products they reach
CHECKED = [(2100, 14000, 1031, 0.3), (2100, 14000, 1096, 0.28), (3000, 7400, 1032, 0.3), (20000, 1000, 300, 0.1),
           (300, 2000, 512, 0.3), (2500, 1000, 129, 0.9), (70, 700, 136, 0.1)]
