"""The orthogonalised update in 64 bits, and the same steps in the arithmetic that the library documents: every float as the sum of two
fp16 numbers scaled by 4096, three products of them for one, fp32 sums.  What the second is away from the first is what a kernel may be
away from it: the tolerances of the accuracy tests are taken from here, before a kernel has run.

Works on CPU and GPU tensors alike (the device of the matrix)."""
import torch

COEF = (3.4445, -4.7750, 2.0315)
SCALE = 4096.0
HALF = {torch.float32: (24, -126), torch.bfloat16: (8, -126), torch.float16: (11, -14)}      # bits of a number, smallest exponent


def exact(g, steps=5, coef=COEF, eps=1e-7):
    """O in 64 bits; P by Horner's rule from the smaller side."""
    a, b, c = coef
    x = g.double()
    x = x / max(float(torch.linalg.vector_norm(x)), eps)
    tall = x.shape[0] > x.shape[1]
    x = x.t().contiguous() if tall else x
    eye = torch.eye(x.shape[0], dtype=x.dtype, device=x.device)
    for _ in range(steps):
        s = x @ x.t().contiguous()
        x = ((c * s + b * eye) @ s + a * eye) @ x
    return x.t().contiguous() if tall else x


def groups(rows, cols, steps):
    """How many steps each X X^T stands for (coefficients near 3.4445, -4.7750, 2.0315)."""
    m, n = min(rows, cols), max(rows, cols)
    if m < 128 or n < 2 * m or m * n < 1 << 18:
        return [1] * steps
    sizes, left = [], steps
    while left:
        sizes.append(min(left, 2 if sizes else 3))
        left -= sizes[-1]
    return sizes


def pieces(v):
    s = v * SCALE
    h = s.half().float()
    return h, (s - h).half().float()


def kept(v):
    """What is left of a matrix that is stored as its two numbers."""
    h, l = pieces(v)
    return (h + l) / SCALE


def product(v, w, numbers=2):
    """v w with fp32 sums; numbers = 1: of the first fp16 numbers alone."""
    (vh, vl), (wh, wl) = pieces(v), pieces(w)
    s = vh @ wh
    if numbers == 2:
        s = (vl @ wh + vh @ wl) + s
    return s * (1.0 / (SCALE * SCALE))


def documented(g, steps=5, coef=COEF, eps=1e-7, sizes=None, last_numbers=2):
    """O in the documented arithmetic, in 32 bits; sizes: of the groups of steps; last_numbers = 1 plants a last product of 11 bits."""
    a, b, c = coef
    tall = g.shape[0] > g.shape[1]
    x = g.float()
    x = (x.double() / max(float(torch.linalg.vector_norm(x.double())), eps)).float()
    x = x.t().contiguous() if tall else x
    sizes = groups(*g.shape, steps) if sizes is None else sizes
    assert sum(sizes) == steps
    eye = torch.eye(x.shape[0], device=x.device)
    x = kept(x)
    for k, size in enumerate(sizes):
        A = kept(product(x, x.t().contiguous()))
        P = kept(a * eye + b * A + c * product(A, A))
        Q, scale = P, 1.0
        for j in range(1, size):
            A = kept(product(kept(product(A, P)), P))
            P = kept(a * eye + b * A + c * product(A, A))
            Q, scale = (kept(product(P, Q) / 16), 16.0) if j == 1 else (kept(product(P, Q)), 16.0)
        x = scale * product(Q, x, last_numbers if k + 1 == len(sizes) else 2)
        x = x if k + 1 == len(sizes) else kept(x)
    return x.t().contiguous() if tall else x


def samples(g, count=3, **kw):
    """`documented` of G and of G with its values moved by up to half of their last place: other roundings of the same problem."""
    gen = torch.Generator(device=g.device).manual_seed(1)
    out = [documented(g, **kw)]
    for _ in range(count - 1):
        noise = 2.0 ** -24 * (2 * torch.rand(g.shape, generator=gen, device=g.device) - 1)
        out.append(documented(g.float() * (1 + noise), **kw))
    return out


def tolerances(g, **kw):
    """(O in 64 bits, what |error|_F may be, what an element's error may be) of a result in fp32.

    Four times the largest of three samples, since a kernel's order of sums makes it one more sample, and a floor of 2^-20 of the size:
    a dozen roundings to 24 bits, for matrices of a few values, whose samples may have no error at all."""
    kw2 = {k: v for k, v in kw.items() if k != "sizes"}
    want = exact(g, **kw2)
    off = [s.double() - want for s in samples(g, **kw)]
    size = float(torch.linalg.vector_norm(want))
    norm = 4 * max(float(torch.linalg.vector_norm(d)) for d in off) + 2.0 ** -20 * size
    each = 4 * max(float(d.abs().max()) for d in off) + 2.0 ** -20 * float(want.abs().max())
    return want, norm, each


def half_place(v, dtype):
    """Half a unit in the last place of a type at |v|: what rounding to it may change."""
    bits, low = HALF[dtype]
    _, e = torch.frexp(v.double())          # |v| in [2^(e-1), 2^e)
    e = torch.where(v == 0, low, (e - 1).clamp(min=low))
    return torch.ldexp(torch.ones_like(v, dtype=torch.float64), e - bits)


def excess(got, want, dtype, each):
    """How far elements of a result that was rounded once to `dtype` are beyond that rounding, at most: no more than `each`, the
    error of what was rounded, if it was rounded once."""
    got, want = got.double(), want.double()
    return float(((got - want).abs() - half_place(want.abs() + each, dtype)).max())


# Calls, and the way that their first and last matrix takes (xconv_orth_plan_info): every kind of launch and every size of tile, where
# the tests of accuracy and of equal bits go.  The host tests hold the library to this table, so that a threshold that moves shows.
SINGLE, GROUPED = 1, 2
WAYS = {
    "one workgroup": ([(64, 576)], dict(kind=0)),
    "one workgroup, largest": ([(768, 64)], dict(kind=0)),
    "both products, 64 rows": ([(64, 769)], dict(kind=SINGLE, gram_tile=64, gram_runs=2, merge_rows=128, merge_cols=32)),
    "both products, 128 rows": ([(100, 900)], dict(kind=SINGLE, gram_tile=64, gram_runs=2, merge_rows=128, merge_cols=32)),
    "both products, 128 rows, 64 columns": ([(120, 2000)] * 20, dict(kind=SINGLE, gram_tile=64, gram_runs=5, merge_rows=128, merge_cols=64)),
    "both products, 256 rows": ([(200, 147)], dict(kind=SINGLE, gram_tile=64, gram_runs=1, merge_rows=256, merge_cols=32)),
    "both products, 256 rows, 64 columns": ([(250, 700)] * 20, dict(kind=SINGLE, gram_tile=64, gram_runs=1, merge_rows=256, merge_cols=64)),
    "steps, tiles of 64": ([(320, 330)], dict(kind=SINGLE, gram_tile=64, square_tile=64, apply_tile=64, gram_runs=1, square_runs=1)),
    "steps, tiles of 128": ([(700, 710)] * 24, dict(kind=SINGLE, gram_tile=128, square_tile=128, apply_tile=128, gram_runs=2, square_runs=1)),
    "steps, split sums": ([(1600, 1700)], dict(kind=SINGLE, gram_tile=64, square_tile=64, apply_tile=64, gram_runs=2, square_runs=2)),
    "groups, 256 rows": ([(256, 1152)], dict(kind=GROUPED, gram_tile=64, square_tile=64, apply_tile=64, gram_runs=3, square_runs=1)),
    "groups, just wide enough": ([(362, 725)], dict(kind=GROUPED, gram_tile=64, square_tile=64, apply_tile=64, gram_runs=2, square_runs=1)),
    "groups, tall": ([(1100, 260)], dict(kind=GROUPED, gram_tile=64, square_tile=64, apply_tile=64, gram_runs=3, square_runs=1)),
    "groups, apply in tiles of 128": ([(300, 1300)] * 8, dict(kind=GROUPED, gram_tile=64, square_tile=64, apply_tile=128, gram_runs=3, square_runs=1)),
    "groups, tiles of 128": ([(640, 1400)] * 24, dict(kind=GROUPED, gram_tile=128, square_tile=128, apply_tile=128, gram_runs=3, square_runs=1)),
    "groups, split products of A": ([(1600, 3300)], dict(kind=GROUPED, gram_tile=128, square_tile=64, apply_tile=128, gram_runs=4, square_runs=2)),
    "groups, split products of A in tiles of 128": ([(2048, 4096)], dict(kind=GROUPED, gram_tile=128, square_tile=128, apply_tile=128, gram_runs=3, square_runs=3)),
}
