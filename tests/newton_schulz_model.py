"""What rounding does to the Newton-Schulz iteration: the iteration with the kernels' arithmetic followed, and its distance from the
same without errors.

A product's operands are numbers in two binary16 planes, hi + lo, which are formed here as they are there; the product of the
lower planes is left out.  The rest is summed in binary32, and matrix instructions round a running sum once per 16 terms, or
three times where both cross terms are added to the same sum (`roundings`).  Those errors are drawn: a sum of K terms with random signs is, at
its k-th, about sqrt(k / K) of s = sqrt(sum of the terms' squares), a rounding is off by up to 2^-24 of it (3/4 of that on
average over where it lies between powers of two), and they add up like random ones: up to 2^-24 3/4 sqrt(K / 32) s for one
rounding per 16 terms.  `bits`: operands are rounded to as many first, for the check that fewer are seen."""


def _planes(torch, v, bits):
    """v as two binary16 planes of 2^e v, e such that the largest is below 2^15"""
    most = float(v.abs().max())
    scale = 2.0 ** (14 - int(torch.tensor(most).log2().floor())) if most > 0 else 1.0
    if bits:
        m, e = torch.frexp(v)
        v = torch.ldexp((m * 2.0 ** bits).round(), e - bits)
    v = v * scale
    hi = v.half().double()
    return hi / scale, (v - hi).half().double() / scale


def _product(torch, left, right, gen, bits, roundings, symmetric=True):
    if gen is None:
        return left @ right
    (a, b), (c, d) = _planes(torch, left, bits), _planes(torch, right, bits)
    got = a @ c + (a @ d + b @ c)
    spread = ((left * left) @ (right * right)).sqrt()
    draw = torch.rand(got.shape, dtype=torch.float64, generator=gen, device=got.device) * 2 - 1
    got = (got + spread * draw * (0.75 * 2.0 ** -24 * (roundings * left.shape[1] / 32) ** 0.5)).float().double()
    return got.tril() + got.tril(-1).t() if symmetric else got


def iterate(torch, g, coefficients, eps=1e-7, gen=None, phase=1, bits=0, roundings=1):
    """g: a matrix; phase: steps between products with X.  gen: None for no errors."""
    x = g.double()
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.t().contiguous()
    norm = float(torch.linalg.vector_norm(x)) + float(torch.tensor(eps, dtype=torch.float32))
    x = x / norm if norm > 0 else x * 0
    co = torch.tensor(coefficients, dtype=torch.float32).double().tolist()
    one = torch.eye(x.shape[0], dtype=torch.float64, device=x.device)
    phases = -(-len(co) // phase)
    step = 0
    for i in range(phases):
        a, q = _product(torch, x, x.t().contiguous(), gen, bits, roundings), None
        end = (len(co) * (i + 1) + phases - 1) // phases
        while step < end:
            ca, cb, cc = co[step]
            p = ca * one + cb * a + cc * _product(torch, a, a, gen, bits, roundings)
            q = p if q is None else _product(torch, p, q, gen, bits, roundings)
            step += 1
            if step < end:
                a = _product(torch, _product(torch, p, a, gen, bits, roundings), p, gen, bits, roundings)
        x = _product(torch, q, x, gen, bits, roundings, False)
    return x.t() if tall else x


def predicted(torch, g, coefficients, eps=1e-7, seeds=2, **how):
    """(the exact result, the largest distance of one with errors from it)"""
    want = iterate(torch, g, coefficients, eps)
    off = 0.0
    for seed in range(seeds):
        gen = torch.Generator(device=g.device).manual_seed(seed)
        off = max(off, float(torch.linalg.vector_norm(iterate(torch, g, coefficients, eps, gen, **how) - want)))
    return want, off


def allowed(torch, g, coefficients, eps=1e-7, phases=(1,), roundings=1):
    """(the exact result, how far off the kernels' may be): twice what the model is off, and eight roundings of the result's
    size, for matrices so small that a few draws say little"""
    off, seeds = 0.0, 8 if g.numel() < 1000 else 2
    for phase in phases:
        want, more = predicted(torch, g, coefficients, eps, seeds, phase=phase, roundings=roundings)
        off = max(off, more)
    return want, 2 * off + 8 * 2.0 ** -24 * float(torch.linalg.vector_norm(want))


def share_allowed(torch, g, coefficients, dtype, phases=(1,), roundings=1, gain=1.0):
    """(the nearest numbers of a 16-bit type to the exact result, what share of a result may be others): twice the model's"""
    near, share = (iterate(torch, g, coefficients) * gain).to(dtype), 0.0
    for phase in phases:
        gen = torch.Generator(device=g.device).manual_seed(phase)
        drawn = (iterate(torch, g, coefficients, gen=gen, phase=phase, roundings=roundings) * gain).to(dtype)
        share = max(share, float((drawn != near).double().mean()))
    return near, 2 * share + 8 / g.numel()
