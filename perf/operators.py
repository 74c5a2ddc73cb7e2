"""Work on rows in few bits and on fitting a query encoder to an index, as cases to be timed and compared.

A case is a plain dict.  ``op`` names what is called:

quantize     rows to the microscaled format and back: one scale byte per 32 elements, elements of 4 bits (e2m1)
             or 6 (e2m3); the outputs are the scales and the values that the codes stand for
scores       inner products of quantised queries with quantised rows: S[q, i]
scores_grad  the gradient of those products, to the queries (G X) or, transposed, to the rows (G^T Q)
distill      the distillation loss of the scores from a teacher's ranked lists (ids and scores, as the
             searches return them), and its gradient: ``step`` in one call, ``pair`` the loss and then
             the gradient in a call each, ``loss`` without the gradient

Rows are unit vectors of a Gaussian mixture (sigma 0.3), queries noisy copies of rows, as in the
repository's own workloads; everything is drawn on the GPU from the seed alone.
"""
from __future__ import annotations

import math

import torch

own = False  # True: run() calls the framework's operators; False: their plain form in torch

DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ELEM = {"f32": 4, "bf16": 2, "f16": 2}
BLOCK = 32
TAU, TAU_TEACHER = 0.05, 0.1
EMAX = 2  # the largest exponent of an element, in both types
LARGEST = {4: 6.0, 6: 7.5}


def listed():
    return [
        # one interactive query on its way to an index in few bits: latency
        {"name": "quantize_query", "op": "quantize", "rows": 1, "dim": 1024, "dtype": "f32", "bits": 6},
        # a batch of rows whose width fills neither a block nor a vector load
        {"name": "quantize_odd", "op": "quantize", "rows": 4099, "dim": 100, "dtype": "f32", "bits": 4},
        # a whole index of a million rows at once
        {"name": "quantize_1m", "op": "quantize", "rows": 1048576, "dim": 768, "dtype": "bf16", "bits": 4},
        # one query over the 32K-chunk index: a pass over the rows
        {"name": "scores_b1", "op": "scores", "batch": 1, "rows": 32768, "dim": 1024, "bits": 6, "row_bits": 4,
         "dtype": "f32"},
        # sizes as they come
        {"name": "scores_ragged", "op": "scores", "batch": 77, "rows": 10007, "dim": 384, "bits": 4, "row_bits": 6,
         "dtype": "f16"},
        # the headline batch, 4 bits on both sides
        {"name": "scores_b256", "op": "scores", "batch": 256, "rows": 32768, "dim": 1024, "bits": 4, "row_bits": 4,
         "dtype": "f32"},
        # one evaluation set against a quarter of a million rows
        {"name": "scores_b1024_long", "op": "scores", "batch": 1024, "rows": 262144, "dim": 768, "bits": 6,
         "row_bits": 4, "dtype": "bf16"},
        # one example's gradient over a long index, with half-precision loss scaling
        {"name": "grad_query_b1", "op": "scores_grad", "batch": 1, "rows": 100003, "dim": 384, "bits": 4,
         "dtype": "f16", "to": "queries"},
        # a training batch against the 32K-chunk index: the queries' gradient
        {"name": "grad_queries_b1024", "op": "scores_grad", "batch": 1024, "rows": 32768, "dim": 1024, "bits": 4,
         "dtype": "f32", "to": "queries"},
        # in-batch training of both encoders: the rows' gradient
        {"name": "grad_rows", "op": "scores_grad", "batch": 1000, "rows": 20011, "dim": 768, "bits": 6,
         "dtype": "bf16", "to": "rows"},
        # a training batch's loss and gradient at once, lists as deep as the hybrid search's
        {"name": "distill_step", "op": "distill", "batch": 1024, "rows": 32768, "k": 100, "dtype": "f32",
         "form": "step"},
        # a few examples over a million rows, the loss and the gradient in a call each
        {"name": "distill_long", "op": "distill", "batch": 3, "rows": 1000003, "k": 16, "dtype": "bf16",
         "form": "pair"},
    ]


def _log_uniform(rng, lo, hi):
    v = int(min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))
    return v - 1 if v == 3072 else v


def _dim(rng, largest=2048):
    # half as index widths are (multiples of 128), half any width
    d = 128 * rng.randint(1, largest // 128) if rng.random() < 0.5 else _log_uniform(rng, 33, largest)
    return min(d, largest)


def draw(rng):
    op = rng.choice(["quantize", "scores", "scores_grad", "distill"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    if op == "quantize":
        dim = _dim(rng)
        rows = _log_uniform(rng, 1, min(1000000, 1048576 * 768 // dim))
        return {"op": op, "rows": rows, "dim": dim, "dtype": dtype, "bits": rng.choice([4, 6])}
    if op == "scores":
        dim = _dim(rng, 1024)
        batch = _log_uniform(rng, 1, 1024)
        rows = _log_uniform(rng, 257, min(400000, 1024 * 262144 * (1 if dtype != "f32" else 0.5) // batch))
        return {"op": op, "batch": batch, "rows": rows, "dim": dim, "bits": rng.choice([4, 6]),
                "row_bits": rng.choice([4, 4, 6]), "dtype": dtype}
    if op == "scores_grad":
        dim = _dim(rng, 1024)
        batch = _log_uniform(rng, 1, 1024)
        rows = _log_uniform(rng, 257, min(200000, 1024 * 32768 // batch))
        return {"op": op, "batch": batch, "rows": rows, "dim": dim, "bits": rng.choice([4, 6]), "dtype": dtype,
                "to": rng.choice(["queries", "queries", "rows"])}
    batch = _log_uniform(rng, 1, 1024)
    rows = _log_uniform(rng, 129, min(1000000, 1024 * 32768 // batch))
    return {"op": op, "batch": batch, "rows": rows, "k": rng.randint(1, 128), "dtype": dtype,
            "form": rng.choice(["step", "pair", "loss"])}


# ------------------------------------------------------------------------------------- inputs
def _unit(x):
    return x / x.norm(dim=1, keepdim=True)


def _mixture(g, n, d, dev):
    centres = torch.randn((256, d), generator=g, device=dev)
    comp = torch.randint(0, 256, (n,), generator=g, device=dev)
    return _unit(torch.randn((n, d), generator=g, device=dev).mul_(0.3).add_(centres[comp]))


def _noisy_copies(g, rows, n, dev):
    src = torch.randint(0, rows.shape[0], (n,), generator=g, device=dev)
    return _unit(rows[src] + 0.1 * torch.randn((n, rows.shape[1]), generator=g, device=dev))


def _pow2(e):
    """2^e of whole numbers -126 <= e <= 127, exactly, fp32."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _quantize(x, bits):
    """Plain quantisation of x [m x d]: (codes uint8 [m, nb, 16 or 24], scales uint8 [m, nb])."""
    m, d = x.shape
    nb = (d + BLOCK - 1) // BLOCK
    x = torch.nn.functional.pad(x.float(), (0, nb * BLOCK - d)).view(m, nb, BLOCK)
    amax = x.abs().amax(dim=2)
    # floor(log2 amax) is frexp's exponent less one; below 2^-125 the smallest scale holds
    e = (torch.frexp(amax)[1] - 1 - EMAX).clamp(-127, 127)
    e = torch.where(amax > 0, e, torch.full_like(e, -127))
    # x / 2^e in two exact steps (2^-e passes the type's range where e is near either end)
    half = torch.div(e, 2, rounding_mode="floor")
    v = x * _pow2(-half)[..., None] * _pow2(half - e)[..., None]
    mag = v.abs().clamp(max=LARGEST[bits])
    # the step between values is `fine` below 2, twice that below 4, four times above; a code is the
    # number of steps up to the value
    fine = 0.5 if bits == 4 else 0.125
    step = torch.where(mag < 2, fine, torch.where(mag < 4, 2 * fine, 4 * fine))
    r = (torch.round(mag / step) * step).clamp(max=LARGEST[bits])
    place = torch.where(r < 4, 2 / fine + (r - 2) / (2 * fine), 3 / fine + (r - 4) / (4 * fine))
    place = torch.where(r < 2, r / fine, place)
    code = place.to(torch.int32) | (torch.signbit(v).to(torch.int32) << (bits - 1))
    if bits == 4:
        code = code.view(m, nb, 16, 2)
        codes = (code[..., 0] | (code[..., 1] << 4)).to(torch.uint8)
    else:
        code = code.view(m, nb, 8, 4)
        word = code[..., 0] | (code[..., 1] << 6) | (code[..., 2] << 12) | (code[..., 3] << 18)
        codes = torch.stack((word & 255, (word >> 8) & 255, word >> 16), dim=3).to(torch.uint8).view(m, nb, 24)
    bad = ~torch.isfinite(x).all(dim=2)
    codes = torch.where(bad[..., None], torch.zeros_like(codes), codes)
    scales = torch.where(bad, torch.full_like(e, 255), e + 127).to(torch.uint8)
    return codes.contiguous(), scales


def _values(codes, scales, dim):
    """What codes and scales stand for, fp32 [m x dim]."""
    m, nb, w = codes.shape
    c = codes.to(torch.int32)
    if w == 16:
        c = torch.stack((c & 15, c >> 4), dim=3).view(m, nb, BLOCK)
        exp, man, sign = (c >> 1) & 3, (c & 1).float() / 2, (c & 8) != 0
    else:
        c = c.view(m, nb, 8, 3)
        word = c[..., 0] | (c[..., 1] << 8) | (c[..., 2] << 16)
        c = torch.stack((word & 63, (word >> 6) & 63, (word >> 12) & 63, word >> 18), dim=3).view(m, nb, BLOCK)
        exp, man, sign = (c >> 3) & 3, (c & 7).float() / 8, (c & 32) != 0
    mag = torch.where(exp > 0, (1 + man) * _pow2(exp - 1), man)
    e = scales.to(torch.int32) - 127
    half = torch.div(e, 2, rounding_mode="floor")
    v = torch.where(sign, -mag, mag) * _pow2(half)[..., None] * _pow2(e - half)[..., None]
    v = torch.where((scales == 255)[..., None], torch.full_like(v, math.nan), v)
    return v.reshape(m, nb * BLOCK)[:, :dim]


def prepare(case, seed):
    dev = torch.device("cuda", 0)
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    op, dt = case["op"], DTYPE[case["dtype"]]
    st = {"case": dict(case)}
    if op == "quantize":
        st["x"] = _mixture(g, case["rows"], case["dim"], dev).to(dt)
        return st
    nq, n = case["batch"], case["rows"]
    if op == "scores":
        rows = _mixture(g, n, case["dim"], dev)
        st["q"] = _quantize(_noisy_copies(g, rows, nq, dev), case["bits"])
        st["rows"] = _quantize(rows, case["row_bits"])
        return st
    if op == "scores_grad":
        # the gradient that a distillation batch's mean loss sends back; fp16 with a loss scale of 1,024
        grad = torch.softmax(4 * torch.randn((nq, n), generator=g, device=dev), dim=1)
        hit = torch.randint(0, n, (nq, 16), generator=g, device=dev)
        grad.scatter_add_(1, hit, -torch.softmax(torch.randn((nq, 16), generator=g, device=dev), dim=1))
        st["grad"] = (grad * ((1024.0 if case["dtype"] == "f16" else 1.0) / nq)).to(dt)
        x = _mixture(g, n if case["to"] == "queries" else nq, case["dim"], dev)
        st["x"] = _quantize(x, case["bits"])
        return st
    # student: cosines over the index; a hundredth of the rows is masked (deleted chunks)
    s = 0.15 * torch.randn((nq, n), generator=g, device=dev)
    gone = torch.rand((n,), generator=g, device=dev) < 0.01
    gone[:case["k"]] = False
    s[:, gone] = -math.inf
    t, ids = torch.topk(s + 0.05 * torch.randn((nq, n), generator=g, device=dev), case["k"], dim=1)
    # lists as searches return them: score descending, some shorter than k and padded, one in 64 empty
    length = torch.randint(0, case["k"] + 1, (nq, 1), generator=g, device=dev)
    full = torch.rand((nq, 1), generator=g, device=dev) < 0.75
    empty = torch.rand((nq, 1), generator=g, device=dev) < 1 / 64
    length = torch.where(full, torch.full_like(length, case["k"]), length)
    length = torch.where(empty, torch.zeros_like(length), length)
    pad = torch.arange(case["k"], device=dev)[None, :] >= length
    st["logits"] = s.to(dt)
    st["ids"] = torch.where(pad, torch.full_like(ids, -1), ids).contiguous()
    st["t"] = torch.where(pad, torch.full_like(t, -math.inf), t).contiguous()
    # each example's share of the batch's mean loss; fp16 with a loss scale of 1,024
    share = (1024.0 if case["dtype"] == "f16" else 1.0) / nq
    st["weight"] = torch.rand((nq,), generator=g, device=dev).add_(0.5).mul_(share)
    return st


# --------------------------------------------------------------------------------- the plain form
def _plain_distill(logits, ids, t, weight, want_grad):
    nq, n = logits.shape
    z = logits.float() / TAU
    zmax = z.amax(dim=1, keepdim=True)
    zmax = torch.where(torch.isfinite(zmax), zmax, torch.zeros_like(zmax))
    ez = torch.exp(z - zmax)
    total = ez.sum(dim=1, keepdim=True)
    lse = zmax + torch.log(total)
    valid = (ids >= 0) & (ids < n) & (t > -math.inf)
    at = torch.where(valid, ids, torch.zeros_like(ids))
    u = torch.where(valid, t / TAU_TEACHER, torch.full_like(t, -math.inf))
    umax = u.amax(dim=1, keepdim=True)
    umax = torch.where(torch.isfinite(umax), umax, torch.zeros_like(umax))
    eu = torch.exp(u - umax)
    mass = eu.sum(dim=1, keepdim=True)
    some = mass > 0
    p = torch.where(some, eu / torch.where(some, mass, torch.ones_like(mass)), torch.zeros_like(eu))
    logp = u - umax - torch.log(mass)
    terms = p * (logp - (torch.gather(z, 1, at) - lse))
    loss = torch.where(p > 0, terms, torch.zeros_like(terms)).sum(dim=1)
    if not want_grad:
        return loss, lse[:, 0], None
    grad = torch.where(some, ez / total, torch.zeros_like(ez))
    grad = grad.scatter_add(1, at, -p)
    grad = grad * (weight[:, None] / TAU)
    return loss, lse[:, 0], grad.to(logits.dtype)


def run(st):
    case = st["case"]
    op, dim, dt = case["op"], case.get("dim"), DTYPE[case["dtype"]]
    if own:
        import paper_2608_08340_amd as oprag

        if op == "quantize":
            r = oprag.mx_quantize(st["x"], case["bits"])
            return {"scales": r.scales, "values": oprag.mx_values(r, dt)}
        if op == "scores":
            return {"scores": oprag.mx_scores(oprag.MxRows(*st["q"], dim), oprag.MxRows(*st["rows"], dim), dt)}
        if op == "scores_grad":
            x = oprag.MxRows(*st["x"], dim)
            return {"grad": oprag.mx_scores_grad(st["grad"], x, transposed=case["to"] == "rows")}
        a = (st["logits"], st["ids"], st["t"])
        tau = {"temperature": TAU, "teacher_temperature": TAU_TEACHER}
        if case["form"] == "step":
            loss, grad = oprag.distill_step(*a, st["weight"], **tau)
            return {"loss": loss, "grad": grad}
        loss, lse = oprag.distill_loss(*a, **tau)
        if case["form"] == "loss":
            return {"loss": loss, "lse": lse}
        return {"loss": loss, "lse": lse, "grad": oprag.distill_grad(*a, lse, st["weight"], **tau)}
    if op == "quantize":
        codes, scales = _quantize(st["x"], case["bits"])
        return {"scales": scales, "values": _values(codes, scales, dim).to(dt)}
    if op == "scores":
        return {"scores": (_values(*st["q"], dim) @ _values(*st["rows"], dim).t()).to(dt)}
    if op == "scores_grad":
        g = st["grad"].float()
        return {"grad": (g.t() if case["to"] == "rows" else g) @ _values(*st["x"], dim)}
    loss, lse, grad = _plain_distill(st["logits"], st["ids"], st["t"], st["weight"], case["form"] != "loss")
    out = {"loss": loss}
    if case["form"] != "step":
        out["lse"] = lse
    if grad is not None:
        out["grad"] = grad
    return out


# -------------------------------------------------------------------------------------- the work
def _stored(m, dim, bits):
    """Bytes of m quantised rows."""
    return m * ((dim + BLOCK - 1) // BLOCK) * (BLOCK * bits // 8 + 1)


def work(case):
    es = ELEM[case["dtype"]]
    if case["op"] == "quantize":
        m, d = case["rows"], case["dim"]
        return {"bytes": 2 * m * d * es + _stored(m, d, case["bits"]), "flops": 3 * m * d}
    nq, n = case["batch"], case["rows"]
    if case["op"] == "scores":
        d = case["dim"]
        return {"bytes": _stored(nq, d, case["bits"]) + _stored(n, d, case["row_bits"]) + nq * n * es, "flops": 2 * nq * n * d}
    if case["op"] == "scores_grad":
        d = case["dim"]
        k, m = (n, nq) if case["to"] == "queries" else (nq, n)
        return {"bytes": nq * n * es + _stored(k, d, case["bits"]) + 4 * m * d, "flops": 2 * nq * n * d}
    passes = {"loss": 1, "step": 2, "pair": 3}[case["form"]]  # pair: the gradient's call reads the logits again
    return {"bytes": passes * nq * n * es + nq * case["k"] * 12 + nq * 8,
            "flops": nq * n * (4 if case["form"] == "loss" else 8)}


# ---------------------------------------------------------------------- the definition, in 64 bits
def _magnitudes(bits, dev):
    """The type's non-negative values in order; their place is their code."""
    if bits == 4:
        return torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=dev)
    f = torch.arange(8, dtype=torch.float64, device=dev) / 8
    return torch.cat((f, 1 + f, 2 * (1 + f), 4 * (1 + f)))


def _exact_values(codes, scales, dim):
    m, nb, w = codes.shape
    bits = w // 4
    mags = _magnitudes(bits, codes.device)
    # one bit after the other, lowest first, as the codes are packed
    bit = (codes.long()[..., None] >> torch.arange(8, device=codes.device)) & 1
    place = (bit.view(m, nb, BLOCK, bits) << torch.arange(bits, device=codes.device)).sum(dim=3)
    v = torch.cat((mags, -mags))[place]
    v *= ((scales.long() - 127 + 1023) << 52).view(torch.float64)[..., None]
    return v.reshape(m, -1)[:, :dim]


def _exact_quantize(x, bits):
    """The nearest value of the format under each block's scale (a tie to the even code), fp64."""
    m, d = x.shape
    nb = (d + BLOCK - 1) // BLOCK
    y = torch.zeros((m, nb * BLOCK), dtype=torch.float64, device=x.device)
    y[:, :d] = x.double()
    y = y.view(m, nb, BLOCK)
    top = y.abs().max(dim=2, keepdim=True).values
    # the exponent field of a double is floor(log2) + 1023
    e = (((top.view(torch.int64) >> 52) & 2047) - EMAX).clamp(min=1023 - 127)
    scale = (e << 52).view(torch.float64)
    mags = _magnitudes(bits, x.device)
    v = (y.abs() / scale).clamp(max=float(mags[-1]))
    hi = torch.searchsorted(mags, v).clamp(max=len(mags) - 1)
    lo = (hi - 1).clamp(min=0)
    up, down = mags[hi] - v, v - mags[lo]
    place = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return (torch.sign(y) * mags[place] * scale).view(m, -1)[:, :d]


def exact(case, seed):
    st = prepare(case, seed)
    op, dim = case["op"], case.get("dim")
    if op == "quantize":
        if case["rows"] * dim > 1 << 28:
            return None  # tens of GB of fp64 intermediates
        return {"scales": None, "values": _exact_quantize(st["x"], case["bits"])}
    if op == "scores":
        return {"scores": _exact_values(*st["q"], dim) @ _exact_values(*st["rows"], dim).t().contiguous()}
    if op == "scores_grad":
        g = st["grad"].double()
        return {"grad": (g.t().contiguous() if case["to"] == "rows" else g) @ _exact_values(*st["x"], dim)}
    n = case["rows"]
    z = st["logits"].double() / TAU
    lse = torch.logsumexp(z, dim=1)
    keep = (st["ids"] >= 0) & (st["ids"] < n) & (st["t"] > -math.inf)
    u = (st["t"].double() / TAU_TEACHER).masked_fill(~keep, -math.inf)
    some = keep.any(dim=1)
    p = torch.softmax(u.masked_fill(~some[:, None], 0.0), dim=1).masked_fill(~keep, 0.0)
    at = st["ids"].clamp(min=0, max=n - 1)
    logq = torch.gather(z, 1, at) - lse[:, None]
    loss = torch.where(p > 0, torch.xlogy(p, p) - p * logq, torch.zeros_like(p)).sum(dim=1)
    out = {"loss": loss}
    if case["form"] != "step":
        out["lse"] = lse
    if case["form"] != "loss":
        grad = torch.exp(z - lse[:, None]).masked_fill(~some[:, None], 0.0)
        grad.scatter_add_(1, at, -p)
        out["grad"] = grad * (st["weight"].double() / TAU)[:, None]
    return out
