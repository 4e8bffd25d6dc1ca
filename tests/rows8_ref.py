"""Plain references of the 8-bit rows and their products, in 64 bits (test infrastructure)."""
import torch


def quantized(x):
    """(values, exponents) of x [R, K]: float64 [R, ceil(K / 128) * 128] as e4m3 holds them, int64 [R, blocks]."""
    R, K = x.shape
    b = torch.zeros((R, -(-K // 128) * 128), dtype=torch.float64, device=x.device)
    b[:, :K] = x.double()
    b = b.view(R, -1, 128)
    fine = torch.isfinite(b)
    part, power = torch.frexp(torch.where(fine, b, 0.0).abs().amax(dim=-1) / 448)
    e = torch.where(part == 0, 0, (power.long() - (part == 0.5).long()).clamp(min=-127))
    y = torch.where(fine, b, torch.nan) * torch.exp2(-e.double())[..., None]
    step = torch.exp2((torch.frexp(y).exponent - 1).clamp(min=-6).double() - 3)
    return (torch.round(y / step) * step).view(R, -1), e


def held(rows8):
    """(values, exponents) of what the buffers hold, element by element of the documented places; also the
    padding's values and scales."""
    R, K = rows8.rows, rows8.cols
    g, nb, nq = -(-R // 16), -(-K // 128), -(-K // 512)
    dev = rows8.data.device
    r, c = torch.arange(16 * g, device=dev)[:, None], torch.arange(128 * nb, device=dev)[None, :]
    at = ((r // 16) * nb + c // 128) * 2048 + (c % 128 // 64) * 1024 + (c // 16 % 4) * 256 + (r % 16) * 16 + c % 16
    b = torch.arange(4 * nq, device=dev)[None, :]
    sc = ((r // 16) * nq + b // 4) * 64 + (r % 16) * 4 + b % 4
    v = rows8.data[at].view(torch.float8_e4m3fn).double()
    return v, rows8.scale[sc].long() - 127


def product(a, w, bias=None):
    """(a . w^T + bias, what sums of 32 bits may be off by, what an instruction of 8-bit numbers may besides).
    The first: each of K products and sums rounds to 2^-24 of the magnitudes' sum.  The second: an instruction
    adds 128 products with the bits below 2^-13 of their largest left out, at most 128 times."""
    av, ae = held(a)
    wv, we = held(w)
    x = (av.view(len(av), -1, 128) * torch.exp2(ae[:, :av.shape[1] // 128].double())[..., None])[:a.rows]
    y = (wv.view(len(wv), -1, 128) * torch.exp2(we[:, :wv.shape[1] // 128].double())[..., None])[:w.rows]
    flat = lambda t: t.reshape(len(t), -1)  # noqa: E731
    out = flat(x) @ flat(y).t().contiguous()
    most = x.abs().amax(-1) @ y.abs().amax(-1).t().contiguous()
    sums = flat(x).abs() @ flat(y).abs().t().contiguous() * (x.shape[1] * 128 + 2) * 2.0 ** -24
    if bias is not None:
        out = out + bias.double()
    return out, sums, most * 2.0 ** -6
