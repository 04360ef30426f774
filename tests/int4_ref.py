"""Plain forms, in 64 bits, of the operators with 4-bit weights and cache (include/confspec_int4.h): what a row is stored
as, where a page keeps it, and what the operators compute from it.  Torch on any device; shares no code with the library."""
import math

import torch

HD, PAGE = 128, 2176


def quantise(x):
    """Rows [..., 128] -> codes (int64), s, z (halves), as the header defines them."""
    x = x.double().clamp(-65504.0, 65504.0)
    z = x.min(-1).values.float().half() + 0.0          # (which of two zeros min and max return is open: never -0)
    s = ((x.max(-1).values - z.double()) / 15.0).float().half() + 0.0
    sd = s.double()[..., None]
    c = torch.round((x - z.double()[..., None]) / torch.where(sd > 0, sd, torch.ones_like(sd)))      # ties to even
    c = torch.where(sd > 0, c, torch.zeros_like(c)).clamp(0, 15).to(torch.int64)
    return c, s, z


def _places(dev):
    """(byte, shift) of every element of a page: [16, 128] for keys and for values."""
    t = torch.arange(16, device=dev)[:, None]
    d = torch.arange(HD, device=dev)[None, :]
    e = d % 8
    kw = ((d % 32 // 8) * 16 + t) * 4 + d // 32
    kbit = 32 * kw + torch.where(e % 2 == 0, 2 * e, 2 * e + 14)
    vbit = 8 * 1024 + 32 * ((t // 4 * 16 + d // 8) * 4 + t % 4) + 4 * e
    return kbit, vbit.expand(16, HD)


def write_row(pages, block, head, slot, codes, s, z, is_v):
    """Stores one row in pages [n_blocks, Hkv, 2176] (uint8)."""
    bit = _places(pages.device)[1 if is_v else 0][slot]
    page = pages[block, head]
    for half in (0, 4):                                   # elements of the low, then of the high four bits of their bytes
        at = bit[bit % 8 == half] // 8
        page[at] = (page[at] & (0xF0 if half == 0 else 0x0F)) | (codes[bit % 8 == half] << half).to(torch.uint8)
    par = torch.stack((s, z)).view(torch.uint8)
    base = (2112 if is_v else 2048) + 4 * slot
    page[base:base + 4] = par


def read_pages(pages):
    """Pages [n, 2176] -> (codes, s, z) of keys and of values: float64 [n, 16, 128], [n, 16], [n, 16]."""
    n = pages.shape[0]
    out = []
    for bit, base in zip(_places(pages.device), (2048, 2112)):
        c = (pages[:, (bit // 8).reshape(-1)].to(torch.int64) >> (bit % 8).reshape(-1)) & 15
        par = pages[:, base:base + 64].contiguous().view(torch.float16).double().view(n, 16, 2)
        out.append((c.double().view(n, 16, HD), par[..., 0], par[..., 1]))
    return out


def random_pages(gen, n_layers, n_blocks, Hkv, dev, k_scale=1.0, v_scale=0.5):
    """A cache of quantised normal rows (every page written)."""
    n = n_layers * n_blocks * Hkv
    pages = torch.zeros(n, PAGE, dtype=torch.uint8, device=dev)
    bits = _places(dev)
    mean = torch.randn(HD, generator=gen, device=dev) * 0.5
    for bit, base, x in ((bits[0], 2048, torch.randn(n, 16, HD, generator=gen, device=dev) * k_scale + mean),
                         (bits[1], 2112, torch.randn(n, 16, HD, generator=gen, device=dev) * v_scale)):
        c, s, z = quantise(x.bfloat16())
        for half in (0, 4):
            sel = (bit % 8 == half)
            at = (bit[sel] // 8)
            pages[:, at] |= (c[:, sel] << half).to(torch.uint8)
        pages[:, base:base + 64] = torch.stack((s, z), -1).view(n, 32).contiguous().view(torch.uint8)
    return pages.view(n_layers, n_blocks, Hkv, PAGE)


def rotate(x, pos, theta):
    """x [T, H, 128] at positions pos [T]: half-split pairing, float64."""
    inv = theta ** (-2.0 * torch.arange(64, dtype=torch.float64, device=x.device) / HD)
    ang = pos.double()[:, None, None] * inv
    lo, hi = x[..., :64].double(), x[..., 64:].double()
    return torch.cat((lo * torch.cos(ang) - hi * torch.sin(ang), hi * torch.cos(ang) + lo * torch.sin(ang)), -1)


def attention(pages, table, q, k, v, cu, lens, Hq, Hkv):
    """pages [n_blocks, Hkv, 2176] of one layer.  Returns out [T, Hq * 128] in float64 and a bound on the error that the
    header's numerics allow, element by element.

    Terms of the bound, beside half a bf16 step of the result (2^-8 |o|):
      - probabilities times s are halves: half a step, 2^-11, of p_j s_j c_j; suffix probabilities have two bf16
        terms, 2^-16;
      - scores are fp32: q c is a sum of 128 products, each exact (elements of q 2^-27 times the row's largest lose what is below 2^-38
        of it), so an error of 136 2^-24 sum |q| 15 s and two roundings of s acc + z sum q, which moves a probability by that times
        log(e) = the same relative to it; twice, for numerator and denominator; exp2 and the shift cost 2^-20 of p (scores up to
        2^6) more;
      - sums over n keys: added in steps of 32, wavefronts and pieces apart: (n / 32 + 64) 2^-24 of the absolute sum,
        in which s c and z count apart."""
    T, G = q.shape[0], Hq // Hkv
    out = torch.empty(T, Hq * HD, dtype=torch.float64, device=q.device)
    tol = torch.empty_like(out)
    for b in range(len(lens)):
        L, t0, S = int(lens[b]), int(cu[b]), int(cu[b + 1] - cu[b])
        ids = torch.as_tensor([min(max(int(x), 0), pages.shape[0] - 1) for x in table[b][:(L + 15) // 16]], dtype=torch.long, device=q.device)
        for h in range(Hkv):
            kc = ks = kz = None
            if L:
                (kc, ks, kz), (vc, vs, vz) = read_pages(pages[ids, h])
                ks, kz, vs, vz = (x.reshape(-1)[:L] for x in (ks, kz, vs, vz))
                K = kz[:, None] + ks[:, None] * kc.reshape(-1, HD)[:L]
                V = vz[:, None] + vs[:, None] * vc.reshape(-1, HD)[:L]
            else:
                K = V = torch.empty(0, HD, dtype=torch.float64, device=q.device)
                ks = kz = torch.empty(0, dtype=torch.float64, device=q.device)
            Ks, Vs = k[t0:t0 + S, h].double(), v[t0:t0 + S, h].double()
            Q = q[t0:t0 + S, h * G:(h + 1) * G].double().reshape(S * G, HD)
            s = Q @ torch.cat((K, Ks)).t() / math.sqrt(HD)
            last = (L + torch.arange(S, device=q.device)).repeat_interleave(G)[:, None]
            s = s.masked_fill(torch.arange(L + S, device=q.device)[None, :] > last, -math.inf)
            p = torch.softmax(s, -1)
            Vall = torch.cat((V, Vs))
            o = p @ Vall
            qa = Q.abs().sum(-1, keepdim=True)
            es = 2.0 ** -24 * qa * torch.cat((138 * (16 * ks + 2 * kz.abs()), 138 * Ks.abs().max(-1).values)) / math.sqrt(HD)
            es = torch.where(p > 0, es, torch.zeros_like(es))
            reach = torch.cat((V.abs(), Vs.abs()))
            apart = torch.cat((vz.abs()[:, None] + (V - vz[:, None]).abs(), Vs.abs())) if L else reach
            spread = (p * es) @ reach + (p * es).sum(-1, keepdim=True) * (p @ reach)
            rel = torch.cat((torch.full((L,), 2.0 ** -11, dtype=torch.float64, device=q.device), torch.full((S,), 2.0 ** -16, dtype=torch.float64, device=q.device)))
            sums = ((L + S) / 32 + 64) * 2.0 ** -24 * 6 + 2.0 ** -19
            w = 2.0 ** -8 * o.abs() + 1.01 * spread + (p * rel) @ torch.cat(((V - vz[:, None]).abs() if L else V, Vs.abs())) + sums * (p @ apart)
            out[t0:t0 + S, h * G * HD:(h + 1) * G * HD] = o.view(S, G * HD)
            tol[t0:t0 + S, h * G * HD:(h + 1) * G * HD] = w.view(S, G * HD)
    return out, tol


def w4_quantise_case(gen, N, K, group, dev, zeros=True):
    """Random codes [N, K / 2] (packed bytes), scales and zeros, and the weights they stand for in float64."""
    c = torch.randint(0, 16, (N, K), generator=gen, device=dev)
    s = ((torch.rand(N, K // group, generator=gen, device=dev) + 0.2) * (0.5 / math.sqrt(K))).half()
    z = torch.randint(0, 32, (N, K // group), generator=gen, device=dev).half() / 2 if zeros else None
    zd = z.double() if zeros else torch.full((N, K // group), 8.0, dtype=torch.float64, device=dev)
    w = (c.double() - zd.repeat_interleave(group, 1)) * s.double().repeat_interleave(group, 1)
    return (c[:, 0::2] | (c[:, 1::2] << 4)).to(torch.uint8).contiguous(), s, z, w


def w4_gemm(a, w, s, z, group):
    """A [M, K] . W [N, K]^T in float64, and a bound on the fp32 error: products of activations and codes (16 + c <= 31, less
    16 + z) are exact, and a result goes through at most group + K / group + 64 roundings, each 2^-24 of the absolute sum."""
    y = a.double() @ w.t()
    K = a.shape[1]
    zd = z.double().abs() if z is not None else torch.full(s.shape, 8.0, dtype=torch.float64, device=a.device)
    reach = a.double().abs() @ ((47 + zd) * s.double().abs()).repeat_interleave(group, 1).t()
    return y, (group + K / group + 64) * 2.0 ** -24 * reach


def swiglu(y, tol):
    """silu(gate) * up of [M, N] = gate | up, with the bound carried through: |silu'| < 1.1, half a bf16 step of the result,
    and 2^-20 for exp and the division."""
    F = y.shape[1] // 2
    g, u, tg, tu = y[:, :F], y[:, F:], tol[:, :F], tol[:, F:]
    act = g / (1.0 + torch.exp(-g))
    out = act * u
    return out, 2.0 ** -8 * out.abs() + 2.0 ** -20 * out.abs() + 1.1 * tg * (u.abs() + tu) + (act.abs() + 1.1 * tg) * tu + 2.0 ** -130
