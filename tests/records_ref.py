"""Plain 64-bit counterparts of the calls on 4-bit records, page accounts and eviction (include/unique.h), on the CPU."""
import math

import torch

LEVELS = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def tile_bytes(S, D):
    return S * D + 2 * S * (D // 32)


def encode(x):
    """[..., D] of any float type -> codes uint8 [..., D], scale bytes uint8 [..., D/32]: the nearest level by comparison with all
    of them, the even code where two are equally near."""
    x = x.double().unflatten(-1, (-1, 32))
    bad = ~torch.isfinite(x).all(-1, keepdim=True)
    x = torch.where(bad, torch.zeros((), dtype=torch.float64), x)
    top = x.abs().amax(-1, keepdim=True)
    e = torch.where(top > 0, torch.frexp(top)[1].double() - 3, torch.full_like(top, -126.0)).clamp(-126, 125)
    y = x.abs() / torch.pow(2.0, e)
    far = (y[..., None] - LEVELS).abs()
    order = torch.arange(8) % 2 + torch.arange(8) / 16  # even codes first
    code = torch.where(far == far.amin(-1, keepdim=True), order, torch.full((), 9.0, dtype=order.dtype)).argmin(-1)
    code = code + 8 * (x < 0)
    scale = torch.where(bad, torch.full_like(e, 255.0), e + 127)
    return code.flatten(-2).to(torch.uint8), scale.squeeze(-1).to(torch.uint8)


def values(code, scale):
    mag = LEVELS[(code & 7).long()] * (1 - 2 * (code >> 3).double())
    s = torch.where(scale == 255, torch.full((), math.nan, dtype=torch.float64), torch.pow(2.0, scale.double() - 127))
    return (mag.unflatten(-1, (-1, 32)) * s[..., None]).flatten(-2)


def k_byte(S, D, t, c):
    return t * (D // 2) + c // 2


def v_byte(S, D, t, c):
    unit = D // 16
    return S * D // 2 + ((t // 8 * 16 + c // unit) * 8 + t % 8) * (unit // 2) + c % unit // 2


def write_token(tile, S, D, t, kc, ks, vc, vs):
    """One token's codes [D] and scales [D/32] into a tile (uint8, one (page, head)), byte by byte."""
    for c in range(0, D, 2):
        tile[k_byte(S, D, t, c)] = int(kc[c]) | int(kc[c + 1]) << 4
        tile[v_byte(S, D, t, c)] = int(vc[c]) | int(vc[c + 1]) << 4
    for i in range(D // 32):
        tile[S * D + i * S + t] = int(ks[i])
        tile[S * D + (D // 32 + i) * S + t] = int(vs[i])


def tiles_of(k, v):
    """[n, S, D] keys and values -> tiles uint8 [n, bytes] with every slot written."""
    n, S, D = k.shape
    (kc, ks), (vc, vs) = encode(k), encode(v)
    out = torch.zeros((n, tile_bytes(S, D)), dtype=torch.uint8)
    t, c = torch.meshgrid(torch.arange(S), torch.arange(0, D, 2), indexing="ij")
    out[:, k_byte(S, D, t, c).reshape(-1)] = (kc[..., 0::2] | kc[..., 1::2] << 4).reshape(n, -1)
    out[:, v_byte(S, D, t, c).reshape(-1)] = (vc[..., 0::2] | vc[..., 1::2] << 4).reshape(n, -1)
    out[:, S * D:S * D + S * (D // 32)] = ks.transpose(1, 2).reshape(n, -1)
    out[:, S * D + S * (D // 32):] = vs.transpose(1, 2).reshape(n, -1)
    return out


def values_of(tiles, S, D):
    """The inverse: tiles [n, bytes] -> float64 keys and values [n, S, D]."""
    n = tiles.shape[0]
    t, c = torch.meshgrid(torch.arange(S), torch.arange(D), indexing="ij")
    got = []
    for at, base in ((k_byte(S, D, t, c), S * D), (v_byte(S, D, t, c), S * D + S * (D // 32))):
        code = (tiles[:, at.reshape(-1)] >> (c % 2 * 4).reshape(-1).to(torch.uint8)) & 15
        scale = tiles[:, base:base + S * (D // 32)].view(n, D // 32, S).transpose(1, 2)
        got.append(values(code.view(n, S, D), scale))
    return got


class Attended:
    """softmax(q k^T scale) v in 64 bits for one KV head's group, and what bounds a 32-bit evaluation of it."""

    def __init__(self, q, k, v, scale):
        """q [G, D], k and v [T, D] of the attended tokens."""
        q, k, v = q.double(), k.double(), v.double()
        self.T, D = k.shape
        G = q.shape[0]
        if self.T == 0:
            self.out, self.lse, self.p = torch.zeros((G, D), dtype=torch.float64), torch.full((G,), -math.inf, dtype=torch.float64), q.new_zeros((G, 0))
            self.mass, self.slack = torch.zeros_like(self.out), torch.zeros((G,), dtype=torch.float64)
            return
        x = q @ k.T * scale
        self.lse = torch.logsumexp(x, -1)
        self.p = torch.exp(x - self.lse[:, None])
        self.out = self.p @ v
        self.mass = self.p @ v.abs()  # sum of p |v|
        # A logit: D products added in fp32, one rounding of the product with scale * log2 e, an exponent of that size rounded once,
        # and the exponential itself. Twice, as the normaliser has the same errors.
        logit = (D + 4) * 2.0 ** -24 * (q.abs() @ k.abs().T).amax(-1) * scale + 2.0 ** -22 * (1 + x.abs().amax(-1))
        # Sums over the tokens: 16 or 32 at a time, the partial sums one after the other.
        self.slack = 2 * logit + 2 * (self.T / 16 + 64) * 2.0 ** -24

    def out_tolerance(self, dtype, part):
        """part: relative size of what the parts of a probability leave out."""
        return torch.finfo(dtype).eps / 2 * self.out.abs() * 1.01 + (self.slack[:, None] + part) * self.mass + 1e-30


def evict(table, lens, weights, S, budget, sinks, recent):
    """Lists of the results for each sequence: kept logical pages, freed physical ids, new length."""
    got = []
    for b, n in enumerate(lens.tolist()):
        P = -(-n // S)
        if P <= budget:
            got.append((list(range(P)), [], n))
            continue
        rank = weights[b, :, :P].double().sum(0).float().tolist()
        fixed = set(range(sinks)) | set(range(P - recent, P))
        rest = sorted((p for p in range(P) if p not in fixed), key=lambda p: (math.isnan(rank[p]), -rank[p] if not math.isnan(rank[p]) else 0, p))
        stay = fixed | set(rest[:budget - len(fixed)])
        keep, gone = sorted(stay), [p for p in range(P) if p not in stay]
        got.append((keep, table[b, gone].tolist(), n - len(gone) * S))
    return got
