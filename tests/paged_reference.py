"""The paged cache's operators written out plainly on the CPU, in 64 bits (and, where the definition is in binary32
operations, in those): what tests/test_gpu_paged.py compares the kernels with.  Shares nothing with the library."""
import math

import torch

E4M3_VALUES = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).to(torch.float64)
EXPONENTS = {torch.float16: (-15, 7), torch.bfloat16: (-100, 118)}


def rotate(x, rope, pos, rot_dim, interleaved, dtype=torch.float32):
    """x [n, H, 128] rotated by pos [n]; every product and sum one operation of `dtype`."""
    y = x.to(dtype).clone()
    if rot_dim == 0:
        return y
    half = rot_dim // 2
    i = torch.arange(half)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    c, s = rope[pos][:, None, :half].to(dtype), rope[pos][:, None, half:].to(dtype)
    xa, xb = y[..., a].clone(), y[..., b].clone()
    y[..., a] = xa * c - xb * s
    y[..., b] = xb * c + xa * s
    return y


def encode(x):
    """float64 values to the nearest e4m3 code value (ties to even), beyond 448 to 448, NaN stays."""
    grid = E4M3_VALUES[:127]                                   # ascending, 0 .. 448
    mag = x.abs().clamp(max=448.0)
    hi = torch.searchsorted(grid, torch.nan_to_num(mag, nan=0.0).contiguous()).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    dl, dh = mag - grid[lo], grid[hi] - mag
    pick = torch.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    y = grid[pick] * torch.where(x < 0, -1.0, 1.0)
    return torch.where(torch.isnan(x), torch.full_like(x, math.nan), y)


def scale_for(x, dtype):
    """Smallest power of two s with |x| <= 448 s over the finite values, exponent within the model type's range."""
    m = x[torch.isfinite(x)].abs()
    top = float(m.max()) if m.numel() else 0.0
    if top == 0.0:
        return 0.0
    lo, hi = EXPONENTS[dtype]
    e = lo
    while e < hi and top > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


class Cache:
    """Pages as the definition has them: values (float64) and, for 8 bits, scales."""

    def __init__(self, k_pages, v_pages, k_scale, v_scale, dtype):
        self.dtype, self.q8 = dtype, k_scale is not None
        self.pool = [p.to(torch.float64) if not self.q8 else E4M3_VALUES[p.view(torch.uint8).long()].clone() for p in (k_pages, v_pages)]
        self.scale = [s.to(torch.float64).clone() if self.q8 else None for s in (k_scale, v_scale)]

    def values(self, which):
        return self.pool[which] * self.scale[which][..., None, None] if self.q8 else self.pool[which]

    def append(self, k, v, start, table, page_size):
        """k, v [m, Hkv, 128] float32 (k rotated) at positions start ...; returns the touched logical pages."""
        m, hkv = k.shape[0], k.shape[1]
        touched = sorted({(start + i) // page_size for i in range(m)})
        for p in touched:
            lo, hi = max(start, p * page_size), min(start + m, (p + 1) * page_size)
            a, z, page = lo - p * page_size, hi - p * page_size, int(table[p])
            for which, x in enumerate((k, v)):
                rows = x[lo - start: hi - start].transpose(0, 1)                   # [Hkv, n, 128]
                if not self.q8:
                    self.pool[which][page, :, a:z] = rows.to(self.dtype).to(torch.float64)
                    continue
                for h in range(hkv):
                    old = float(self.scale[which][page, h]) if a else 0.0
                    now = max(old, scale_for(rows[h], self.dtype))
                    if a and now > old:
                        self.pool[which][page, h, :a] = encode(self.pool[which][page, h, :a] * (old / now))
                    self.scale[which][page, h] = now
                    y = rows[h].to(torch.float64)
                    self.pool[which][page, h, a:z] = encode(y / now if now > 0 else torch.where(torch.isnan(y), y, y * 0.0))
        return touched


def attend(q, K, V, scale):
    """q [Hq, 128], K, V [Hkv, n, 128] float64 -> out, lse, and the largest scale * sum |q k| (for tolerances)."""
    hq, hkv = q.shape[0], K.shape[0]
    g = hq // hkv
    out, lse, reach = torch.zeros(hq, 128, dtype=torch.float64), torch.full((hq,), -math.inf, dtype=torch.float64), 0.0
    if K.shape[1] == 0:
        return out, lse, reach
    for h in range(hkv):
        z = (q[h * g: (h + 1) * g] @ K[h].T) * scale
        reach = max(reach, float((q[h * g: (h + 1) * g].abs() @ K[h].abs().T).max()) * abs(scale))
        m = z.amax(1, keepdim=True)
        p = torch.exp(z - m)
        out[h * g: (h + 1) * g] = (p @ V[h]) / p.sum(1, keepdim=True)
        lse[h * g: (h + 1) * g] = (m + p.sum(1, keepdim=True).log())[:, 0]
    return out, lse, reach
