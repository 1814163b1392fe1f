"""Batches of latent attention for the tests, and the operators' definition in 64 bits, on the CPU or the GPU, with the bound that
rounding allows.  Shares no code with the library."""
from __future__ import annotations

import pytest
import torch

P = 64
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}  # a rounding is off by at most this, relatively


def quantise(c):
    """Latent values [n, R] as the 8-bit pool holds them, in 64 bits: (values, exponents)."""
    x = c.double()
    top = x.abs().amax(1)
    k = torch.zeros_like(top)
    for _ in range(3):  # smallest k with top 2^-k <= 448: from log2 by single steps, so that its rounding does not matter
        guess = torch.where(top > 0, torch.floor(torch.log2(top.clamp(min=1e-300) / 448)), k) if _ == 0 else k
        k = torch.where((top > 0) & (top > 448 * torch.pow(2.0, guess)), guess + 1, guess)
    k = torch.where(top > 0, k.round().clamp(-100, 119), torch.zeros_like(k))
    two_k = torch.ldexp(torch.ones_like(k), k.int()).double() if not k.is_cuda else torch.ldexp(torch.ones_like(k).cpu(), k.int().cpu()).to(k.device)
    y = (x / two_k[:, None]).clamp(-448, 448)
    m, e = torch.frexp(y.abs().clamp(min=2.0 ** -6))
    step = torch.ldexp(torch.ones_like(m).cpu(), (e - 4).cpu()).to(y.device)
    return torch.round(y / step) * step * two_k[:, None], k.int()


# The absorbed form goes by tiles of 32, 64 or 128 rows, according to the rows and to how many keys it is told of at most: of 100,000, batches with enough
# rows take 64, of 10,000,000 as many as their rows fill.
TOLD = [0, 100_000, 10_000_000]
FORMS_TOLD = [("absorbed", x) for x in TOLD] + [("expanded", 0)]


@pytest.fixture
def told(request):
    Batch.told = request.param
    yield request.param
    Batch.told = 0


class Batch:
    """prefix, ext: lengths per request; share: requests whose cached rows are those of request share[r] as far as they go."""

    told = 0  # keys that the absorbed form is told of, if more than there are

    def __init__(self, device, prefix, ext, H, R, dtype=torch.bfloat16, kv8=False, seed=0, num_slots=None, share=None, spread=1.0, gap=0):
        g = torch.Generator().manual_seed(seed)
        self.prefix, self.ext, self.H, self.R, self.dtype, self.kv8, self.device = list(prefix), list(ext), H, R, dtype, kv8, device
        need = sum(prefix) + 1
        self.num_slots = num_slots or -(-need // 16) * 16
        order = torch.randperm(self.num_slots, generator=g)
        at, lists = 0, []
        for r, n in enumerate(prefix):
            if share and share[r] != r:
                lists.append(lists[share[r]][:n])
                assert len(lists[-1]) == n
            else:
                lists.append(order[at:at + n])
                at += n
        self.slots = lists
        self.T = sum(ext)
        self.rows_pool = (torch.randn(self.num_slots, R + P, generator=g) * spread).to(dtype).to(device)
        self.c = torch.randn(self.T, R + P, generator=g).to(dtype).to(device)
        self.q = torch.randn(self.T, H, R + P, generator=g).to(dtype).to(device)
        self.scale = (R + P) ** -0.5
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=device)
        self.slot_idx = torch.cat([torch.cat([s, torch.full((e + gap,), -1)]) for s, e in zip(lists, ext)]).int().to(device)
        starts = lambda x: i32([sum(x[:i]) for i in range(len(x) + 1)])
        self.offsets, self.ext_offsets = starts([p + e + gap for p, e in zip(prefix, ext)]), starts(list(ext))
        self.prefix_len, self.ext_len = i32(list(prefix)), i32(list(ext))
        self.max_kv_len = max([p + e for p, e in zip(prefix, ext)] or [0])
        self.kw = dict(num_slots=self.num_slots, kv8=kv8)

    def fill(self, pa):
        self.pool = torch.zeros(pa.latent_pool_bytes(self.num_slots, self.R, P, self.dtype, self.kv8), dtype=torch.uint8, device=self.device)
        pa.append_latent(self.pool, torch.arange(self.num_slots, dtype=torch.int32, device=self.device), self.rows_pool, rope_dim=P, **self.kw)
        return self

    def batch(self):
        return self.slot_idx, self.offsets, self.prefix_len, self.ext_len, self.ext_offsets, self.scale

    def absorbed(self, pa, **kw):
        kw.setdefault("max_kv_len", max(self.max_kv_len, Batch.told))
        return pa.latent_attention(self.q, self.c, self.pool, *self.batch(), rope_dim=P, **self.kw, **kw)

    def weights(self, N, seed=1, std=1.0):
        g = torch.Generator().manual_seed(seed)
        self.N = N
        mk = lambda: (torch.randn(self.H, N, self.R, generator=g) * std * self.R ** -0.5).to(self.dtype).to(self.device)
        self.w_k, self.w_v = mk(), mk()
        self.q = torch.randn(self.T, self.H, N + P, generator=g).to(self.dtype).to(self.device)
        self.scale = (N + P) ** -0.5
        return self

    def expanded(self, pa, **kw):
        kw.setdefault("max_kv_len", self.max_kv_len)
        return pa.latent_attention_expanded(self.q, self.c, self.w_k, self.w_v, self.pool, *self.batch(), **self.kw, **kw)

    def stored(self):
        if not self.kv8:
            return self.rows_pool.double()
        return torch.cat([quantise(self.rows_pool[:, :self.R])[0], self.rows_pool[:, self.R:].double()], 1)

    def reference(self, form="absorbed", stored=None):
        """-> (out, bound) in 64 bits, [T, H, width].

        The bound: the result is rounded once (h |out|, h = half a step of the type).  In 16 bits the probabilities are rounded
        before the second product (h sum p |v|).  Scores are fp32 sums of n products: off by at most (n + 2) 2^-24 times the sum
        of the products' magnitudes; a probability is off by twice that (its own and the maximum's or the sum's) relatively, and
        by 2^-20 for the exponential (its argument, of magnitude up to 2^7, in fp32, and 2 units of the function).  Sums over K
        keys: K 2^-24 sum p |v|.  Expanded form: keys and values are rounded once more, to 2^-11 of the largest of a block of
        them at worst 2^-21 below its top (a value): h16 on each |k| inside a score, and on each |v|; a probability in fp16 is off by
        2^-25 where that is more (their largest is 1 at least)."""
        dt, h = self.dtype, HALF[self.dtype]
        rows = self.stored() if stored is None else stored
        outs, bounds, t = [], [], 0
        for r, (n, e) in enumerate(zip(self.prefix, self.ext)):
            if e == 0:
                continue
            keys = torch.cat([rows[self.slots[r].to(rows.device)], self.c[t:t + e].double()])
            q = self.q[t:t + e].double()
            hidden = torch.arange(n + e, device=q.device)[None] > n + torch.arange(e, device=q.device)[:, None]
            o_r, b_r = [], []
            for x in range(self.H):
                lat, rope = keys[:, :self.R], keys[:, self.R:]
                h16 = 0.0
                if form == "absorbed":
                    k, v, width = keys, lat, self.R + P
                    mag_k, mag_v = k.abs(), v.abs()
                else:
                    wk, wv = self.w_k[x].double(), self.w_v[x].double()
                    k, v, width = torch.cat([lat @ wk.T, rope], 1), lat @ wv.T, self.N + P
                    mag_k, mag_v = k.abs(), v.abs()
                    sums = (self.R + 2) * 2.0 ** -24                 # fp32 sums of the expansion
                    grow_k, grow_v = torch.cat([lat.abs() @ wk.abs().T, torch.zeros_like(rope)], 1) * sums, lat.abs() @ wv.abs().T * sums
                    if dt != torch.float32:
                        h16 = HALF[torch.float16]
                        top_k, top_v = k[:, :self.N].abs().max(), v.abs().max()
                        grow_k[:, :self.N] += h16 * mag_k[:, :self.N] + 2.0 ** -21 * top_k
                        grow_v += h16 * mag_v + 2.0 ** -21 * top_v
                    else:  # through the latent form: sums over R and over N
                        grow_k[:, :self.N] += (self.N + 2) * 2.0 ** -24 * (lat.abs() @ wk.abs().T)
                z = (q[:, x] @ k.T * self.scale).masked_fill(hidden, -torch.inf)
                p = torch.softmax(z, 1)
                out = p @ v
                a = p @ mag_v
                dz = (width + 2) * 2.0 ** -24 * (q[:, x].abs() @ mag_k.T) * self.scale
                if form != "absorbed":
                    dz = dz + self.scale * (q[:, x].abs() @ grow_k.T)
                dz = dz.masked_fill(hidden, 0).amax(1, keepdim=True)
                hp = 0.0 if dt == torch.float32 else (h if form == "absorbed" else h16)
                b = a * (2 * dz + 2.0 ** -20 + (n + e + 64) * 2.0 ** -24 + hp) + h * out.abs() + 1e-30
                if form != "absorbed":
                    b = b + p @ grow_v * (1 + h)
                    if h16:
                        b = b + 2.0 ** -25 * (~hidden).double() @ mag_v
                o_r.append(out)
                b_r.append(b)
            outs.append(torch.stack(o_r, 1))
            bounds.append(torch.stack(b_r, 1))
            t += e
        return torch.cat(outs), torch.cat(bounds)


def check(out, ref, bound, what=""):
    d = (out.double() - ref).abs()
    worst = float((d / bound).max())
    print(f"  {what} max abs {float(d.max()):.3e}, {worst:.3f} of the bound, rel {float(d.norm() / ref.norm()):.2e}", flush=True)
    assert out.dtype != torch.float64 and worst <= 1.0, (what, worst)
