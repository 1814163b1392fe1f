"""Latent attention on the host: sizes, refusals, the stored format's statement.  No kernel is launched here."""
import ctypes as C

import pytest
import torch

from latent_side import quantise


@pytest.fixture(scope="module")
def pa():
    from paper_2407_00023_amd import binding
    return binding


def test_sizes(pa):
    assert pa.latent_pool_bytes(100, 512, 64, torch.bfloat16) == 100 * 1152
    assert pa.latent_pool_bytes(100, 256, 64, torch.float32) == 100 * 1280
    assert pa.latent_pool_bytes(100, 512, 64, torch.bfloat16, kv8=True) == 100 * 641
    for bad in [(0, 512, 64), (1 << 31, 512, 64), (16, 384, 64), (16, 512, 32), (16, 0, 64), (-1, 512, 64)]:
        with pytest.raises(ValueError):
            pa.latent_pool_bytes(*bad, torch.bfloat16)
    with pytest.raises(TypeError):
        pa.latent_pool_bytes(16, 512, 64, torch.float32, kv8=True)
    sizes = [pa.latent_workspace_bytes(4, t, 1000, 16, 512, 64, torch.bfloat16) for t in (1, 10, 100, 1000)]
    assert sizes == sorted(sizes) and sizes[0] > 0
    for bad in [(-1, 4, 10, 16, 512, 64), (65537, 4, 10, 16, 512, 64), (1, -1, 10, 16, 512, 64), (1, 1 << 31, 10, 16, 512, 64),
                (1, 4, -1, 16, 512, 64), (1, 4, 1 << 31, 16, 512, 64), (1, 4, 10, 0, 512, 64), (1, 4, 10, 16, 500, 64), (1, 4, 10, 16, 512, 128)]:
        with pytest.raises(ValueError):
            pa.latent_workspace_bytes(*bad, torch.bfloat16)
        with pytest.raises(ValueError):
            pa.latent_expanded_workspace_bytes(*bad, 128, 4096, torch.bfloat16)
    for N, slots in [(32, 100), (0, 100), (256, 100), (128, 0), (128, 1 << 31)]:
        with pytest.raises(ValueError):
            pa.latent_expanded_workspace_bytes(1, 4, 10, 16, 512, 64, N, slots, torch.bfloat16)


# (a pointer the host never follows: every call below is refused, or has nothing to do, before a kernel could be launched)
NOWHERE = 1 << 20


def attention(pa, **over):
    a = dict(q=NOWHERE, c=2 * NOWHERE, pool=3 * NOWHERE, slots=4 * NOWHERE, so=5 * NOWHERE, pl=6 * NOWHERE, el=7 * NOWHERE, eo=8 * NOWHERE,
             B=1, T=1, mk=10, H=16, R=512, P=64, N=128, wk=9 * NOWHERE, wv=10 * NOWHERE, ns=16, dt=1, scale=0.1, out=11 * NOWHERE,
             ws=12 * NOWHERE, nws=0, expanded=False)
    a.update(over)
    p = C.c_void_p
    head = [p(a["q"]), p(a["c"])] + ([p(a["wk"]), p(a["wv"])] if a["expanded"] else [])
    mid = [p(a[k]) for k in ("pool", "slots", "so", "pl", "el", "eo")] + [a[k] for k in ("B", "T", "mk", "H", "R", "P")]
    tail = ([a["N"]] if a["expanded"] else []) + [a["ns"], a["dt"], a["scale"], p(a["out"]), p(a["ws"]), a["nws"], None]
    rc = getattr(pa._lib, "pa_latent_attention_expanded" if a["expanded"] else "pa_latent_attention")(*head, *mid, *tail)
    return rc, pa._lib.pa_last_error().decode()


@pytest.mark.parametrize("expanded", [False, True])
def test_refusals(pa, expanded):
    ok = dict(expanded=expanded)
    assert attention(pa, B=0, **ok)[0] == 0 and attention(pa, T=0, **ok)[0] == 0        # nothing to do: no pointer is looked at
    assert attention(pa, B=0, q=0, out=0, ws=0, **ok)[0] == 0
    rc, text = attention(pa, nws=0, **ok)
    assert rc == -2 and "needed" in text
    assert attention(pa, ws=0, nws=1 << 40, **ok)[0] == -2
    for bad in [dict(dt=3), dict(dt=-1), dict(H=0), dict(H=-1), dict(R=128), dict(P=32), dict(B=-1), dict(T=-1), dict(mk=-1), dict(B=65537),
                dict(T=1 << 31), dict(mk=1 << 31), dict(ns=0), dict(ns=1 << 31), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")),
                dict(scale=float("nan")), dict(q=0), dict(c=0), dict(pool=0), dict(so=0), dict(pl=0), dict(el=0), dict(eo=0), dict(out=0),
                dict(q=NOWHERE + 8), dict(c=NOWHERE + 4), dict(pool=NOWHERE + 2), dict(out=NOWHERE + 8), dict(out=NOWHERE), dict(out=2 * NOWHERE),
                dict(ws=NOWHERE + 16, nws=1 << 50)]:
        rc, text = attention(pa, **{**dict(nws=1 << 50), **ok, **bad})
        assert rc == -1 and text.startswith("pa_latent_attention"), (bad, rc, text)
    if expanded:
        for bad in [dict(N=32), dict(N=0), dict(wk=0), dict(wv=0), dict(wk=NOWHERE + 8), dict(out=9 * NOWHERE), dict(out=10 * NOWHERE)]:
            rc, text = attention(pa, **{**dict(nws=1 << 50), **ok, **bad})
            assert rc == -1 and text.startswith("pa_latent_attention_expanded"), (bad, rc, text)


@pytest.mark.parametrize("fn", ["pa_append_latent", "pa_gather_latent"])
def test_pool_refusals(pa, fn):
    p = C.c_void_p

    def call(pool=NOWHERE, slots=2 * NOWHERE, rows=3 * NOWHERE, n=1, R=512, P=64, ns=16, dt=1):
        order = [p(pool), p(slots)] + ([p(rows), n, R, P, ns, dt] if fn == "pa_append_latent" else [n, R, P, ns, dt, p(rows)])
        return getattr(pa._lib, fn)(*order, None)

    assert call(n=0) == 0 and call(n=0, pool=0, rows=0, slots=0) == 0
    for bad in [dict(n=-1), dict(n=1 << 31), dict(R=128), dict(P=0), dict(ns=0), dict(ns=1 << 31), dict(dt=3), dict(pool=0), dict(slots=0),
                dict(rows=0), dict(pool=NOWHERE + 8), dict(rows=NOWHERE + 8)]:
        assert call(**bad) == -1, bad
        assert pa._lib.pa_last_error().decode().startswith(fn)


def test_calls_refuse_what_is_no_device_tensor(pa):
    x = torch.zeros(4, 576, dtype=torch.bfloat16)
    i = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(TypeError):
        pa.append_latent(x, i, x, rope_dim=64, num_slots=4)
    with pytest.raises(TypeError):
        pa.gather_latent(x, i, latent_dim=512, rope_dim=64, dtype=torch.bfloat16, num_slots=4)
    with pytest.raises(TypeError):
        pa.latent_attention(x, x, x, i, i, i, i, i, 1.0, rope_dim=64, num_slots=4, max_kv_len=4)
    with pytest.raises(TypeError):
        pa.latent_attention_expanded(x, x, x, x, x, i, i, i, i, i, 1.0, num_slots=4, max_kv_len=4)
    with pytest.raises(TypeError):
        pa.latent_attention(x, x, None, i, i, i, i, i, 1.0, rope_dim=64, num_slots=4, max_kv_len=4)
    with pytest.raises(TypeError):
        pa.append_latent(x, i, "rows", rope_dim=64, num_slots=4)


def test_the_stored_format_against_a_search_over_all_codes():
    """quantise() against the nearest of all 127 magnitudes, ties to the even code."""
    g = torch.Generator().manual_seed(0)
    x = torch.cat([torch.randn(40, 64, generator=g) * 2.0 ** torch.randint(-30, 30, (40, 1), generator=g), torch.zeros(1, 64)]).bfloat16()
    x[3, 5], x[4] = 0, torch.arange(64).bfloat16() * 7
    table = torch.tensor([(c & 7) * 2.0 ** -9 if c < 8 else (1 + (c & 7) / 8) * 2.0 ** ((c >> 3) - 7) for c in range(127)], dtype=torch.float64)
    got, k = quantise(x)
    for row, want_k, values in zip(x.double(), k.tolist(), got):
        top = float(row.abs().max())
        if top == 0:
            assert want_k == 0 and not values.any()
            continue
        assert top <= 448 * 2.0 ** want_k and top > 448 * 2.0 ** (want_k - 1)
        y = row.abs() / 2.0 ** want_k
        d = (y[:, None] - table[None]).abs()
        best = d.amin(1, keepdim=True)
        code = torch.where(d == best, torch.arange(127)[None] % 2 * 1000 + torch.arange(127)[None], torch.tensor(10 ** 6)).amin(1) % 1000
        assert torch.equal(values, table[code] * 2.0 ** want_k * torch.sign(row).double())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_empty_batches_have_a_workspace_size(pa, dtype):
    """(0 would mean that the arguments are invalid.)  In a process of its own, which a fault on the host would end."""
    import subprocess
    import sys
    code = ("import torch\nfrom paper_2407_00023_amd import binding as pa\n"
            "for B, T, most in [(0, 0, 0), (0, 0, 100), (1, 0, 0), (3, 0, 10), (0, 5, 0)]:\n"
            f"    assert pa.latent_workspace_bytes(B, T, most, 16, 512, 64, {dtype}) > 0\n"
            f"    assert pa.latent_expanded_workspace_bytes(B, T, most, 16, 512, 64, 128, 4096, {dtype}) > 0")
    run = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True)
    assert run.returncode == 0, run.stderr[-300:]


@pytest.mark.parametrize("form", ["absorbed", "expanded"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("H,R,N", [(1, 256, 64), (16, 512, 128), (32, 512, 128), (128, 512, 128), (130, 256, 64)])
def test_a_workspace_is_enough_for_smaller_batches(pa, form, dtype, H, R, N):
    """Sizes do not fall when B, T or max_kv_len rises, across the places where the expanded form holds fewer heads at once."""
    def size(B, T, most):
        if form == "absorbed":
            return pa.latent_workspace_bytes(B, T, most, H, R, 64, dtype)
        return pa.latent_expanded_workspace_bytes(B, T, most, H, R, 64, N, 1 << 20, dtype)

    of_T = [0, 1, 2, 3, 31, 32, 33, 64, 65, 500, 512, 2048, 2112, 5000, 8192, 30000, 60000]
    of_most = [1, 31, 32, 100, 1000, 2000, 4000, 7800, 8100, 8200, 16000, 16500, 33000, 65000, 70000, 131072, 260096]
    for B in [1, 2, 3, 8, 100]:
        sizes = [[size(B, T, most) for most in of_most] for T in of_T]
        for row, below in zip(sizes, sizes[1:] + [None]):
            assert row == sorted(row), (B, row)
            if below:
                assert all(x <= y for x, y in zip(row, below)), (B, row, below)
    for T in of_T:
        for most in of_most:
            sizes = [size(B, T, most) for B in [0, 1, 2, 3, 4, 7, 8, 9, 16, 17, 100, 1000]]
            assert sizes == sorted(sizes), (T, most, sizes)


def test_the_absorbed_forms_workspace_goes_by_its_tiles(pa):
    """Partial results of 256 workgroups, three tiles each, of 32 rows where a call has no more, of 128 at most."""
    size = lambda T, most, H: pa.latent_workspace_bytes(1, T, most, H, 512, 64, torch.bfloat16) / (3 * 256 * 512 * 4)
    assert 32 <= size(1, 2133, 16) < 33 and 32 <= size(2, 10 ** 6, 16) < 33
    assert 64 <= size(4, 10 ** 6, 16) < 65 and 128 <= size(128, 7800, 128) < 129
