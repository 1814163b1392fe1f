"""GPU tests of latent attention: the pool's rows bit for bit, both forms of the attention against their definition in 64 bits within
the bound that rounding allows (latent_side.py derives it)."""
import threading

import pytest
import torch

from latent_side import FORMS_TOLD, TOLD, Batch, P, check, quantise, told

pytestmark = pytest.mark.gpu
KINDS = {"f32": (torch.float32, False), "bf16": (torch.bfloat16, False), "bf16_kv8": (torch.bfloat16, True)}


@pytest.fixture(scope="module")
def pa(gpu_device):
    from paper_2407_00023_amd import binding
    return binding


def bits(t):
    return t.view(torch.int32 if t.dtype == torch.float32 else torch.int16)


# ---- the pool ---------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("R", [256, 512])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n", [1, 3, 4, 5, 63, 1000, 20001])
def test_rows_stored_and_read_back(pa, gpu_device, kind, n, R):
    dt, kv8 = KINDS[kind]
    g = torch.Generator().manual_seed(n)
    num_slots = n + 5
    rows = (torch.randn(n, R + P, generator=g) * 2.0 ** torch.randint(-20, 20, (n, 1), generator=g)).to(dt)
    rows[n // 2, :R] = 0
    slots = torch.randperm(num_slots, generator=g)[:n]
    bad = torch.tensor([num_slots, -1, 2 ** 31 - 1])                       # slots outside the pool: skipped
    kw = dict(rope_dim=P, num_slots=num_slots, kv8=kv8)
    pool = torch.zeros(pa.latent_pool_bytes(num_slots, R, P, dt, kv8), dtype=torch.uint8, device=gpu_device)
    pa.append_latent(pool, torch.cat([slots, bad]).int().to(gpu_device), torch.cat([rows, torch.ones(3, R + P, dtype=dt)]).to(gpu_device), **kw)
    every = torch.cat([torch.arange(num_slots), bad, torch.arange(num_slots).flip(0)]).int().to(gpu_device)  # (slots may repeat)
    mark = torch.full((len(every), R + P), 7.0, dtype=dt, device=gpu_device)
    got = pa.gather_latent(pool, every, latent_dim=R, dtype=dt, out=mark, **kw)
    assert got is mark
    want = torch.zeros(num_slots, R + P, dtype=dt)
    want[slots] = torch.cat([quantise(rows[:, :R])[0].to(dt), rows[:, R:]], 1) if kv8 else rows
    left = torch.full((3, R + P), 7.0, dtype=dt)
    want = torch.cat([want, left, want.flip(0)])
    assert torch.equal(got.cpu(), want)                                     # (equal: -0 and 0 are not told apart)
    if not kv8:
        assert torch.equal(bits(got.cpu()), bits(want))


def test_every_bf16_value_through_the_8_bit_pool(pa, gpu_device):
    """All finite bf16 bit patterns, under row maxima of several magnitudes."""
    every = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    every = every[torch.isfinite(every)]
    order = torch.argsort(every.abs().float(), stable=True)
    v = every[order]
    v = torch.cat([v, v[-(-len(v) % 512):]])[:len(v) // 512 * 512].view(-1, 512)
    rows = torch.cat([v, v.roll(17, 0), v.flip(0) * 0 + v[:, :1]])
    rows = torch.cat([rows, torch.zeros(len(rows), P, dtype=torch.bfloat16)], 1)
    n = len(rows)
    pool = torch.zeros(pa.latent_pool_bytes(n, 512, P, torch.bfloat16, True), dtype=torch.uint8, device=gpu_device)
    at = torch.arange(n, dtype=torch.int32, device=gpu_device)
    kw = dict(rope_dim=P, num_slots=n, kv8=True)
    pa.append_latent(pool, at, rows.to(gpu_device), **kw)
    got = pa.gather_latent(pool, at, latent_dim=512, dtype=torch.bfloat16, **kw).cpu()
    want = quantise(rows[:, :512])[0]
    # (bf16 subnormals count as zero: far below half the smallest code at every exponent allowed)
    assert torch.equal(got[:, :512].double(), want)


# ---- attention --------------------------------------------------------------------------------------------------------------

SHAPES = {  # name: prefix lengths, extend lengths, heads
    "one token, nothing cached": ([0], [1], 16),
    "one token, one cached": ([1], [1], 1),
    "decode, ragged": ([31, 32, 33, 700, 0, 64, 1], [1] * 7, 16),
    "decode, 128 heads": ([100, 1000, 5], [1, 1, 1], 128),
    "decode, long": ([5003, 40], [1, 1], 16),
    "decode, odd heads": ([90, 200], [1, 1], 5),
    "few rows, ragged": ([31, 95, 0, 640], [2, 1, 7, 3], 20),
    "extend, 128 heads": ([64, 0, 97], [3, 5, 2], 128),
    "extend, few heads": ([300, 0, 31, 7], [40, 90, 33, 1], 4),
    "requests without extend tokens": ([50, 60, 0, 70, 5], [0, 9, 0, 1, 0], 16),
    "long extend": ([513], [200], 8),
    "heads beyond a tile": ([70], [2], 150),
}


@pytest.mark.parametrize("told", TOLD, indirect=True)
@pytest.mark.parametrize("R", [512, 256])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("name", SHAPES)
def test_absorbed(pa, gpu_device, name, kind, R, told):
    dt, kv8 = KINDS[kind]
    prefix, ext, H = SHAPES[name]
    b = Batch(gpu_device, prefix, ext, H, R, dt, kv8, seed=len(name)).fill(pa)
    check(b.absorbed(pa), *b.reference(), f"{name}, {kind}, R {R}")


@pytest.mark.parametrize("N,R", [(128, 512), (64, 512), (128, 256)])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("name", SHAPES)
def test_expanded(pa, gpu_device, name, kind, N, R):
    dt, kv8 = KINDS[kind]
    prefix, ext, H = SHAPES[name]
    b = Batch(gpu_device, prefix, ext, H, R, dt, kv8, seed=len(name)).fill(pa).weights(N)
    check(b.expanded(pa), *b.reference("expanded"), f"{name}, {kind}, N {N}, R {R}")


@pytest.mark.parametrize("form", ["absorbed", "expanded"])
def test_the_two_forms_are_one(pa, gpu_device, form):
    """q W_k absorbed, W_v applied to the output: the forms agree, each within its own bound of the same 64-bit result (fp32)."""
    b = Batch(gpu_device, [200, 17], [5, 30], 4, 512, torch.float32, seed=3).fill(pa).weights(128)
    ref, bound = b.reference("expanded")
    if form == "expanded":
        check(b.expanded(pa), ref, bound)
    else:
        q = torch.cat([torch.matmul(b.q[:, :, None, :128].double(), b.w_k.double()[None]).squeeze(2), b.q[:, :, 128:].double()], 2).float()
        b.q, out_w = q, b.w_v
        out = torch.matmul(b.absorbed(pa).double()[:, :, None], out_w.double().transpose(1, 2)[None]).squeeze(2).float()
        check(out, ref, bound + 1e-4 * ref.abs().amax())  # (the queries are rounded to fp32 between the two)


@pytest.mark.parametrize("form,told", FORMS_TOLD, indirect=["told"])
@pytest.mark.parametrize("kind", KINDS)
def test_rows_of_no_request_are_left_alone(pa, gpu_device, kind, form, told):
    """Rows before the first request's, between two requests' and behind the last one's stay as they were."""
    dt, kv8 = KINDS[kind]
    b = Batch(gpu_device, [40, 33], [3, 4], 16, 512, dt, kv8, seed=5).fill(pa)
    if form == "expanded":
        b.weights(128)
    ref, bound = b.reference(form)
    pad = lambda x: torch.cat([x[:2] * 0 + 1, x[:3], x[:1] * 0 + 1, x[3:7], x[:2] * 0 + 1]).contiguous()
    b.q, b.c = pad(b.q), pad(b.c)
    b.ext_offsets = torch.tensor([2, 6, 12], dtype=torch.int32, device=gpu_device)
    out = torch.full((12, 16, ref.shape[2]), 9.0, dtype=dt, device=gpu_device)
    (b.absorbed if form == "absorbed" else b.expanded)(pa, out=out)
    check(torch.cat([out[2:5], out[6:10]]), ref, bound)
    assert bool((out[[0, 1, 5, 10, 11]] == 9.0).all())


@pytest.mark.parametrize("form,told", FORMS_TOLD, indirect=["told"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("H", [2, 16, 128])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_what_a_row_does_not_see_does_not_reach_it(pa, gpu_device, kind, H, value, form, told):
    """A later extend token holds an infinity or NaN: rows before it are what they are without it; so is a request beside it, whose
    cached rows end inside a tile."""
    dt, kv8 = KINDS[kind]
    b = Batch(gpu_device, [45, 10], [40, 3], H, 512, dt, kv8, seed=6).fill(pa)
    if form == "expanded":
        b.weights(128)
    call = lambda: (b.absorbed if form == "absorbed" else b.expanded)(pa)
    ref, bound = b.reference(form)
    b.c[21, 3] = value
    b.c[21, 400] = -value
    b.c[39, 511] = value
    out = call()
    keep = [i for i in range(43) if i < 21 or i >= 40]
    check(out[keep], ref[keep], bound[keep], f"H {H}")
    assert not bool(torch.isfinite(out[21:40].float()).all(-1).any())


@pytest.mark.parametrize("told", TOLD, indirect=True)
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("H", [4, 128])
def test_an_infinity_in_a_cached_row(pa, gpu_device, kind, H, told):
    """An infinite latent value in the last cached row, with queries that do not look at its place: infinity in its column, for every
    row, and the other columns as ever."""
    dt, kv8 = KINDS[kind]
    b = Batch(gpu_device, [67], [2], H, 512, dt, kv8, seed=8)
    b.q[..., 300] = 0
    b.rows_pool[:, 300] = 0
    b.c[:, 300] = 0
    b.fill(pa)
    ref, bound = b.reference()
    at = int(b.slots[0][-1])
    b.rows_pool[at, 300] = 3e38                                   # (finite, so that 0 times it is 0)
    b.fill(pa)
    out = b.absorbed(pa)
    keep = [d for d in range(512) if d != 300]
    check(out[..., keep], ref[..., keep], bound[..., keep])
    assert bool((out[..., 300] > 1e30).all())


@pytest.mark.parametrize("told", TOLD, indirect=True)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("H", [16, 128])
@pytest.mark.parametrize("order", ["rising", "falling", "jump"])
def test_scores_that_outgrow_the_running_maximum(pa, gpu_device, kind, H, order, told):
    dt, kv8 = KINDS[kind]
    b = Batch(gpu_device, [400], [3], H, 512, dt, kv8, seed=9)
    factor = {"rising": torch.linspace(0, 12, 400), "falling": torch.linspace(12, 0, 400), "jump": (torch.arange(400) // 150).float() * 6}[order]
    direction = torch.randn(512 + P, generator=torch.Generator().manual_seed(1))
    at = b.slots[0].to(gpu_device)
    b.rows_pool[at] = (b.rows_pool[at].float() * 0.3 + (factor[:, None] * direction[None]).to(gpu_device)).to(dt)
    b.q = (b.q.float() * 0.2 + direction.to(gpu_device)).to(dt)
    b.fill(pa)
    check(b.absorbed(pa), *b.reference(), f"{order} H {H}")


@pytest.mark.parametrize("form,told", FORMS_TOLD, indirect=["told"])
@pytest.mark.parametrize("kind", KINDS)
def test_requests_that_share_cached_rows(pa, gpu_device, kind, form, told):
    dt, kv8 = KINDS[kind]
    b = Batch(gpu_device, [300, 300, 200, 50, 300], [4, 1, 33, 2, 1], 16, 512, dt, kv8, seed=10, share=[0, 0, 0, 3, 0], gap=3).fill(pa)
    if form == "expanded":
        b.weights(128)
    check((b.absorbed if form == "absorbed" else b.expanded)(pa), *b.reference(form))


@pytest.mark.parametrize("form,told", FORMS_TOLD, indirect=["told"])
@pytest.mark.parametrize("kind", KINDS)
def test_slots_outside_the_pool_are_clamped(pa, gpu_device, kind, form, told):
    """No fault, and requests beside the one with bad slots are what they are."""
    dt, kv8 = KINDS[kind]
    b = Batch(gpu_device, [70, 64], [2, 3], 16, 512, dt, kv8, seed=11).fill(pa)
    if form == "expanded":
        b.weights(128)
    ref, bound = b.reference(form)
    b.slot_idx[3] = -5
    b.slot_idx[40] = b.num_slots
    b.slot_idx[41] = 2 ** 31 - 1
    out = (b.absorbed if form == "absorbed" else b.expanded)(pa)
    check(out[2:], ref[2:], bound[2:])


def test_calls_refuse_mismatched_tensors(pa, gpu_device):
    b = Batch(gpu_device, [10], [2], 4, 512).fill(pa).weights(128)
    b8 = Batch(gpu_device, [10], [2], 4, 512)
    ok = dict(rope_dim=P, max_kv_len=12, **b.kw)
    args = [b8.q, b.c, b.pool, *b.batch()]
    pa.latent_attention(*args, **ok)

    def refused(error, i=None, x=None, **over):
        a = list(args)
        if i is not None:
            a[i] = x
        with pytest.raises(error):
            pa.latent_attention(*a, **{**ok, **over})

    refused(TypeError, 0, b8.q.float())
    refused(TypeError, 0, b8.q.half())
    refused(TypeError, 0, b8.q.transpose(0, 1))
    refused(TypeError, 1, b.c.cpu())
    refused(TypeError, 3, b.slot_idx.long())
    refused(TypeError, 2, b.pool.cpu())
    refused(ValueError, 1, b.c[:1])
    refused(ValueError, 0, b8.q[:, :, :100].contiguous())
    refused(ValueError, 2, b.pool[:-1].contiguous())
    refused(ValueError, 4, b.offsets[:1])
    refused(ValueError, 6, b.ext_len[:0])
    refused(TypeError, 8, "scale")
    refused(pa.PrefixAttnError, 8, -1.0)
    refused(pa.PrefixAttnError, 8, float("nan"))
    refused(ValueError, rope_dim=32)
    refused(ValueError, num_slots=b.num_slots + 1)
    refused(ValueError, out=torch.empty(2, 4, 576, dtype=torch.bfloat16, device=gpu_device))
    refused(TypeError, max_kv_len=None)
    refused(TypeError, rope_dim=None)
    refused(TypeError, num_slots="16")
    refused(TypeError, kv8=True, x=b8.q.float(), i=0)
    refused(pa.PrefixAttnError, workspace=torch.empty(0, dtype=torch.uint8, device=gpu_device))
    with pytest.raises(ValueError):
        pa.latent_attention_expanded(b.q, b.c, b.w_k, b.w_v[:, :64].contiguous(), b.pool, *b.batch(), max_kv_len=12, **b.kw)
    with pytest.raises(ValueError):
        pa.latent_attention_expanded(b.q, b.c, b.w_k[:3].contiguous(), b.w_v[:3].contiguous(), b.pool, *b.batch(), max_kv_len=12, **b.kw)
    with pytest.raises(ValueError):
        pa.append_latent(b.pool, b.slot_idx[:1], b.c, rope_dim=P, num_slots=b.num_slots)
    with pytest.raises(TypeError):
        pa.gather_latent(b.pool, b.slot_idx, latent_dim=512, rope_dim=P, dtype="bf16", num_slots=b.num_slots)
