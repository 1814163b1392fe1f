"""GPU tests of latent attention over the range of values: sizes that differ by orders of magnitude within a call, weights far below the largest,
infinities, scores beyond 2^24.  Every result against the definition in 64 bits."""
import pytest
import torch

from latent_side import HALF, TOLD, Batch, P, check, told

pytestmark = pytest.mark.gpu
KINDS = {"f32": (torch.float32, False), "bf16": (torch.bfloat16, False), "bf16_kv8": (torch.bfloat16, True)}


@pytest.fixture(scope="module")
def pa(gpu_device):
    from paper_2407_00023_amd import binding
    return binding


def bits(t):
    return t.view(torch.int32 if t.dtype == torch.float32 else torch.int16)


def part_of(b, pa, rows, r):
    """Request r of a batch of its own."""
    one = Batch(b.device, [b.prefix[r]], [b.ext[r]], b.H, b.R, b.dtype, b.kv8).weights(b.N)
    one.q, one.c, one.w_k, one.w_v, one.scale = b.q[rows].contiguous(), b.c[rows].contiguous(), b.w_k, b.w_v, b.scale
    one.slots, one.rows_pool, one.num_slots, one.kw = [b.slots[r]], b.rows_pool, b.num_slots, b.kw
    one.slot_idx = torch.cat([b.slots[r], torch.full((b.ext[r],), -1)]).int().to(b.device)
    return one.fill(pa)


# ---- sizes of values within a call ---------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kind", ["bf16", "bf16_kv8"])
@pytest.mark.parametrize("prefix,ext,H", [([300, 40], [90, 70], 3), ([4000], [5], 2)])
@pytest.mark.parametrize("of", [-6.5, -7, -8, -9, -10, -12])
def test_expanded_values_some_of_which_are_small(pa, gpu_device, kind, prefix, ext, H, of):
    b = Batch(gpu_device, prefix, ext, H, 512, *KINDS[kind], seed=3).fill(pa).weights(128)
    b.w_v = (b.w_v.float() * 2.0 ** of).to(b.dtype)
    check(b.expanded(pa), *b.reference("expanded"), f"2^{of}, {kind}")


@pytest.mark.parametrize("kind", ["bf16", "bf16_kv8"])
@pytest.mark.parametrize("of", [-20, -14, -12, -10, -9, -8, 8, 14])
@pytest.mark.parametrize("prefix,ext", [([1024, 1024], [3, 5]), ([100, 33], [40, 200])])
def test_expanded_requests_whose_rows_differ_in_size(pa, gpu_device, kind, of, prefix, ext):
    """The latent parts of request 1 are 2^of times those of request 0: each is held to what it would be by itself, and a call repeats its bits."""
    b = Batch(gpu_device, prefix, ext, 4, 512, *KINDS[kind], seed=4).weights(128)
    e0 = ext[0]
    at = b.slots[1].to(gpu_device)
    b.rows_pool[at, :512] = b.rows_pool[at, :512] * 2.0 ** of
    b.c[e0:, :512] = b.c[e0:, :512] * 2.0 ** of
    b.q[e0:, :, :128] = b.q[e0:, :, :128] * 2.0 ** -of
    b.fill(pa)
    ref, bound = b.reference("expanded")
    out = b.expanded(pa)
    check(out[:e0], ref[:e0], bound[:e0], f"request 0 beside 2^{of}, {kind}")
    check(out[e0:], ref[e0:], bound[e0:], f"request 1, 2^{of}, {kind}")
    for _ in range(3):
        assert torch.equal(bits(b.expanded(pa)), bits(out))
    for r, rows in ((0, slice(0, e0)), (1, slice(e0, None))):
        check(part_of(b, pa, rows, r).expanded(pa), ref[rows], bound[rows], f"request {r} alone")


@pytest.mark.parametrize("kind", ["bf16", "bf16_kv8"])
@pytest.mark.parametrize("of", [-20, 20])
def test_expanded_rows_that_differ_in_size_within_a_request(pa, gpu_device, kind, of):
    """Every third cached row is 2^of times the others; over 2,000 of them, so that tiles are cut."""
    b = Batch(gpu_device, [2000, 64], [3, 150], 3, 512, *KINDS[kind], seed=5).weights(128)
    b.rows_pool[::3, :512] = b.rows_pool[::3, :512] * 2.0 ** of
    b.c[1::3, :512] = b.c[1::3, :512] * 2.0 ** of
    b.w_k = b.w_k * 2.0 ** -max(of, 0)
    b.fill(pa)
    out = b.expanded(pa)
    check(out, *b.reference("expanded"), f"2^{of}, {kind}")
    assert torch.equal(bits(b.expanded(pa)), bits(out))


@pytest.mark.parametrize("kind", ["bf16", "bf16_kv8"])
@pytest.mark.parametrize("value", [1e30, 3e38, float("inf"), float("nan")])
def test_expanded_rows_of_no_request_may_hold_anything(pa, gpu_device, kind, value):
    """A batch padded to a fixed T, whose rows behind (before, between) the requests' are of any value."""
    b = Batch(gpu_device, [40, 33], [3, 4], 16, 512, *KINDS[kind], seed=5).fill(pa).weights(128)
    ref, bound = b.reference("expanded")
    alone = b.expanded(pa).clone()
    pad = lambda x: torch.cat([x[:2] * 0 + value, x[:3], x[:1] * 0 + value, x[3:7], x[:7] * 0 + value]).contiguous()
    b.q, b.c = pad(b.q), pad(b.c)
    b.ext_offsets = torch.tensor([2, 6, 17], dtype=torch.int32, device=gpu_device)
    out = torch.full((17, 16, 128), 9.0, dtype=b.dtype, device=gpu_device)
    b.expanded(pa, out=out)
    got = torch.cat([out[2:5], out[6:10]])
    check(got, ref, bound, f"{value}, {kind}")
    assert torch.equal(bits(got), bits(alone)) and bool((out[[0, 1, 5, 10, 16]] == 9.0).all())
