"""GPU tests of the latent calls' arguments: empty batches, workspaces."""
import pytest
import torch

from latent_side import Batch, P, check

pytestmark = pytest.mark.gpu
KINDS = {"f32": (torch.float32, False), "bf16": (torch.bfloat16, False), "bf16_kv8": (torch.bfloat16, True)}


@pytest.fixture(scope="module")
def pa(gpu_device):
    from paper_2407_00023_amd import binding
    return binding


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("form", ["absorbed", "expanded"])
@pytest.mark.parametrize("prefix,ext", [([], []), ([5, 3], [0, 0])])
def test_empty_batches(pa, gpu_device, form, kind, prefix, ext):
    """No requests, or none with extend tokens: an empty result."""
    b = Batch(gpu_device, prefix + [9], ext + [1], 4, 512, *KINDS[kind], seed=1).fill(pa)
    if form == "expanded":
        b.weights(128)
    n = len(prefix)
    b.q, b.c = b.q[:0], b.c[:0]
    b.slot_idx, b.offsets, b.prefix_len = b.slot_idx[:sum(prefix)], b.offsets[:n + 1], b.prefix_len[:n]
    b.ext_len, b.ext_offsets, b.max_kv_len = b.ext_len[:n], b.ext_offsets[:n + 1], max(prefix, default=0)
    out = (b.absorbed if form == "absorbed" else b.expanded)(pa)
    assert tuple(out.shape) == (0, 4, 512 if form == "absorbed" else 128)
    none = torch.zeros(0, dtype=torch.int32, device=gpu_device)
    pa.append_latent(b.pool, none, b.c, rope_dim=P, **b.kw)
    assert tuple(pa.gather_latent(b.pool, none, latent_dim=512, rope_dim=P, dtype=b.dtype, **b.kw).shape) == (0, 576)


@pytest.mark.parametrize("most,less", [(8200, 7800), (9000, 8100)])
def test_a_workspace_sized_once(pa, gpu_device, most, less):
    """Sized for the largest batch, used for a smaller one that holds more heads at once."""
    H, slots = 128, 1 << 17
    size = pa.latent_expanded_workspace_bytes(8, 512, most, H, 512, P, 128, slots, torch.bfloat16)
    b = Batch(gpu_device, [less - 2] + [200] * 7, [2] * 8, H, 512, num_slots=slots, seed=2).fill(pa).weights(128)
    assert b.max_kv_len == less
    out = b.expanded(pa, workspace=torch.empty(size, dtype=torch.uint8, device=gpu_device))
    assert torch.equal(out.view(torch.int16), b.expanded(pa).view(torch.int16))
    ref, bound = b.reference("expanded")
    check(out, ref, bound, f"{less} of {most}")
