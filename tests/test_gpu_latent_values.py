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
@pytest.mark.parametrize("of", [-20, -14, -12, -10, -9, -8, 8, 14, 30, 60])
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


@pytest.mark.parametrize("kind", ["bf16", "bf16_kv8"])
@pytest.mark.parametrize("prefix,ext", [([6000], [2]), ([200], [2]), ([40000, 300], [3, 130])])
@pytest.mark.parametrize("of", [90, 112, 120, -100])
def test_expanded_values_at_the_ends_of_the_range(pa, gpu_device, kind, of, prefix, ext):
    """Results of up to 2^120, from whole tiles and from tiles in parts: no sum on the way is larger than fp32 holds."""
    b = Batch(gpu_device, prefix, ext, 2, 512, *KINDS[kind], seed=20).fill(pa).weights(128)
    b.w_v = b.w_v * 2.0 ** of
    check(b.expanded(pa), *b.reference("expanded"), f"2^{of}, {kind}")


def test_expanded_heads_of_different_sizes_in_several_groups(pa, gpu_device):
    """Keys and values of all heads take more than the workspace holds at a time; some heads of each group have values of powers of their own."""
    b = Batch(gpu_device, [70000], [2], 130, 512, seed=2).fill(pa).weights(128)
    b.w_v[::3] = b.w_v[::3] * 2.0 ** -12
    b.w_k[1::7] = b.w_k[1::7] * 2.0 ** -14
    check(b.expanded(pa), *b.reference("expanded"), "130 heads")


# ---- scores --------------------------------------------------------------------------------------------------------------------

def check_winners(b, out, form):
    """Scores so large that one key has all the weight: its value comes out.  Which key it is may be left to rounding only where two scores are nearer to
    one another than fp32 sums of their magnitude are exact, (width + 2) 2^-24 times the sum of the products' magnitudes, for each of the two, and e^-30."""
    rows, t, told_apart = b.stored(), 0, 0
    h, h16 = HALF[b.dtype], 0.0 if b.dtype == torch.float32 else HALF[torch.float16]
    for r, (n, e) in enumerate(zip(b.prefix, b.ext)):
        keys = torch.cat([rows[b.slots[r].to(rows.device)], b.c[t:t + e].double()])
        q, lat, rope = b.q[t:t + e].double(), keys[:, :b.R], keys[:, b.R:]
        hidden = torch.arange(n + e, device=q.device)[None] > n + torch.arange(e, device=q.device)[:, None]
        for x in range(b.H):
            if form == "absorbed":
                k, v, size = keys, lat, (b.R + P + 2) * 2.0 ** -24 * (q[:, x].abs() @ keys.abs().T)
                tol_v = v.abs() * h
            else:
                wk, wv = b.w_k[x].double(), b.w_v[x].double()
                k, v = torch.cat([lat @ wk.T, rope], 1), lat @ wv.T
                sums = (b.R + 2) * 2.0 ** -24 + (b.N + 2) * 2.0 ** -24 * (b.dtype == torch.float32)
                grow = torch.cat([lat.abs() @ wk.abs().T * sums + k[:, :b.N].abs() * h16 + 2.0 ** -17 * h16 / HALF[torch.float16] * k[:, :b.N].abs().amax(1, True), rope * 0], 1)
                size = (b.N + P + 2) * 2.0 ** -24 * (q[:, x].abs() @ k.abs().T) + q[:, x].abs() @ grow.T
                tol_v = v.abs() * (h + h16) * 1.01 + 2.0 ** -17 * v.abs().amax(1, True) * (h16 > 0) + lat.abs() @ wv.abs().T * sums
            z = (q[:, x] @ k.T).masked_fill(hidden, -torch.inf)
            best = z.amax(1, keepdim=True)
            off = (size.masked_fill(hidden, 0)).amax(1, keepdim=True)
            rival = (z + 2 * off + 30 / b.scale >= best) & ~hidden
            alone = rival.sum(1) == 1
            told_apart += int(alone.sum())
            got = out[t:t + e, x].double()
            win = z.argmax(1)
            assert bool(((got - v[win]).abs() <= tol_v[win] + h * v[win].abs())[alone].all()), (r, x)
            low = torch.where(rival[..., None], v - tol_v, torch.inf).amin(1)       # beside rivals: between their values
            high = torch.where(rival[..., None], v + tol_v, -torch.inf).amax(1)
            room = 2 * h * torch.maximum(low.abs(), high.abs())
            assert bool(((got >= low - room) & (got <= high + room)).all()), (r, x)
        t += e
    return told_apart


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("of_q,of_c", [(12, 10), (14, 12), (15, 13), (20, 10), (17, 16), (22, 18), (40, 20)])
@pytest.mark.parametrize("prefix,ext", [([400, 33], [3, 40]), ([3000], [5])])
def test_expanded_scores_beyond_the_steps_of_fp32(pa, gpu_device, kind, of_q, of_c, prefix, ext):
    """Scores of 2^22 to 2^60."""
    b = Batch(gpu_device, prefix, ext, 3, 512, *KINDS[kind], seed=12).weights(128)
    b.rows_pool, b.c, b.q = b.rows_pool * 2.0 ** of_c, b.c * 2.0 ** of_c, b.q * 2.0 ** of_q
    b.fill(pa)
    apart = check_winners(b, b.expanded(pa), "expanded")
    assert apart >= b.T * b.H // 2


KINDS_TOLD = [("f32", 0)] + [(k, x) for k in ("bf16", "bf16_kv8") for x in TOLD]   # (fp32 has no tiles)


@pytest.mark.parametrize("kind,told", KINDS_TOLD, indirect=["told"])
@pytest.mark.parametrize("R", [512, 256])
@pytest.mark.parametrize("H", [3, 64])
@pytest.mark.parametrize("of_q,of_c", [(12, 10), (16, 16), (18, 15), (22, 18), (60, 20)])
def test_absorbed_scores_beyond_the_steps_of_fp32(pa, gpu_device, kind, R, H, of_q, of_c, told):
    b = Batch(gpu_device, [400, 33, 1500], [3, 40 if H == 3 else 2, 1], H, R, *KINDS[kind], seed=13)
    b.rows_pool, b.c, b.q = b.rows_pool * 2.0 ** of_c, b.c * 2.0 ** of_c, b.q * 2.0 ** of_q
    b.fill(pa)
    apart = check_winners(b, b.absorbed(pa), "absorbed")
    assert apart >= b.T * b.H // 2


def weights_far_below(b):
    """The expanded form's definition and a bound that knows of the probabilities' fp16 only that they are off by 2^-11 of themselves or by 2^-33 of their row's
    largest, whichever is more.  The queries have no latent part here: scores are products of rotary parts, as given."""
    h, outs, bounds, t = HALF[b.dtype], [], [], 0
    h16, rows = 0.0 if b.dtype == torch.float32 else HALF[torch.float16], b.stored()
    for r, (n, e) in enumerate(zip(b.prefix, b.ext)):
        keys = torch.cat([rows[b.slots[r].to(rows.device)], b.c[t:t + e].double()])
        lat, q_r = keys[:, :b.R], b.q[t:t + e, :, b.N:].double()
        assert not bool(b.q[t:t + e, :, :b.N].any())
        hidden = torch.arange(n + e, device=keys.device)[None] > n + torch.arange(e, device=keys.device)[:, None]
        for x in range(b.H):
            v, size_v = lat @ b.w_v[x].double().T, lat.abs() @ b.w_v[x].double().abs().T
            z = (q_r[:, x] @ keys[:, b.R:].T * b.scale).masked_fill(hidden, -torch.inf)
            p = torch.softmax(z, 1)
            out = p @ v
            dz = ((P + 2) * 2.0 ** -24 * (q_r[:, x].abs() @ keys[:, b.R:].abs().T) * b.scale).masked_fill(hidden, 0).amax(1, keepdim=True)
            grow_v = size_v * (b.R + 2) * 2.0 ** -24 + (h16 * v.abs() + (2.0 ** -17 if h16 else 0.0) * v.abs().amax(1, keepdim=True))
            bound = (p @ v.abs()) * (2 * dz + 2.0 ** -20 + (n + e + 64) * 2.0 ** -24 + h16) + h * out.abs() + p @ grow_v * (1 + h) + 1e-30
            if h16:
                bound = bound + 2.0 ** -33 * p.amax(1, keepdim=True) * ((~hidden).double() @ v.abs())
            outs.append(out)
            bounds.append(bound)
        t += e
    lay = lambda ys: torch.cat([torch.stack(ys[r * b.H:(r + 1) * b.H], 1) for r in range(len(b.prefix))])
    return lay(outs), lay(bounds)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("far", [6, 14, 17.3, 19.3, 20.4, 22.6, 24.5, 26])
@pytest.mark.parametrize("where", ["first", "last"])
def test_expanded_many_keys_far_below_the_largest(pa, gpu_device, kind, far, where):
    """A key takes nearly all the weight and has a value of zero; what comes out are the many others, 2^-far of it each."""
    prefix, ext, H = [3000, 700], [3, 40], 2
    b = Batch(gpu_device, prefix, ext, H, 512, *KINDS[kind], seed=14).weights(128)
    g = torch.Generator().manual_seed(15)
    row = torch.randn(1, 512, generator=g)
    b.rows_pool = torch.cat([row + 0.05 * torch.randn(b.num_slots, 512, generator=g), torch.zeros(b.num_slots, P)], 1).to(b.dtype).to(gpu_device)
    b.c = torch.cat([row + 0.05 * torch.randn(b.T, 512, generator=g), torch.zeros(b.T, P)], 1).to(b.dtype).to(gpu_device)
    b.q = torch.zeros_like(b.q)
    b.q[..., b.N] = 8
    for s in b.slots:
        at = s[0] if where == "first" else s[-1]
        b.rows_pool[at] = 0
        b.rows_pool[at, 512] = far * 0.6931471805599453 / (8 * b.scale)
    b.fill(pa)
    check(b.expanded(pa), *weights_far_below(b), f"2^-{far}, {kind}")


# ---- infinities ----------------------------------------------------------------------------------------------------------------

def definition_with_infinities(b, form):
    """The definition row by row over the keys that the row sees, as arithmetic has it: a score of +infinity or NaN makes the row NaN, one of -infinity gives its
    key the weight 0, and 0 times an infinite value is NaN in its column.  The bound (elsewhere) is that of Batch.reference over the keys that have a weight."""
    h, rows, t = HALF[b.dtype], b.stored(), 0
    h16 = HALF[torch.float16] if form == "expanded" and b.dtype != torch.float32 else 0.0
    ref = torch.full((b.T, b.H, b.R if form == "absorbed" else b.N), torch.nan, dtype=torch.float64, device=rows.device)
    bound = torch.ones_like(ref)
    for r, (n, e) in enumerate(zip(b.prefix, b.ext)):
        keys = torch.cat([rows[b.slots[r].to(rows.device)], b.c[t:t + e].double()])
        lat, rope = keys[:, :b.R], keys[:, b.R:]
        for x in range(b.H):
            if form == "absorbed":
                k, v, grow_k, grow_v = keys, lat, torch.zeros_like(keys), torch.zeros_like(lat)
            else:
                wk, wv = b.w_k[x].double(), b.w_v[x].double()
                k, v = torch.cat([lat @ wk.T, rope], 1), lat @ wv.T
                sums = (b.R + b.N + 2) * 2.0 ** -24
                grow_k = torch.cat([lat.abs() @ wk.abs().T * sums + h16 * k[:, :b.N].abs() + (2.0 ** -17 * k[:, :b.N].abs().amax(1, True) if h16 else 0.0), rope * 0], 1)
                grow_v = lat.abs() @ wv.abs().T * sums + h16 * v.abs() + (2.0 ** -17 * v.abs().amax(1, True) if h16 else 0.0)
            for i in range(e):
                seen, q = n + i + 1, b.q[t + i, x].double()
                z = (k[:seen] * q).sum(1) * b.scale
                if bool(torch.isnan(z).any()) or bool((z == torch.inf).any()) or not bool(torch.isfinite(z).any()):
                    continue
                keep = torch.isfinite(z)
                p, vk = torch.softmax(z[keep], 0), v[:seen][keep]
                out = p @ vk
                dz = float((((k.shape[1] + 2) * 2.0 ** -24 * k[:seen][keep].abs() + grow_k[:seen][keep]) @ q.abs()).max()) * b.scale
                hp = 0.0 if b.dtype == torch.float32 else h16 or h
                bound[t + i, x] = (p @ vk.abs()) * (2 * dz + 2.0 ** -20 + (seen + 64) * 2.0 ** -24 + hp) + h * out.abs() + p @ grow_v[:seen][keep] * (1 + h) + 1e-30
                if h16:
                    bound[t + i, x] += 2.0 ** -33 * vk.abs().sum(0)
                ref[t + i, x] = torch.where(torch.isfinite(v[:seen]).all(0), out, torch.nan)
        t += e
    return ref, bound


def check_with_infinities(out, ref, bound, what=""):
    assert torch.equal(torch.isnan(out), torch.isnan(ref)), (what, int(torch.isnan(out).sum()), int(torch.isnan(ref).sum()))
    there = ~torch.isnan(ref)
    check(out[there], ref[there], bound[there], what)


FORMS_KINDS_TOLD = [("absorbed",) + x for x in KINDS_TOLD] + [("expanded", k, 0) for k in KINDS]


def looking_away(b, form, where, value):
    """Queries of heads 0, 4, 8, ... whose score with a latent `value` at column `where` is -infinity, those of 1, 5, ... +infinity, 2, 6, ... NaN;
    3, 7, ... as they are."""
    s = 1.0 if value > 0 else -1.0
    for x in range(b.H):
        if x % 4 == 3:
            continue
        if form == "absorbed":
            b.q[:, x, where] = [-s, s, 0][x % 4]
        else:
            at = torch.sign(b.w_k[x, :, where].float())
            b.q[:, x, :b.N] = ((-s if x % 4 == 0 else s) * at * b.q[:, x, :b.N].float().abs().clamp(min=0.01)).to(b.dtype)
            if x % 4 == 2:
                b.q[:, x, 0] = 0


@pytest.mark.parametrize("form,kind,told", FORMS_KINDS_TOLD, indirect=["told"])
@pytest.mark.parametrize("value", [float("inf"), -float("inf")])
@pytest.mark.parametrize("prefix,ext,row", [([45, 10], [40, 3], 21), ([2000], [4], 1), ([3, 64], [2, 1], 1)])
def test_infinite_latent_values_in_new_rows(pa, gpu_device, form, kind, value, prefix, ext, row, told):
    b = Batch(gpu_device, prefix, ext, 8, 512, *KINDS[kind], seed=16).fill(pa)
    if form == "expanded":
        b.weights(128)
    looking_away(b, form, 300, value)
    b.c[row, 300] = value
    out = (b.absorbed if form == "absorbed" else b.expanded)(pa)
    check_with_infinities(out, *definition_with_infinities(b, form), f"{value} in row {row}, {kind}")


@pytest.mark.parametrize("form,kind,told", [x for x in FORMS_KINDS_TOLD if x[1] != "bf16_kv8"], indirect=["told"])
@pytest.mark.parametrize("value", [float("inf"), -float("inf")])
@pytest.mark.parametrize("at", [0, 500, 1998, 1999])
def test_infinite_latent_values_in_cached_rows(pa, gpu_device, form, kind, value, at, told):
    b = Batch(gpu_device, [2000, 90], [3, 2], 8, 512, *KINDS[kind], seed=17)
    b.rows_pool[b.slots[0][at], 300] = value
    b.fill(pa)
    if form == "expanded":
        b.weights(128)
    looking_away(b, form, 300, value)
    out = (b.absorbed if form == "absorbed" else b.expanded)(pa)
    check_with_infinities(out, *definition_with_infinities(b, form), f"{value} in key {at}, {kind}")


@pytest.mark.parametrize("form,kind,told", FORMS_KINDS_TOLD, indirect=["told"])
@pytest.mark.parametrize("far,sign", [(10, 1), (40, 1), (200, 1), (10, -1)])
@pytest.mark.parametrize("hidden,prefix,ext", [(40, 90, 3), (1, 0, 5), (700, 1500, 2), (32, 32, 1)])
def test_infinite_rotary_values(pa, gpu_device, form, kind, far, sign, hidden, prefix, ext, told):
    """The first `hidden` keys have scores of -infinity (or +infinity) from a rotary value, those behind them scores 2^-far below 0: they have no weight, and with
    none left a row is NaN."""
    b = Batch(gpu_device, [prefix, 70], [ext, 2], 4, 512, *KINDS[kind], seed=18)
    if form == "expanded":
        b.weights(128)
    at = b.q.shape[2] - P
    b.q[..., :at] = b.q[..., :at] * 0.1
    b.q[..., at] = 1
    b.q[..., at + 1] = 8
    b.rows_pool[:, 512:] = 0
    b.c[:, 512:] = 0
    keys = [b.rows_pool[s] for s in b.slots[0]] + [b.c[i] for i in range(ext)]
    for i, key in enumerate(keys):
        key[512] = sign * -float("inf") if i < hidden else 0
        key[513] = -far * 0.6931471805599453 / (8 * b.scale)
    b.fill(pa)
    out = (b.absorbed if form == "absorbed" else b.expanded)(pa)
    check_with_infinities(out, *definition_with_infinities(b, form), f"{far}, {sign}, {kind}")


# ---- the ends of the range -----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("form", ["absorbed", "expanded"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("of_q,of_scale", [(-118, -30), (-100, -40), (-10, -100), (100, -140)])
def test_queries_and_scales_so_small_that_all_keys_weigh_the_same(pa, gpu_device, form, kind, of_q, of_scale):
    b = Batch(gpu_device, [300, 5], [3, 40], 4, 512, *KINDS[kind], seed=19).fill(pa)
    if form == "expanded":
        b.weights(128)
    b.q, b.scale = b.q * 2.0 ** of_q, 2.0 ** of_scale
    check((b.absorbed if form == "absorbed" else b.expanded)(pa), *b.reference(form), f"2^{of_q}, scale 2^{of_scale}, {kind}")
