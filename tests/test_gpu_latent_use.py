"""GPU tests of latent attention as programs use it: matched prefixes and chunks, large and small batches, captured graphs, other streams, calls at
the same time, workspaces that hold anything, pools beyond 4 GiB, values beyond fp16's range."""
import numpy as np
import pytest
import torch

from latent_side import FORMS_TOLD, TOLD, Batch, P, check, quantise, told

pytestmark = pytest.mark.gpu
KINDS = {"f32": (torch.float32, False), "bf16": (torch.bfloat16, False), "bf16_kv8": (torch.bfloat16, True)}
FORMS = ["absorbed", "expanded"]


@pytest.fixture(scope="module")
def pa(gpu_device):
    from paper_2407_00023_amd import binding
    return binding


def make(pa, device, prefix, ext, H, R=512, kind="bf16", form="absorbed", N=128, **kw):
    dt, kv8 = KINDS[kind]
    b = Batch(device, prefix, ext, H, R, dt, kv8, **kw).fill(pa)
    return b.weights(N) if form == "expanded" else b


def run(pa, b, form, **kw):
    return (b.absorbed if form == "absorbed" else b.expanded)(pa, **kw)


def bits(t):
    return t.view(torch.int32 if t.dtype == torch.float32 else torch.int16)


def need(pa, b, form, T=None, max_kv_len=None):
    T, most = b.T if T is None else T, b.max_kv_len if max_kv_len is None else max_kv_len
    if form == "absorbed":
        return pa.latent_workspace_bytes(len(b.prefix), T, most, b.H, b.R, P, b.dtype)
    return pa.latent_expanded_workspace_bytes(len(b.prefix), T, most, b.H, b.R, P, b.N, b.num_slots, b.dtype)


# ---- sizes ------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("told", TOLD, indirect=True)
@pytest.mark.parametrize("R", [256, 512])
@pytest.mark.parametrize("kind", ["bf16", "bf16_kv8"])
@pytest.mark.parametrize("H,ext", [(64, 1), (48, 1), (33, 1), (16, 4), (64, 2)])
def test_tiles_of_64_and_128_rows(pa, gpu_device, kind, R, H, ext, told):
    b = make(pa, gpu_device, [31, 32, 33, 2000, 0, 64], [ext] * 6, H, R, kind, seed=H)
    check(b.absorbed(pa), *b.reference(), f"{H} heads, {ext} tokens, {kind}")


@pytest.mark.parametrize("form,told", FORMS_TOLD, indirect=["told"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("B", [257, 700, 2500])
def test_many_requests(pa, gpu_device, B, kind, form, told):
    """More requests than workgroups, and than a workgroup looks at together; some without extend tokens."""
    g = np.random.default_rng(B)
    prefix, ext = g.integers(0, 90, B).tolist(), g.integers(0, 3, B).tolist()
    b = make(pa, gpu_device, prefix, ext, 2, 256, kind, form, N=64, seed=B)
    check(run(pa, b, form), *b.reference(form), f"{B} requests, {kind}, {form}")


@pytest.mark.parametrize("told", TOLD, indirect=True)
@pytest.mark.parametrize("kind", ["bf16", "bf16_kv8"])
@pytest.mark.parametrize("prefix,ext,H", [([40000], [1], 16), ([30011], [3], 128), ([20000, 3, 17], [1, 1, 2], 5)])
def test_long_requests_cut_into_many_parts(pa, gpu_device, kind, prefix, ext, H, told):
    b = make(pa, gpu_device, prefix, ext, H, kind=kind, seed=H)
    check(b.absorbed(pa), *b.reference(), f"{prefix} cached, {H} heads, {kind}")
    b = make(pa, gpu_device, prefix, ext, min(H, 16), kind=kind, form="expanded", seed=H)
    check(b.expanded(pa), *b.reference("expanded"), f"{prefix} cached, expanded, {kind}")


def test_expanded_heads_in_several_groups(pa, gpu_device):
    """Expanded keys and values of all heads take more than the workspace holds at a time."""
    b = make(pa, gpu_device, [70000], [2], 130, form="expanded", seed=2)
    assert 4 * 128 * 70000 * 130 > 1 << 32
    check(b.expanded(pa), *b.reference("expanded"), "130 heads, 70 002 rows")


@pytest.mark.parametrize("form,told", FORMS_TOLD, indirect=["told"])
@pytest.mark.parametrize("kind", ["bf16", "bf16_kv8"])
def test_pool_beyond_4_gib(pa, gpu_device, kind, form, told):
    """Slots on both sides of 4 GiB and at the end of the pool."""
    dt, kv8 = KINDS[kind]
    row = 640 if kv8 else 1152
    b = Batch(gpu_device, [500, 90], [3, 70], 8, 512, dt, kv8, seed=4)
    if form == "expanded":
        b.weights(128)
    ref, bound = b.reference(form)
    big = (9 << 29) // row                                  # 4.5 GiB
    line = (1 << 32) // row
    where = torch.cat([torch.arange(line - 300, line + 200), torch.arange(0, 20), torch.arange(big - (b.num_slots - 520), big)])
    assert len(where) == b.num_slots
    pool = torch.empty(pa.latent_pool_bytes(big, 512, P, dt, kv8), dtype=torch.uint8, device=gpu_device)
    to = where.int().to(gpu_device)
    pa.append_latent(pool, to, b.rows_pool, rope_dim=P, num_slots=big, kv8=kv8)
    back = pa.gather_latent(pool, to, latent_dim=512, rope_dim=P, dtype=dt, num_slots=big, kv8=kv8)
    want = torch.cat([quantise(b.rows_pool[:, :512])[0], b.rows_pool[:, 512:].double()], 1) if kv8 else b.rows_pool.double()
    assert torch.equal(back.double(), want)
    b.pool, b.num_slots, b.kw = pool, big, dict(num_slots=big, kv8=kv8)
    idx = b.slot_idx.cpu().long()
    b.slot_idx = torch.where(idx >= 0, where[idx.clamp(min=0)], idx).int().to(gpu_device)
    check(run(pa, b, form), ref, bound, f"pool of {big} rows, {kind}, {form}")


# ---- values -----------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kind", ["bf16", "bf16_kv8"])
@pytest.mark.parametrize("of_k,of_v,of_c", [(-14, 0, 0), (0, 22, 0), (-14, -40, 0), (0, 0, -18), (2, 60, 3)])
def test_expanded_keys_and_values_out_of_half_precisions_range(pa, gpu_device, kind, of_k, of_v, of_c):
    """Powers of two on the weights, and on the rows of the extend tokens alone: blocks of keys and values with powers of their own."""
    b = make(pa, gpu_device, [300, 40], [90, 70], 3, kind=kind, form="expanded", seed=8)
    b.w_k, b.w_v, b.c = b.w_k * 2.0 ** of_k, b.w_v * 2.0 ** of_v, b.c * 2.0 ** of_c
    b.w_k[1] = b.w_k[1] * 2.0 ** -of_k   # (one head as usual)
    b.q[..., :128] = b.q[..., :128] * 2.0 ** min(-of_k, 8)
    check(b.expanded(pa), *b.reference("expanded"), f"2^{of_k}, 2^{of_v}, 2^{of_c}, {kind}")


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("order", ["rising", "falling", "jump"])
def test_expanded_scores_that_outgrow_the_running_maximum(pa, gpu_device, kind, order):
    dt, kv8 = KINDS[kind]
    b = Batch(gpu_device, [400], [3], 4, 512, dt, kv8, seed=9)
    factor = {"rising": torch.linspace(0, 12, 400), "falling": torch.linspace(12, 0, 400), "jump": (torch.arange(400) // 150).float() * 6}[order]
    direction = torch.randn(P, generator=torch.Generator().manual_seed(1))
    at = b.slots[0].to(gpu_device)
    b.rows_pool[at, 512:] = (factor[:, None] * direction[None]).to(gpu_device).to(dt)   # (the rotary part is a key as it is)
    b.fill(pa).weights(128)
    b.q[..., 128:] = direction.to(gpu_device).to(dt)
    check(b.expanded(pa), *b.reference("expanded"), order)


# ---- workspaces, streams, graphs -------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("form,told", FORMS_TOLD, indirect=["told"])
@pytest.mark.parametrize("kind", KINDS)
def test_whatever_the_workspace_holds(pa, gpu_device, kind, form, told):
    b = make(pa, gpu_device, [900, 33, 0], [2, 60, 5], 16, kind=kind, form=form, seed=1)
    ref, bound = b.reference(form)
    n = need(pa, b, form)
    for fill in (0xFF, 0x7F, 0x00):
        ws = torch.full((n + 256,), fill, dtype=torch.uint8, device=gpu_device)
        check(run(pa, b, form, workspace=ws[:n]), ref, bound, f"workspace of {fill:#x}")
        assert bool((ws[n:] == fill).all())


@pytest.mark.parametrize("form,told", FORMS_TOLD, indirect=["told"])
@pytest.mark.parametrize("kind", KINDS)
def test_two_streams_at_once(pa, gpu_device, kind, form, told):
    """Two calls at the same time, each with a workspace of its own, on streams other than the current one."""
    bs = [make(pa, gpu_device, [3000, 500], [1, 40], 16, kind=kind, form=form, seed=s) for s in (1, 2)]
    refs = [b.reference(form) for b in bs]
    ws = [torch.zeros(need(pa, b, form), dtype=torch.uint8, device=gpu_device) for b in bs]
    outs = [torch.zeros(r[0].shape, dtype=b.dtype, device=gpu_device) for r, b in zip(refs, bs)]
    streams = [torch.cuda.Stream() for _ in bs]
    torch.cuda.synchronize()
    for _ in range(3):
        for b, w, o, s in zip(bs, ws, outs, streams):
            run(pa, b, form, workspace=w, out=o, stream=s)
    torch.cuda.synchronize()
    for o, (ref, bound) in zip(outs, refs):
        check(o, ref, bound, f"{kind}, {form}, on a stream")


@pytest.mark.parametrize("form,told", FORMS_TOLD, indirect=["told"])
@pytest.mark.parametrize("kind", KINDS)
def test_captured_and_replayed(pa, gpu_device, kind, form, told):
    """Append and attention in one graph, two batches in two graphs on one workspace, replayed in turn with other inputs and eager work between."""
    bs = [make(pa, gpu_device, p, e, 16, kind=kind, form=form, seed=s) for s, (p, e) in enumerate([([700, 0, 90], [1, 3, 1]), ([40, 1500], [30, 1])])]
    ws = torch.zeros(max(need(pa, b, form) for b in bs), dtype=torch.uint8, device=gpu_device)
    graphs, outs = [], []
    every = [torch.arange(b.num_slots, dtype=torch.int32, device=gpu_device) for b in bs]
    for b, at in zip(bs, every):
        out = run(pa, b, form, workspace=ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            pa.append_latent(b.pool, at, b.rows_pool, rope_dim=P, **b.kw)
            run(pa, b, form, workspace=ws, out=out)
        graphs.append(graph)
        outs.append(out)
    for turn in range(3):
        for b, graph, out in zip(bs, graphs, outs):
            g = torch.Generator().manual_seed(100 + turn)
            b.q.copy_(torch.randn(b.q.shape, generator=g).to(b.dtype))
            b.rows_pool.copy_(torch.randn(b.rows_pool.shape, generator=g).to(b.dtype))
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            got = out.clone()
            check(got, *b.reference(form), f"replay {turn}")
            assert torch.equal(bits(run(pa, b, form, workspace=torch.empty_like(ws))), bits(got))
            torch.cuda.synchronize()


@pytest.mark.parametrize("form,told", FORMS_TOLD, indirect=["told"])
@pytest.mark.parametrize("kind", KINDS)
def test_same_inputs_same_bits(pa, gpu_device, kind, form, told):
    b = make(pa, gpu_device, [2000, 31, 500], [1, 50, 3], 16, kind=kind, form=form, seed=6, share=[0, 1, 2])
    first = run(pa, b, form).clone()
    for _ in range(4):
        assert torch.equal(bits(run(pa, b, form)), bits(first))


@pytest.mark.parametrize("form,less", [("absorbed", "T"), ("expanded", "T"), ("expanded", "keys")])
def test_a_batch_larger_than_the_host_was_told(pa, gpu_device, form, less):
    """The device's lengths add up to more than T, or to more keys than the expanded form has room for: nothing is written, and pa_extend_status says so."""
    b = make(pa, gpu_device, [100, 900], [300, 200], 16, form=form, seed=3)
    T, most = (60, b.max_kv_len) if less == "T" else (b.T, 500)
    n = need(pa, b, form, T, most)
    ws = torch.zeros(n, dtype=torch.uint8, device=gpu_device)
    ref, bound = b.reference(form)
    out = torch.full(ref.shape, 7.0, dtype=b.dtype, device=gpu_device)
    q, c, o = b.q, b.c, out
    b.q, b.c = q[:T], c[:T]
    run(pa, b, form, workspace=ws, out=o[:T], max_kv_len=most)
    with pytest.raises(pa.PrefixAttnError) as e:
        pa.extend_status(ws)
    assert e.value.code == -5 and bool((out == 7.0).all())
    b.q, b.c = q, c
    ws = torch.zeros(need(pa, b, form), dtype=torch.uint8, device=gpu_device)
    check(run(pa, b, form, workspace=ws), ref, bound)
    pa.extend_status(ws)


# ---- together ---------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("kind", KINDS)
def test_prompts_in_chunks_over_a_shared_prefix(pa, gpu_device, kind, form):
    """Serving: prompts are matched against the tree, what is missing goes through the attention in two chunks, whose rows are appended to the pool, then one
    new token each; the tree takes the prompts in.  Every result against the definition over the rows as the pool holds them."""
    dt, kv8 = KINDS[kind]
    g = torch.Generator().manual_seed(11)
    H, R, N, slots = 16, 512, 128, 2048
    doc = torch.randint(0, 1000, (300,), generator=g, dtype=torch.int32)
    prompts = [torch.cat([doc[:n], torch.randint(1000, 2000, (m,), generator=g, dtype=torch.int32)]) for n, m in ((300, 40), (300, 7), (120, 90), (0, 65))]
    rows = {tuple(p[:i + 1].tolist()): torch.randn(R + P, generator=g).to(dt) for p in prompts for i in range(len(p))}   # of a token behind its past
    row = lambda p, i: rows[tuple(p[:i + 1].tolist())]
    pool = torch.zeros(pa.latent_pool_bytes(slots, R, P, dt, kv8), dtype=torch.uint8, device=gpu_device)
    kw = dict(rope_dim=P, num_slots=slots, kv8=kv8)
    free = torch.randperm(slots, generator=g).int()
    doc_slots, free = free[:300], free[300:]
    pa.append_latent(pool, doc_slots.to(gpu_device), torch.stack([row(prompts[0], i) for i in range(300)]).to(gpu_device), **kw)
    tree = pa.Tree()
    tree.insert(doc.numpy(), doc_slots.numpy())
    tree.upload()
    w = torch.randn(2, H, N, R, generator=g).mul(R ** -0.5).to(dt).to(gpu_device)
    d = (N if form == "expanded" else R) + P
    held = [None] * len(prompts)
    done = [0] * len(prompts)
    stage = 0
    while True:
        if stage == 0:
            toks = torch.cat(prompts).to(gpu_device)
            offsets = torch.tensor(np.cumsum([0] + [len(p) for p in prompts]), dtype=torch.int32, device=gpu_device)
            lens, idx = pa.match_prefixes(tree, toks, offsets)
            done = [min(n, len(p) - 1) for n, p in zip(lens.tolist(), prompts)]
            assert done == [300, 300, 120, 0]
            held = [idx[offsets[r]:offsets[r] + done[r]].cpu().int() for r in range(len(prompts))]
        todo = [(len(p) - n) // 2 if stage == 0 else len(p) - 1 - n if stage == 1 else 1 for p, n in zip(prompts, done)]
        T = sum(todo)
        lists = [torch.cat([h, torch.full((e,), -1, dtype=torch.int32)]) for h, e in zip(held, todo)]
        b = Batch.__new__(Batch)
        b.prefix, b.ext, b.H, b.R, b.N, b.dtype, b.kv8, b.device, b.T = list(done), todo, H, R, N, dt, kv8, gpu_device, T
        b.num_slots, b.slots, b.kw, b.pool = slots, [h.long() for h in held], dict(num_slots=slots, kv8=kv8), pool
        b.c = torch.stack([row(p, i) for p, n, e in zip(prompts, done, todo) for i in range(n, n + e)]).to(gpu_device)
        b.q = torch.randn(T, H, d, generator=g).to(dt).to(gpu_device)
        b.scale, b.w_k, b.w_v = d ** -0.5, w[0].contiguous(), w[1].contiguous()
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=gpu_device)
        b.slot_idx, b.offsets = torch.cat(lists).to(gpu_device), i32(np.cumsum([0] + [len(x) for x in lists]).tolist())
        b.prefix_len, b.ext_len, b.ext_offsets = i32(done), i32(todo), i32(np.cumsum([0] + todo).tolist())
        b.max_kv_len = max(n + e for n, e in zip(done, todo))
        out = run(pa, b, form)
        new, free = free[:T], free[T:]
        pa.append_latent(pool, new.to(gpu_device), b.c, **kw)
        everything = torch.arange(slots, dtype=torch.int32, device=gpu_device)
        stored = pa.gather_latent(pool, everything, latent_dim=R, rope_dim=P, dtype=dt, num_slots=slots, kv8=kv8).double()
        check(out, *b.reference(form, stored), f"stage {stage}, {kind}, {form}")
        at = 0
        for r, e in enumerate(todo):
            held[r] = torch.cat([held[r], new[at:at + e]])
            at += e
            done[r] += e
            tail = torch.stack([row(prompts[r], i) for i in range(done[r])]).to(gpu_device)
            want = torch.cat([quantise(tail[:, :R])[0], tail[:, R:].double()], 1) if kv8 else tail.double()
            assert torch.equal(stored[held[r].long().to(gpu_device)], want)
        stage += 1
        if stage == 3:
            break
    assert done == [len(p) for p in prompts]
    for p, s in zip(prompts, held):
        tree.insert(p.numpy(), s.numpy())
    tree.upload()
    lens, idx = pa.match_prefixes(tree, toks, offsets)
    assert lens.tolist() == [len(p) for p in prompts]


def test_profile_names(pa, gpu_device):
    bs = [make(pa, gpu_device, [3000], [1], 16, kind=k, form=f, seed=1) for k in ("bf16", "f32") for f in FORMS]
    pa.profile_enable(True)
    for b, f in zip(bs, FORMS * 2):
        run(pa, b, f)
        pa.gather_latent(b.pool, b.slot_idx[:5], latent_dim=512, rope_dim=P, dtype=b.dtype, **b.kw)
    torch.cuda.synchronize()
    for name, least in {"latent_attention": 1, "latent_merge": 2, "latent_attention_f32": 2, "latent_expand": 4, "latent_attention_expanded": 1, "gather_latent": 4,
                        "append_latent": 0}.items():
        ms, n = pa.profile_read(name)
        assert n >= least and (ms > 0 or n == 0), (name, ms, n)
    pa.profile_enable(False)


@pytest.mark.parametrize("told", TOLD, indirect=True)
@pytest.mark.parametrize("kind", ["bf16", "bf16_kv8"])
def test_128_heads_many_times_over(pa, gpu_device, kind, told):
    """Calls behind one another: the same bits every time, within the bound (a result that was read a few cycles too early showed now and then)."""
    b = make(pa, gpu_device, [100, 1000, 5], [1, 1, 1], 128, kind=kind, seed=17)
    ref, bound = b.reference()
    first = b.absorbed(pa).clone()
    check(first, ref, bound, f"128 heads, {kind}")
    for _ in range(40):
        assert torch.equal(bits(b.absorbed(pa)), bits(first))
