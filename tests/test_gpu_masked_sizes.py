"""Masked attention where the kernels for few and for many query rows meet, the kernel for many rows with bf16 caches (it takes
calls whose rows fill the chip: 64 sequences here, most of them short), and calls as a serving loop makes them: prepared buffers,
another stream, tensors inside larger ones."""
import math

import pytest
import torch

from paper_2502_07864_amd import layer, mla
from test_gpu_masked import (BF, Cache, DEV, F32, FP8, SCALE, check, gen, queries, run_prefill, run_tree, run_window, tree_of, tree_sees,
                             window_sees)

pytestmark = pytest.mark.gpu


def crowd(lens, low=0):
    """As many sequences as fill the chip with 128 query rows each, the given ones between short ones."""
    out = [low + b % 4 for b in range(64)]
    for i, l in enumerate(lens):
        out[(i * 11 + 5) % 64] = l
    return out


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("d_c", [256, 512])
@pytest.mark.parametrize("T, H", [(20, 28), (64, 9), (5, 103)])
def test_many_rows(kind, d_c, T, H):
    run_tree(kind, crowd([31, 32, 33, 64, 65, 200, 447]), T, H, d_c)


@pytest.mark.parametrize("d_c", [256, 512])
@pytest.mark.parametrize("window, sinks", [(1, 0), (33, 1), (64, 64), (100, 100), (5000, 3)])
def test_many_rows_under_a_window(d_c, window, sinks):
    run_window("bf16", crowd([31, 64, 65, 130, 700, 1025], 1), 20, 28, window, sinks, d_c)


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("d_c", [256, 512])
def test_many_rows_in_chunks(kind, d_c):
    run_tree(kind, [16000, 9000], 20, 28, d_c)


@pytest.mark.parametrize("kind, d_c, longest", [("bf16", 512, 14700), ("bf16", 256, 14700), ("fp8", 512, 14700), ("fp8", 256, 29500)])
def test_few_rows_of_a_large_cache(kind, d_c, longest):
    """64 MB of rows and more for 32 query rows go past the caches."""
    (out, lse), c, (q, qr), mask, lens = run_tree(kind, [longest, 3, 9000, 0, 31, 700, 64, 2000], 2, 16, d_c)
    for _ in range(3):
        o, l = mla.decode_paged_tree(q, qr, c.kv, c.table, lens, mask, SCALE, kv_scale=c.scale, return_lse=True)
        assert torch.equal(o, out) and torch.equal(l, lse)


@pytest.mark.parametrize("page", [32, 96])
def test_many_rows_pages(page):
    run_tree("bf16", crowd([95, 96, 97, 300]), 20, 28, page=page)


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("d_c", [256, 512])
@pytest.mark.parametrize("page", [16, 48, 80])
def test_pages_that_end_inside_a_tile(kind, d_c, page):
    run_tree(kind, [0, 15, 16, 17, 47, 48, 49, 500], 5, 28, d_c, page=page)
    run_tree(kind, crowd([47, 95, 96, 97, 300]), 20, 28, d_c, page=page)
    run_window(kind, [15, 16, 17, 700, 1111], 3, 20, 100, 20, d_c, page=page)
    run_window(kind, [3000], 1, 32, 2500, 4, d_c, page=page)


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("H, T", [(28, 20), (8, 4)])
def test_half_tiles_that_are_not_there(kind, H, T):
    """Pages of 16 rows: either half of a tile may be missing, and the table may end inside one."""
    prefix, cache = crowd([200, 90, 23]), FP8 if kind == "fp8" else BF
    c = Cache([p + T for p in prefix], 512, 64, 16, cache, 3)
    a, b, e = prefix.index(200), prefix.index(90), prefix.index(23)
    c.table[a, 0], c.table[a, 3], c.table[a, 10], c.table[b, 1], c.table[e, 0] = -1, c.kv.shape[0], 1 << 30, -5, -1
    masks = [tree_of(T, 5 + k) for k in range(64)]
    q, qr = queries(64, T, H, 512, 64, BF)
    mask = torch.tensor(masks, dtype=torch.int64, device=DEV)
    lens = torch.tensor(prefix, dtype=torch.int32, device=DEV)
    for width in (c.table.shape[1], 3):
        c.table = c.table[:, :width].contiguous()
        check(c, q, qr, tree_sees([min(p, 16 * width) for p in prefix], masks, T, min(200 + T, 16 * width)),
              lambda: mla.decode_paged_tree(q, qr, c.kv, c.table, lens, mask, SCALE, kv_scale=c.scale, return_lse=True), BF)


@pytest.mark.parametrize("scale", [-SCALE, 0.0, 3.0])
def test_many_rows_scales(scale):
    run_tree("bf16", crowd([40, 300]), 20, 28, scale=scale)


@pytest.mark.parametrize("d_c", [256, 512])
@pytest.mark.parametrize("where", [0, 40, 447, 500])
def test_many_rows_score_that_dominates(d_c, where):
    T, H, prefix = 20, 28, crowd([490])
    c = Cache([p + T for p in prefix], d_c, 64, 64, BF, 8)
    q, qr = queries(64, T, H, d_c, 64, BF)
    b = prefix.index(490)
    c.put(b, [where], torch.cat((q[b, 2, 5], qr[b, 2, 5])).float()[None] * 12.0)
    masks = [tree_of(T, 2 + k) for k in range(64)]
    masks[b][2] |= 1 << 10
    mask = torch.tensor(masks, dtype=torch.int64, device=DEV)
    lens = torch.tensor(prefix, dtype=torch.int32, device=DEV)
    check(c, q, qr, tree_sees(prefix, masks, T, max(prefix) + T),
          lambda: mla.decode_paged_tree(q, qr, c.kv, c.table, lens, mask, SCALE, return_lse=True), BF)


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("d_c", [256, 512])
def test_many_rows_other_branches_do_not_leak(kind, d_c):
    T, H, prefix = 20, 28, crowd([70, 45, 64])
    masks = [tree_of(T, b) for b in range(64)]
    (out, lse), c, (q, qr), mask, lens = run_tree(kind, prefix, T, H, d_c, masks=masks)
    rows = c.scale.view(-1) if kind == "fp8" else c.kv.view(-1, d_c + 64)
    for b in (prefix.index(70), prefix.index(45), 0):
        for bad in (0, 7, 19):
            at = c.places(b, [prefix[b] + bad])
            kept = rows[at].clone()
            for what in (math.nan, math.inf):
                rows[at] = what
                got, l2 = mla.decode_paged_tree(q, qr, c.kv, c.table, lens, mask, SCALE, kv_scale=c.scale, return_lse=True)
                for i in range(T):
                    if masks[b][i] >> bad & 1:
                        assert not torch.isfinite(got[b, i].float()).any()
                    else:
                        assert torch.equal(got[b, i], out[b, i]) and torch.equal(l2[b, i], lse[b, i]), (b, bad, i)
                others = torch.arange(64, device=DEV) != b
                assert torch.equal(got[others], out[others])
            rows[at] = kept


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
def test_many_rows_pages_that_are_not_there(kind):
    T, H, prefix = 20, 28, crowd([200, 90])
    cache = FP8 if kind == "fp8" else BF
    c = Cache([p + T for p in prefix], 512, 64, 64, cache, 3)
    a, b = prefix.index(200), prefix.index(90)
    c.table[a, 0], c.table[a, 3], c.table[b, 1], c.table[1, 0] = -1, c.kv.shape[0], 1 << 30, -1
    masks = [tree_of(T, 5 + k) for k in range(64)]
    q, qr = queries(64, T, H, 512, 64, BF)
    mask = torch.tensor(masks, dtype=torch.int64, device=DEV)
    lens = torch.tensor(prefix, dtype=torch.int32, device=DEV)
    check(c, q, qr, tree_sees(prefix, masks, T, 220),
          lambda: mla.decode_paged_tree(q, qr, c.kv, c.table, lens, mask, SCALE, kv_scale=c.scale, return_lse=True), BF)


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("T, H", [(1, 31), (1, 33), (1, 65), (1, 127), (43, 3), (1, 255), (1, 257), (61, 17)])
def test_query_rows_about_a_workgroups(kind, T, H):
    run_tree(kind, [0, 63, 500], T, H)
    run_window(kind, [64, 63, 500], T, H, 70, 4)


@pytest.mark.parametrize("T", [127, 128, 129, 250])
def test_prompts_about_a_workgroups_rows(T):
    run_prefill([T, 700], T, 2, 65, 5, 256)


# ------------------------------------------------------------------ calls as they are made

def prepared(kind, T=6, H=32, prefix=(700, 40)):
    cache = {"bf16": BF, "fp8": FP8}[kind]
    _, c, (q, qr), mask, lens = run_tree(kind, list(prefix), T, H)
    rows, B = c.table.shape[1] * 64, len(prefix)
    n = max(mla.decode_tree_workspace_bytes(B, T, H, 512, rows), mla.decode_window_workspace_bytes(B, T, H, 512, rows, 300, 4))
    ws = torch.full((max(n, 256),), 255, dtype=torch.uint8, device=DEV)
    def tree(**kw):
        return mla.decode_paged_tree(q, qr, c.kv, c.table, lens, mask, SCALE, kv_scale=c.scale, **kw)
    def window(**kw):
        return mla.decode_paged_window(q, qr, c.kv, c.table, lens + T, 300, 4, SCALE, kv_scale=c.scale, **kw)
    return q, ws, tree, window


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
def test_prepared_buffers_give_the_same_bits_either_way(kind, monkeypatch):
    """With every buffer given the native argument path takes the call, without it the binding."""
    q, ws, tree, window = prepared(kind)
    for call in (tree, window):
        ref, lse = call(return_lse=True)
        for native in (True, False):
            if not native:
                monkeypatch.setattr(mla, "_fast", None)
            out, l2 = torch.full_like(q, math.nan), torch.full_like(lse, math.nan)
            call(workspace=ws, out=out, lse=l2, return_lse=True)
            assert torch.equal(out, ref) and torch.equal(l2, lse), native
            out.fill_(math.nan)
            assert torch.equal(call(workspace=ws, out=out), ref)
        monkeypatch.undo()


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
def test_nothing_beside_the_results_is_written(kind):
    q, ws, tree, window = prepared(kind)
    for call in (tree, window):
        ref, lse = call(return_lse=True)
        room, room2 = torch.full((q.numel() + 128,), 7.0, dtype=BF, device=DEV), torch.full((lse.numel() + 64,), 7.0, device=DEV)
        work = torch.full((ws.numel() + 512,), 77, dtype=torch.uint8, device=DEV)
        out, l2 = room[64:-64].view(q.shape), room2[32:-32].view(lse.shape)
        call(workspace=work[256:-256], out=out, lse=l2, return_lse=True)
        assert torch.equal(out, ref) and torch.equal(l2, lse)
        assert (room[:64] == 7).all() and (room[-64:] == 7).all() and (room2[:32] == 7).all() and (room2[-32:] == 7).all()
        assert (work[:256] == 77).all() and (work[-256:] == 77).all()


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
def test_another_stream_waits_for_nobody_else(kind):
    """Two calls on two streams, each with buffers of its own."""
    q, ws, tree, window = prepared(kind)
    refs = [tree(), window()]
    torch.cuda.synchronize()
    streams, outs, work = [torch.cuda.Stream() for _ in range(2)], [torch.empty_like(q) for _ in range(2)], [ws, ws.clone()]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, call, o, w in zip(streams, (tree, window), outs, work):
            with torch.cuda.stream(s):
                call(workspace=w, out=o)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, refs))


def test_tensors_off_sixteen_bytes():
    """bf16 queries and caches that begin two bytes on go through the kernel that takes any alignment."""
    T, H, prefix = 5, 32, [200, 31]
    c = Cache([p + T for p in prefix], 512, 64, 64, BF, 3)
    masks = [tree_of(T, 5), tree_of(T, 6)]
    def off(x):
        y = torch.empty(x.numel() + 1, dtype=x.dtype, device=DEV)[1:].view(x.shape)
        return y.copy_(x)
    q, qr = (off(x) for x in queries(2, T, H, 512, 64, BF))
    c.kv = off(c.kv)
    mask = torch.tensor(masks, dtype=torch.int64, device=DEV)
    lens = torch.tensor(prefix, dtype=torch.int32, device=DEV)
    check(c, q, qr, tree_sees(prefix, masks, T, 205),
          lambda: mla.decode_paged_tree(q, qr, c.kv, c.table, lens, mask, SCALE, return_lse=True), BF)
    check(c, q, qr, window_sees([205, 36], T, 50, 3, 205),
          lambda: mla.decode_paged_window(q, qr, c.kv, c.table, lens + T, 50, 3, SCALE, return_lse=True), BF)


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
def test_rows_past_four_gigabytes(kind):
    """Pages whose bytes lie past 32 bits of the pool."""
    T, H, prefix, cache = 4, 32, [300, 64], FP8 if kind == "fp8" else BF
    c = Cache([p + T for p in prefix], 512, 64, 64, cache, 3)
    pages = (5 << 30) // (64 * 576 * c.kv.element_size())
    kv = torch.empty((pages, 64, 576), dtype=cache, device=DEV)
    n = c.kv.shape[0]
    kv.view(torch.uint8)[-n:] = c.kv.view(torch.uint8)
    c.kv, c.table = kv, torch.where(c.table >= 0, c.table + (pages - n), c.table)
    if cache == FP8:
        scale = torch.zeros((pages, 64), device=DEV)
        scale[-n:] = c.scale
        c.scale = scale
    masks = [tree_of(T, 5), tree_of(T, 6)]
    mask, lens = torch.tensor(masks, dtype=torch.int64, device=DEV), torch.tensor(prefix, dtype=torch.int32, device=DEV)
    q, qr = queries(2, T, H, 512, 64, BF)
    check(c, q, qr, tree_sees(prefix, masks, T, 304),
          lambda: mla.decode_paged_tree(q, qr, c.kv, c.table, lens, mask, SCALE, kv_scale=c.scale, return_lse=True), BF)
    check(c, q, qr, window_sees([304, 68], T, 90, 3, 304),
          lambda: mla.decode_paged_window(q, qr, c.kv, c.table, lens + T, 90, 3, SCALE, kv_scale=c.scale, return_lse=True), BF)
    src = torch.tensor([[300, 302]], dtype=torch.int32, device=DEV)
    want = c.kv.view(torch.uint8).view(-1, 576 * c.kv.element_size())[c.places(0, [300, 302])].clone()
    layer.cache_move(c.kv, c.table[:1], src, torch.tensor([[10, 11]], dtype=torch.int32, device=DEV), kv_scale=c.scale)
    assert torch.equal(c.kv.view(torch.uint8).view(-1, 576 * c.kv.element_size())[c.places(0, [10, 11])], want)


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
def test_results_off_sixteen_bytes(kind):
    """Outputs that begin anywhere, whole and in chunks."""
    for T, H, prefix in ((6, 32, [700, 40]), (20, 28, crowd([90]))):
        (ref, lse), c, (q, qr), mask, lens = run_tree(kind, prefix, T, H)
        room, room2 = torch.full((q.numel() + 9,), 7.0, dtype=BF, device=DEV), torch.full((lse.numel() + 3,), 7.0, device=DEV)
        out, l2 = room[1:-8].view(q.shape), room2[1:-2].view(lse.shape)
        mla.decode_paged_tree(q, qr, c.kv, c.table, lens, mask, SCALE, kv_scale=c.scale, out=out, lse=l2)
        assert torch.equal(out, ref) and torch.equal(l2, lse)
        assert (room[:1] == 7).all() and (room[-8:] == 7).all() and (room2[:1] == 7).all() and (room2[-2:] == 7).all()
        n, wide = lens + T, 2 ** 32 + 3
        a = mla.decode_paged_window(q, qr, c.kv, c.table, n, wide, wide, SCALE, kv_scale=c.scale)
        b = mla.decode_paged_window(q, qr, c.kv, c.table, n, 2 ** 31 - 1, 0, SCALE, kv_scale=c.scale)
        assert (a.double() - b.double()).abs().max() <= 0.02 * b.double().abs().max()


def test_prompts_and_fp8_trees_in_graphs():
    """Captured once, replayed on changing inputs and lengths beside eager calls: a prompt whose keys are cut into chunks, a tree over an fp8 cache."""
    T, L = 5, 3000
    _, c8, (q, qr), mask, lens = run_tree("fp8", [L, 40], T, 28)
    ws = torch.empty(max(256, mla.decode_tree_workspace_bytes(2, T, 28, 512, c8.table.shape[1] * 64)), dtype=torch.uint8, device=DEV)
    o8 = torch.empty_like(q)
    _, _, (qn, pr, UK, UV), c, n = run_prefill([L], 70, 3, 2500, 4, 256)
    wp = torch.empty(mla.prefill_window_workspace_bytes(1, 70, 3, 256, c.table.shape[1], 2500, 4), dtype=torch.uint8, device=DEV)
    op, lp = torch.empty_like(qn), torch.empty((1, 70, 3), device=DEV)
    tree = lambda o: mla.decode_paged_tree(q, qr, c8.kv, c8.table, lens, mask, SCALE, kv_scale=c8.scale, workspace=ws, out=o)
    prompt = lambda o, l: mla.prefill_window(qn, pr, UK, UV, c.kv, c.table, n, 2500, 4, SCALE, workspace=wp, out=o, lse=l)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        tree(o8), prompt(op, lp)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tree(o8), prompt(op, lp)
    for step in range(4):
        q.copy_(queries(2, T, 28, 512, 64, BF, 70 + step)[0])
        qn.copy_(torch.randn(qn.shape, generator=gen(step), device=DEV))
        lens.copy_(torch.tensor([L - 131 * step, 40 - step], dtype=torch.int32))
        n.fill_(L - 67 * step)
        graph.replay()
        a, b, l = tree(torch.empty_like(q)), torch.empty_like(qn), torch.empty_like(lp)
        prompt(b, l)
        torch.cuda.synchronize()
        # (bits: lengths that shrink meet rows that were given back and hold NaN)
        assert torch.equal(a.view(torch.int16), o8.view(torch.int16)), step
        assert torch.equal(b.view(torch.int16), op.view(torch.int16)) and torch.equal(l.view(torch.int32), lp.view(torch.int32)), step


def test_a_workspace_of_what_the_calls_own_kernel_needs():
    """The size is asked for without the types: a call on the matrix cores in one chunk takes any workspace."""
    q, ws, tree, window = prepared("bf16", 2, 28, (150,))
    assert ws.numel() > 256               # (the portable kernel would cut the sequences)
    for call in (tree, window):
        ref, small = call(workspace=ws), torch.empty(256, dtype=torch.uint8, device=DEV)
        assert torch.equal(call(workspace=small), ref) and torch.equal(call(workspace=small, out=torch.empty_like(q)), ref)
