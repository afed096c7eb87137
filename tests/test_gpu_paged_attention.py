"""gr4ad_op_paged_attention against the definition in 64 bits, computed sequence by sequence on the CPU: types, head layouts, page sizes, lengths from one
token to long ones, windows, empty and inconsistent sequences, page numbers that do not exist, and values that no row may see."""
import math

import pytest
import torch

from paper_2602_22732_amd import binding
from test_gpu_canary import Guarded

pytestmark = pytest.mark.gpu

TD = {"f32": torch.float32, "bf16": torch.bfloat16}


class Case:
    """A cache and a batch on the CPU: sequences of `lens` tokens whose last `new` are new; every slot that belongs to no sequence holds `stale`."""

    def __init__(self, dtype, dh, H, H_kv, page, new, lens, seed=0, lead=0, tail=0, stale=float("nan"), extra_pages=2):
        g = torch.Generator().manual_seed(seed)
        td, B = TD[dtype], len(new)
        self.dtype, self.dh, self.H, self.H_kv, self.page, self.new, self.lens = td, dh, H, H_kv, page, new, lens
        per = [max(1, -(-n // page)) for n in lens]
        self.n_pages, self.max_pages = sum(per) + extra_pages, max(per)
        ids = torch.randperm(self.n_pages, generator=g).to(torch.int32)
        self.table = torch.full((B, self.max_pages), -7, dtype=torch.int32)
        at = 0
        for b, n in enumerate(per):
            self.table[b, :n] = ids[at:at + n]
            at += n
        starts = [lead]
        for m in new:
            starts.append(starts[-1] + m)
        self.starts, self.N = starts, starts[-1] + tail
        self.q = torch.randn(self.N, H, dh, generator=g).to(td)
        self.k_new = torch.randn(self.N, H_kv, dh, generator=g).to(td)
        self.v_new = torch.randn(self.N, H_kv, dh, generator=g).to(td)
        self.k = torch.full((self.n_pages, H_kv, page, dh), stale, dtype=td)
        self.v = torch.full((self.n_pages, H_kv, dh, page), stale, dtype=td)
        for b, n in enumerate(lens):
            for j in range(max(0, n - new[b])):
                pg, s = int(self.table[b, j // page]), j % page
                self.k[pg, :, s] = torch.randn(H_kv, dh, generator=g).to(td)
                self.v[pg, :, :, s] = torch.randn(H_kv, dh, generator=g).to(td)

    def after(self):
        """The pages with the new tokens in them."""
        k, v = self.k.clone(), self.v.clone()
        for b, n in enumerate(self.lens):
            for i in range(self.new[b]):
                j = n - self.new[b] + i
                if j < 0:
                    continue
                pg, s, row = int(self.table[b, j // self.page]), j % self.page, self.starts[b] + i
                if 0 <= pg < self.n_pages:
                    k[pg, :, s], v[pg, :, :, s] = self.k_new[row], self.v_new[row]
        return k, v

    def expected(self, window=0, sinks=0, scale=None):
        """(result, tolerance) in 64 bits; rows in no sequence: NaN."""
        scale = self.dh ** -0.5 if scale is None else scale
        k_all, v_all = self.after()
        group = self.H // self.H_kv
        out = torch.full((self.N, self.H, self.dh), float("nan"), dtype=torch.float64)
        tol = torch.zeros_like(out)
        half = torch.finfo(self.dtype).eps / 2
        for b, n in enumerate(self.lens):
            for i in range(self.new[b]):
                p, row = n - self.new[b] + i, self.starts[b] + i
                js = [j for j in range(p + 1) if not window or p - j < window or j < sinks]
                js = [j for j in js if 0 <= int(self.table[b, j // self.page]) < self.n_pages]
                if not js:
                    out[row] = 0.0
                    continue
                j = torch.tensor(js)
                pg, s = self.table[b, j // self.page].long(), j % self.page
                k = k_all[pg, :, s].double().repeat_interleave(group, 1)      # [keys, H, dh]
                v = v_all[pg, :, :, s].double().repeat_interleave(group, 1)
                q = self.q[row].double()[None]
                x = (q * k).sum(-1) * scale
                w = torch.softmax(x, 0)[..., None]
                out[row] = (w * v).sum(0)
                mag = (w * v.abs()).sum(0)
                # float32: a score is off by at most (dh + 4) 2^-24 of its terms' magnitudes, its weight by twice that relative to the others, and sums of n
                # terms by n 2^-24; bf16 adds one rounding of every weight and one of the result (2^-8 each)
                score = (dh_terms(self.dh) * 2.0 ** -24) * ((q * k).abs().sum(-1) * scale).amax(0)
                f32 = (2 * score[:, None] + (len(js) + 16) * 2.0 ** -24) * mag
                tol[row] = f32 + (half * (mag + out[row].abs()) if self.dtype == torch.bfloat16 else half * out[row].abs())
        return out, tol


def dh_terms(dh):
    return dh + 8  # the products' sum, the scale, the base-2 exponent and the exponential


def run(c, window=0, sinks=0, append=True, **kw):
    dev = lambda t: t.cuda()  # noqa: E731
    k, v = c.after() if not append else (c.k, c.v)
    kd, vd = dev(k), dev(v)
    out = torch.full((c.N, c.H, c.dh), 7.0, dtype=c.dtype, device="cuda")
    got = binding.op_paged_attention(dev(c.q), kd, vd, dev(c.table), torch.tensor(c.starts, dtype=torch.int32).cuda(), torch.tensor(c.lens, dtype=torch.int32).cuda(),
                                     k_new=dev(c.k_new) if append else None, v_new=dev(c.v_new) if append else None, window=window, sinks=sinks, out=out, **kw)
    torch.cuda.synchronize()
    assert got is out
    return out.cpu(), kd.cpu(), vd.cpu()


def same(a, b):
    return torch.equal(a.view(torch.int16 if a.dtype == torch.bfloat16 else torch.int32), b.view(torch.int16 if b.dtype == torch.bfloat16 else torch.int32))


def check(c, window=0, sinks=0, append=True):
    want, tol = c.expected(window, sinks)
    got, k, v = run(c, window, sinks, append)
    inside = ~torch.isnan(want[:, 0, 0])
    lone = [r for r in range(c.N) if not any(c.starts[b] <= r < c.starts[b + 1] for b in range(len(c.lens)))]
    assert (got[lone] == 7.0).all(), "rows in no sequence were written"
    x = got.double()[inside]
    assert torch.isfinite(x).all()
    far = (x - want[inside]).abs() - tol[inside]
    assert (far <= 1e-30).all(), float(far.max())
    ka, va = c.after()
    assert same(k, ka) and same(v, va), "the pages differ from the definition"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh,H,H_kv,page", [(16, 4, 4, 16), (32, 6, 2, 64), (64, 8, 1, 16), (128, 4, 2, 32), (64, 5, 1, 256), (128, 40, 2, 128)])
def test_ragged_batches(dtype, dh, H, H_kv, page):
    check(Case(dtype, dh, H, H_kv, page, new=[1, 0, 3, 17, 1, 40], lens=[1, 9, 3, 50, 131, 300], seed=dh + H))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (5, 1), (16, 4), (33, 64), (100, 0), (2147483647, 7)])
def test_window_and_first_tokens(dtype, window, sinks):
    c = Case(dtype, 64, 4, 2, 16, new=[1, 20, 70, 5], lens=[300, 257, 70, 5], seed=3)
    check(c, window, sinks)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("new,lens", [([1], [1]), ([1], [2049]), ([2], [5003]), ([200], [200]), ([130], [1500]), ([1, 1, 1], [4097, 1, 16])])
def test_lengths(dtype, new, lens):
    check(Case(dtype, 128, 8, 2, 64, new, lens, seed=len(lens) + lens[0]))
    check(Case(dtype, 32, 2, 2, 16, new, lens, seed=lens[0]), window=700, sinks=3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_without_new_tokens_in_hand(dtype):
    check(Case(dtype, 64, 4, 4, 32, new=[4, 1], lens=[90, 33], seed=5), append=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_outside_sequences_and_inconsistent_lengths(dtype):
    # rows before the first and behind the last sequence stay; a sequence shorter than its new tokens: those at negative positions are zero
    check(Case(dtype, 64, 4, 2, 16, new=[3, 8, 2], lens=[40, 5, 0], seed=6, lead=2, tail=5))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_page_numbers_that_do_not_exist(dtype):
    c = Case(dtype, 64, 4, 2, 16, new=[1, 20, 1], lens=[70, 100, 10], seed=7)
    c.table[0, 1], c.table[1, 5], c.table[1, 2], c.table[2, 0] = -1, c.n_pages, 2 ** 31 - 1, -2 ** 31
    check(c)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("poison", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("single", [True, False])
def test_what_a_row_does_not_see_never_reaches_it(dtype, poison, single):
    # a later new token, and a token that left the window, hold values that are no numbers
    if single:
        c = Case(dtype, 128, 4, 2, 16, new=[1], lens=[200], seed=8)
        c.k[c.table[0, 3].long(), :, 4], c.v[c.table[0, 3].long(), :, :, 4] = poison, poison
        check(c, window=60, sinks=2)
        return
    c = Case(dtype, 64, 4, 2, 16, new=[40], lens=[100], seed=9)
    c.k_new[30], c.v_new[30] = poison, poison
    want, tol = c.expected()
    got, _, _ = run(c)
    assert torch.isfinite(want[:30]).all() and ((got.double()[:30] - want[:30]).abs() <= tol[:30]).all()
    assert torch.isnan(got[30:]).any(dim=2).all()


def test_scores_of_large_magnitude():
    c = Case("f32", 64, 2, 1, 16, new=[30], lens=[90], seed=10)
    c.q, c.k, c.k_new = c.q * 30, c.k * 4, c.k_new * 4
    check(c)
    check(c, window=20)


def test_strided_rows_and_scale():
    c = Case("bf16", 64, 4, 2, 32, new=[9, 1, 30], lens=[40, 77, 30], seed=11)
    qkv = torch.full((c.N, 4 * 64 + 2 * 2 * 64 + 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    q, k_new, v_new = qkv[:, :256].view(c.N, 4, 64), qkv[:, 256:384].view(c.N, 2, 64), qkv[:, 384:512].view(c.N, 2, 64)
    q.copy_(c.q)
    k_new.copy_(c.k_new)
    v_new.copy_(c.v_new)
    args = (c.table.cuda(), torch.tensor(c.starts, dtype=torch.int32).cuda(), torch.tensor(c.lens, dtype=torch.int32).cuda())
    got = binding.op_paged_attention(q, c.k.cuda(), c.v.cuda(), *args, k_new=k_new, v_new=v_new, scale=0.3)
    want, tol = c.expected(scale=0.3)
    assert ((got.cpu().double() - want).abs() <= tol).all()


def test_pages_behind_four_gigabytes():
    page, H_kv, dh = 64, 8, 128
    n_pages = (1 << 31) // (page * H_kv * dh) + 40       # 2^31 values and more in each array
    k = torch.empty(n_pages, H_kv, page, dh, dtype=torch.bfloat16, device="cuda")
    v = torch.empty(n_pages, H_kv, dh, page, dtype=torch.bfloat16, device="cuda")
    small = Case("bf16", dh, 16, H_kv, page, new=[1, 30], lens=[700, 30], seed=12)
    table = small.table.clone()
    for i in range(small.n_pages):
        at = n_pages - 1 - i
        k[at], v[at] = small.k[i].cuda(), small.v[i].cuda()
        table[small.table == i] = at
    got = binding.op_paged_attention(small.q.cuda(), k, v, table.cuda(), torch.tensor(small.starts, dtype=torch.int32).cuda(), torch.tensor(small.lens, dtype=torch.int32).cuda(),
                                     k_new=small.k_new.cuda(), v_new=small.v_new.cuda())
    want, tol = small.expected()
    assert ((got.cpu().double() - want).abs() <= tol).all()
    ka, _ = small.after()
    pg = int(small.table[0, 699 // page])
    assert same(k[n_pages - 1 - pg].cpu(), ka[pg])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_writes_nothing_outside_its_buffers(dtype):
    c = Case(dtype, 64, 8, 2, 16, new=[1, 37, 1], lens=[900, 37, 1], seed=13, stale=0.5)
    L, e = binding.lib(), 2 if dtype == "bf16" else 4
    gk, gv, go = Guarded(c.k.numel() * e), Guarded(c.v.numel() * e), Guarded(c.q.numel() * e)
    k, v, out = gk.typed(c.dtype, c.k.shape), gv.typed(c.dtype, c.v.shape), go.typed(c.dtype, c.q.shape)
    k.copy_(c.k)
    v.copy_(c.v)
    import ctypes as C
    cache = binding.PagedCacheDesc(k.data_ptr(), v.data_ptr(), 16, c.n_pages, c.page, c.max_pages, c.H_kv, c.dh)
    gw = Guarded(max(256, int(L.gr4ad_op_paged_attention_workspace_bytes(binding.dtype_code(c.dtype), C.byref(cache), 3, c.N, c.H, 0, 0))))
    gt, gs, gl = Guarded(c.table.numel() * 4), Guarded(16), Guarded(12)
    table, starts, lens = gt.typed(torch.int32, c.table.shape), gs.typed(torch.int32, (4,)), gl.typed(torch.int32, (3,))
    table.copy_(c.table)
    starts.copy_(torch.tensor(c.starts))
    lens.copy_(torch.tensor(c.lens))
    binding.op_paged_attention(c.q.cuda(), k, v, table, starts, lens, k_new=c.k_new.cuda(), v_new=c.v_new.cuda(), out=out, workspace=gw.view)
    torch.cuda.synchronize()
    for g in (gk, gv, go, gw, gt, gs, gl):
        assert g.intact()
    want, tol = c.expected()
    assert ((out.cpu().double() - want).abs() <= tol).all()


def test_two_graphs_that_share_a_workspace_and_another_stream():
    cases = [Case("bf16", 128, 8, 2, 64, new=[1, 1], lens=[3000, 777], seed=14), Case("bf16", 128, 8, 2, 64, new=[60, 1], lens=[500, 64], seed=15)]
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    side, graphs, outs = torch.cuda.Stream(), [], []
    for c in cases:
        args = [t.cuda() for t in (c.q, c.k, c.v, c.table, torch.tensor(c.starts, dtype=torch.int32), torch.tensor(c.lens, dtype=torch.int32))]
        new = dict(k_new=c.k_new.cuda(), v_new=c.v_new.cuda())
        out = torch.empty_like(args[0])
        torch.cuda.synchronize()
        binding.op_paged_attention(*args, **new, out=out, workspace=ws, stream=side)
        torch.cuda.synchronize()
        want, tol = c.expected()
        assert ((out.cpu().double() - want).abs() <= tol).all()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            binding.op_paged_attention(*args, **new, out=out, workspace=ws)
        graphs.append((graph, args, new))
        outs.append((out, out.clone()))
    for _ in range(4):
        for (graph, args, new), (out, eager) in zip(graphs, outs):
            out.zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert same(out, eager)
            again = binding.op_paged_attention(*args, **new)
            torch.cuda.synchronize()
            assert same(again, eager)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_more_sequences_than_a_wavefront_counts_at_once(dtype):
    new = [1] * 70 + [0, 5] + [1] * 60 + [33]
    check(Case(dtype, 64, 4, 1, 16, new=new, lens=[max(m, 1 + 7 * i % 90) for i, m in enumerate(new)], seed=16))


@pytest.mark.parametrize("dh,H,H_kv,page", [(32, 4, 2, 16), (64, 8, 2, 64), (128, 8, 2, 32), (128, 16, 2, 128)])
def test_long_chunks(dh, H, H_kv, page):
    # tiles of 256 rows, of 128, several of them, under a window and without
    for new, lens in (([300, 40], [1000, 41]), ([100], [700])):
        c = Case("bf16", dh, H, H_kv, page, new, lens, seed=dh + H)
        check(c)
        check(c, window=150, sinks=9)


def test_a_captured_long_chunk_and_values_that_are_no_numbers_in_it():
    c = Case("bf16", 128, 16, 2, 64, new=[300], lens=[900], seed=17)
    c.v_new[250] = float("inf")
    want, tol = c.expected()
    args = [t.cuda() for t in (c.q, c.k, c.v, c.table, torch.tensor(c.starts, dtype=torch.int32), torch.tensor(c.lens, dtype=torch.int32))]
    new = dict(k_new=c.k_new.cuda(), v_new=c.v_new.cuda())
    eager = binding.op_paged_attention(*args, **new)
    torch.cuda.synchronize()
    assert ((eager.cpu().double()[:250] - want[:250]).abs() <= tol[:250]).all()
    assert (eager[250:] == float("inf")).all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = binding.op_paged_attention(*args, **new)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert same(out, eager)


@pytest.mark.parametrize("dtype,dh,H,H_kv,page", [("bf16", 64, 4, 1, 64), ("bf16", 128, 8, 1, 16), ("bf16", 16, 2, 2, 256), ("f32", 128, 2, 1, 32), ("f32", 32, 4, 2, 1024), ("f32", 16, 3, 1, 64)])
def test_keys_shared_by_workgroups(dtype, dh, H, H_kv, page):
    # up to 20 stretches of keys for a tile, most of which short sequences leave empty
    c = Case(dtype, dh, H, H_kv, page, new=[1, 2, 1, 0, 3], lens=[5000, 2, 1300, 900, 2600], seed=dh)
    check(c)
    check(c, window=2000, sinks=3)


def test_a_long_chunk_whose_keys_workgroups_share():
    c = Case("bf16", 64, 2, 1, 64, new=[70, 0, 9], lens=[6000, 40, 2100], seed=18)
    c.table[0, 20], c.table[2, 3] = -1, c.n_pages
    check(c)
    check(c, window=1500, sinks=100)


def test_two_streams_at_once():
    cases = [Case("bf16", 64, 4, 1, 64, new=[1, 1, 20], lens=[3000, 40, 400], seed=19), Case("f32", 32, 4, 2, 16, new=[2, 1], lens=[100, 2500], seed=20)]
    streams = [torch.cuda.Stream() for _ in cases]
    on_gpu = [[t.cuda() for t in (c.q, c.k, c.v, c.table, torch.tensor(c.starts, dtype=torch.int32), torch.tensor(c.lens, dtype=torch.int32), c.k_new, c.v_new)] for c in cases]
    torch.cuda.synchronize()
    outs = [[] for _ in cases]
    for _ in range(4):
        for i, args in enumerate(on_gpu):
            with torch.cuda.stream(streams[i]):
                outs[i].append(binding.op_paged_attention(*args))
    torch.cuda.synchronize()
    for c, got in zip(cases, outs):
        want, tol = c.expected()
        assert all(same(g, got[0]) for g in got)
        assert ((got[0].cpu().double() - want).abs() <= tol).all()


@pytest.mark.parametrize("dh,page", [(128, 16), (128, 64), (64, 16)])
def test_float32_chunks(dh, page):
    c = Case("f32", dh, 8, 2, page, new=[60, 1, 17, 0, 3], lens=[500, 200, 17, 30, 1400], seed=21)
    check(c)
    check(c, window=90, sinks=5)


@pytest.mark.parametrize("dh,H,H_kv,page", [(32, 4, 2, 16), (32, 2, 1, 128), (64, 4, 1, 16), (128, 4, 1, 64)])
def test_chunks_among_finite_values(dh, H, H_kv, page):
    # no value anywhere is a NaN, and what the compute units' local memory holds from before is finite too: a tile that was not loaded shows as a wrong result
    assert torch.isfinite(run(Case("bf16", 128, 8, 1, 64, new=[300] * 40, lens=[320] * 40, seed=22, stale=0.25), 0, 0, True)[0].float()).all()
    c = Case("bf16", dh, H, H_kv, page, new=[300, 40], lens=[1000, 41], seed=23, stale=0.25)
    check(c)
    check(c, window=300, sinks=3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh,H,H_kv,page", [(16, 4, 2, 16), (32, 4, 1, 32), (64, 6, 1, 64), (128, 8, 2, 16), (128, 8, 1, 1024)])
@pytest.mark.parametrize("new,lens", [([1, 1, 2], [1, 700, 90]), ([1, 1], [40, 3000]), ([30, 9], [400, 9]), ([90, 60, 1], [90, 800, 33])])
def test_all_kinds_among_finite_values(dtype, dh, H, H_kv, page, new, lens):
    # with the test above: no tile may be right only because a NaN sent its rows to the plain form
    c = Case(dtype, dh, H, H_kv, page, new=new, lens=lens, seed=24, stale=0.25)
    check(c)
    check(c, window=60, sinks=2)
