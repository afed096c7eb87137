"""gr4ad_op_adjust_logits and its half-precision form against their definition in 64 bits, rule by rule and together, and a whole step through the operators in
front of the selection."""
import pytest
import torch

from paper_2602_22732_amd import binding
from test_gpu_canary import Guarded

pytestmark = pytest.mark.gpu


def definition(x, r):
    x = x.double().clone()
    rows, V = x.shape
    mag = x.abs()
    for i in range(rows):
        h = r.get("history")
        if h is not None:
            n = h.shape[1] if r.get("history_len") is None else min(max(int(r["history_len"][i]), 0), h.shape[1])
            h = h[i, :n].long()
            c = torch.bincount(h[(h >= 0) & (h < V)], minlength=V).double()
            seen = c > 0
            if r.get("repetition") is not None:
                f = float(r["repetition"][i])
                x[i] = torch.where(seen, torch.where(x[i] > 0, x[i] / f, x[i] * f), x[i])
            fr = 0.0 if r.get("frequency") is None else float(r["frequency"][i])
            pr = 0.0 if r.get("presence") is None else float(r["presence"][i])
            x[i] -= fr * c + pr * seen
            mag[i] = torch.maximum(mag[i], x[i].abs()) + abs(fr) * c + abs(pr)
        if r.get("bias") is not None:
            b = 0 if r.get("bias_row") is None else int(r["bias_row"][i])
            if 0 <= b < r["bias"].shape[0]:
                x[i] += r["bias"][b].double()
                mag[i] += r["bias"][b].double().abs()
        if r.get("mask") is not None:
            m = 0 if r.get("mask_row") is None else int(r["mask_row"][i])
            if m >= r["mask"].shape[0]:
                x[i] = -float("inf")
            elif m >= 0:
                v = torch.arange(V)
                x[i][((r["mask"][m][v // 32].long() >> (v % 32)) & 1) == 0] = -float("inf")
    return x, mag


def rules(g, rows, V, names):
    r = {}
    ints = lambda lo, hi, *s: torch.randint(lo, hi, s, generator=g, dtype=torch.int32)  # noqa: E731
    if "history" in names:
        r["history"] = ints(-2, V + 2, rows, 70)              # entries outside the vocabulary among them
        r["history"][:, ::3] = r["history"][:, :1]            # repeats
        r["history_len"] = ints(-1, 75, rows)
        r["frequency"], r["presence"], r["repetition"] = torch.rand(rows, generator=g), torch.rand(rows, generator=g) - 0.5, 1 + torch.rand(rows, generator=g)
    if "bias" in names:
        r["bias"], r["bias_row"] = torch.randn(3, V, generator=g), ints(-1, 4, rows)
    if "mask" in names:
        r["mask"] = ints(-2 ** 31, 2 ** 31 - 1, 4, -(-V // 32))
        r["mask"][1] = 0
        r["mask_row"] = ints(-1, 6, rows)
    return r


def check(x, r, out=None):
    got = binding.op_adjust_logits(x.cuda(), **{k: v.cuda() for k, v in r.items() if v is not None}, out=out)
    want, mag = definition(x, r)
    got = got.cpu().double()
    gone = torch.isinf(want) & (want < 0) & ~torch.isinf(x)
    assert (got[gone] == -float("inf")).all()
    fine = torch.isfinite(want)
    assert torch.isfinite(got[fine]).all()
    # four float32 operations of at most half a step each, then one rounding to the type (and half's smallest step)
    tol = mag * 6 * 2.0 ** -24 + (want.abs() * 2.0 ** -11 + 2.0 ** -25 if x.dtype == torch.float16 else 0.0)
    assert ((got - want).abs()[fine] <= tol[fine]).all()
    return got


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("rows,V", [(1, 1), (3, 7), (64, 1024), (5, 33), (2, 16384), (7, 8195), (1, 151936), (300, 257)])
@pytest.mark.parametrize("names", [(), ("history",), ("bias",), ("mask",), ("history", "bias", "mask")])
def test_rules(dtype, rows, V, names):
    g = torch.Generator().manual_seed(rows + V)
    x = (2 * torch.randn(rows, V, generator=g)).to(dtype)
    check(x, rules(g, rows, V, names))


@pytest.mark.parametrize("only", ["repetition", "presence", "frequency", None])
def test_single_penalties_and_defaults(only):
    g = torch.Generator().manual_seed(4)
    r = rules(g, 9, 500, ("history", "bias", "mask"))
    for k in ("repetition", "presence", "frequency"):
        if k != only:
            r[k] = None
    r["history_len"] = r["bias_row"] = r["mask_row"] = None   # the whole history; row 0 of the tables for everyone
    check(2 * torch.randn(9, 500, generator=g), r)


def test_in_place_and_values_that_are_no_numbers():
    g = torch.Generator().manual_seed(5)
    x = torch.randn(6, 100, generator=g)
    x[0, 3], x[1, 4], x[2, 5], x[3, 6] = float("nan"), float("inf"), -float("inf"), torch.finfo(torch.float32).min
    mask = torch.full((2, 4), -1, dtype=torch.int32)
    mask[1] = 0
    xd = x.cuda()
    got = binding.op_adjust_logits(xd, mask=mask.cuda(), mask_row=torch.zeros(6, dtype=torch.int32).cuda(), out=xd)
    assert got is xd
    assert torch.equal(xd.cpu().nan_to_num(7.0), x.nan_to_num(7.0))                    # allowed: as they are
    got = binding.op_adjust_logits(x.cuda(), mask=mask.cuda(), mask_row=torch.ones(6, dtype=torch.int32).cuda())
    assert (got == -float("inf")).all()                                              # forbidden: whatever they hold
    assert binding.op_adjust_logits(x.view(2, 3, 100).cuda()).shape == (2, 3, 100)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_writes_nothing_outside(dtype):
    for rows, V in [(3, 4097), (1, 5), (17, 640)]:
        go = Guarded(rows * V * dtype.itemsize)
        g = torch.Generator().manual_seed(V)
        check(torch.randn(rows, V, generator=g).to(dtype), rules(g, rows, V, ("history", "bias", "mask")), out=go.typed(dtype, (rows, V)))
        assert go.intact()


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_large_outputs_are_those_of_their_parts(dtype):
    # beyond the sizes from which results pass the caches and a thread takes two pieces
    g = torch.Generator().manual_seed(8)
    rows, V = 2100, 4104
    x, r = torch.randn(rows, V, generator=g).to(dtype).cuda(), {k: v.cuda() for k, v in rules(g, rows, V, ("history", "bias", "mask")).items()}
    got = binding.op_adjust_logits(x, **r)
    for a, b in ((0, 700), (700, 2100)):
        part = {k: v if k in ("bias", "mask") else v[a:b] for k, v in r.items()}
        assert torch.equal(got[a:b], binding.op_adjust_logits(x[a:b], **part))


def test_a_step_through_the_operators():
    """Attention over pages -> projection and classifier on FP8 blocks -> masks and penalties -> selection, captured and replayed: the selection keeps only
    allowed tokens and agrees with the definition on the logits it was given, and every replay with eager calls."""
    torch.manual_seed(6)
    B, n, H, dh, page, V, k = 3, 4, 8, 64, 16, 1024, 6
    d, rows = H * dh, 12                                             # n beams of every request are sequences of their own
    lens = torch.tensor([40 + 3 * i for i in range(rows)], dtype=torch.int32, device="cuda")
    table = torch.randperm(rows * 8, device="cuda").to(torch.int32).view(rows, 8)
    kp, vp = torch.randn(rows * 8, H, page, dh, device="cuda").bfloat16(), torch.randn(rows * 8, H, dh, page, device="cuda").bfloat16()
    start = torch.arange(rows + 1, dtype=torch.int32, device="cuda")
    wo, cls = [binding.op_quantize_blocks(torch.randn(m, d, device="cuda") / d ** 0.5, 128) for m in (d, V)]
    qkv = torch.randn(rows, 3 * d, device="cuda").bfloat16()
    cum = -torch.rand(B, n, device="cuda")
    mask = torch.randint(-2 ** 31, 2 ** 31 - 1, (5, V // 32), dtype=torch.int32, device="cuda")
    state = torch.arange(rows, dtype=torch.int32, device="cuda") % 5
    history = torch.randint(0, V, (rows, 9), dtype=torch.int32, device="cuda")
    rep = torch.full((rows,), 1.3, device="cuda")

    def step():
        q, kn, vn = (qkv[:, i * d:(i + 1) * d].view(rows, H, dh) for i in range(3))
        o = binding.op_paged_attention(q, kp, vp, table, start, lens, k_new=kn, v_new=vn, window=32, sinks=4)
        h = binding.op_linear_fp8_block(*binding.op_quantize_blocks(o.view(rows, d)), *wo)
        logits = binding.op_linear_fp8_block(*binding.op_quantize_blocks(h), *cls, out_dtype=torch.float16).view(B, n, V)
        final = binding.op_adjust_logits(logits, history=history, repetition=rep, mask=mask, mask_row=state)
        return (final,) + binding.op_select(final, cum, k)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for seed in range(4):
        qkv.copy_(torch.randn(rows, 3 * d, generator=torch.Generator().manual_seed(seed)))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        eager = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, eager))
        final, parent, tok, score = (t.cpu() for t in got)
        sc = (cum.cpu()[:, :, None].double() + torch.log_softmax(final.double(), dim=2)).view(B, n * V)
        best = torch.sort(sc, dim=1, descending=True)[0][:, :k]
        assert (sc.gather(1, (parent.long() * V + tok)) - score).abs().max() < 1e-4 and (best - score).abs().max() < 1e-4
        row = torch.arange(B)[:, None] * n + parent
        m = mask.cpu()[state.cpu().long()[row], (tok // 32).long()].long()
        assert ((m >> (tok % 32)) & 1 == 1).all()
