"""The norm's and AdamW's instances for calls that go past the caches: separately compiled kernels with non-temporal accesses, taken from 96 MB (norm, bf16) and 160 MB (AdamW; with copies
of that size for the copies too) on.  Every element is its row's or its tensor's business alone, so that each result has to have the bits that the same rows or tensors get
in smaller calls, by the instances that the other tests hold against float64; dgamma, a sum over all rows, is held against float64 here."""
import pytest
import torch

from paper_1709_05011_amd import larsconv as lc

import gpu_util as gu

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
ELEMENTS = 17_500_000                  # of a norm's tensor: 105 MB of what the gradient moves without dtotal, 122 MB and 140 MB of the forward pass
# whole waves of 1024 and of 512 columns, columns by eights, odd ones; sixteen columns a thread in the gradient (over 8192); several rows of a wave (under 257) with 8, 16, 32 lanes each
WIDTHS = [1024, 4096, 512, 1536, 4104, 520, 480, 5001, 517, 301, 12288, 9728, 12296, 12289, 64, 40, 39, 128, 100, 101, 256, 200, 201]


def wide(rows, c, seed, pad=0, offset=0):
    """bf16 rows c + pad elements apart, `offset` elements past an aligned address."""
    whole = torch.randn(rows * (c + pad) + offset, generator=torch.Generator(device=gu.DEV).manual_seed(seed), device=gu.DEV, dtype=torch.bfloat16)
    return whole[offset:].view(rows, c + pad)[:, :c]


def pieces(rows):
    """Thirds of the rows (under 96 MB each), more than 256 rows each where a row is narrow."""
    cut = [0, rows // 3, 2 * rows // 3, rows]
    return list(zip(cut, cut[1:]))


@pytest.mark.parametrize("c", WIDTHS)
@pytest.mark.parametrize("pad,offset", [(0, 0), (3, 1)])
def test_norm(c, pad, offset):
    rows = ELEMENTS // c + 1
    x, r = wide(rows, c, 1, pad, offset), wide(rows, c, 2, 2 * pad, offset)
    gamma = 1 + 0.3 * torch.randn(c, generator=torch.Generator(device=gu.DEV).manual_seed(3), device=gu.DEV)
    groups = -(-c // 128)

    def run(parts):
        out = {k: gu.guarded(shape, t, offset=offset * torch.empty((), dtype=t).element_size()) for k, shape, t in
               [("total", (rows, c), torch.bfloat16), ("y", (rows, c), torch.bfloat16), ("rstd", (rows,), torch.float32), ("total8", (rows, c), torch.bfloat16),
                ("codes", (rows, c), torch.float8_e4m3fn), ("scales", (rows, groups), torch.float32), ("codes1", (rows, c), torch.float8_e4m3fn), ("scales1", (rows,), torch.float32)]}
        o = {k: v for k, (v, _) in out.items()}
        for a, b in parts:
            d = lc.RmsNormDesc(b - a, c, x_ld=c + pad, residual_ld=c + 2 * pad, dtype=lc.LC_BF16)
            lc.rmsnorm_fwd(d, x[a:b], r[a:b], gamma, o["total"][a:b], o["y"][a:b], o["rstd"][a:b])
            lc.rmsnorm_fwd_q8(d, x[a:b], r[a:b], gamma, o["total8"][a:b], o["codes"][a:b], o["scales"][a:b], 128)
            lc.rmsnorm_fwd_q8(d, x[a:b], r[a:b], gamma, o["total8"][a:b], o["codes1"][a:b], o["scales1"][a:b], 0)
        torch.cuda.synchronize()
        for _, check in out.values():
            check()
        return o

    got, want = run([(0, rows)]), run(pieces(rows))
    for k in got:
        assert torch.equal(got[k].view(torch.uint8 if "codes" in k else got[k].dtype), want[k].view(torch.uint8 if "codes" in k else want[k].dtype)), k


@pytest.mark.parametrize("c", WIDTHS)
@pytest.mark.parametrize("joined,pad,offset", [(True, 0, 0), (False, 0, 0), (True, 3, 1)])
def test_norm_gradient(c, joined, pad, offset):
    rows = ELEMENTS // c + 1
    h, dy, dt = wide(rows, c, 4, pad, offset), wide(rows, c, 5, 0, offset), wide(rows, c, 6, 0, offset) if joined else None
    gamma = 1 + 0.3 * torch.randn(c, generator=torch.Generator(device=gu.DEV).manual_seed(7), device=gu.DEV)
    rstd = torch.rand(rows, generator=torch.Generator(device=gu.DEV).manual_seed(8), device=gu.DEV) + 0.5

    def run(parts):
        (dx, check_x), (dg, check_g) = gu.guarded((rows, c), torch.bfloat16, offset=2 * offset), gu.guarded((c,), torch.float32)
        for a, b in parts:
            d = lc.RmsNormDesc(b - a, c, dtype=lc.LC_BF16)
            lc.rmsnorm_bwd(d, h[a:b], dy[a:b], dt[a:b] if joined else None, gamma, rstd[a:b], dx[a:b], dg, gu.workspace(lc.rmsnorm_bwd_workspace_bytes(d)), h_ld=c + pad)
        torch.cuda.synchronize()
        check_x()
        check_g()
        return dx, dg

    (dx, dg), (want, _) = run([(0, rows)]), run(pieces(rows))
    assert torch.equal(dx, want)
    exact, size = torch.zeros(c, dtype=torch.float64, device=gu.DEV), torch.zeros(c, dtype=torch.float64, device=gu.DEV)
    for a, b in pieces(rows):
        term = dy[a:b].double() * h[a:b].double() * rstd[a:b, None].double()
        exact += term.sum(0)
        size += term.abs().sum(0)
    assert bool(((dg.double() - exact).abs() <= (rows + 64) * U * size).all())


MILLION4 = 1 << 22
# 16 million elements: past the caches but for bf16 copies; 88 million: these too
LISTS = {"16 million": [MILLION4 + 3, 5, MILLION4 + 256, 0, MILLION4 + 1, 300, MILLION4 - 77], "88 million": [MILLION4 + 64 * i + i % 3 for i in range(21)] + [1000, 1]}


@pytest.mark.parametrize("sizes", LISTS)
@pytest.mark.parametrize("q8", [False, True])
@pytest.mark.parametrize("g_type", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offset", [0, 1])
def test_adamw(sizes, q8, g_type, offset):
    sizes, lead = LISTS[sizes], 256

    def tensors(t, fill, seed):
        """A tensor of each size, `offset` elements past a line of 128 bytes, and what lies around each."""
        gen, out = torch.Generator(device=gu.DEV).manual_seed(seed), []
        for n in sizes:
            whole = torch.full((n + 2 * lead + offset,), 7, dtype=t, device=gu.DEV)
            inner = whole[lead + offset:lead + offset + n]
            if fill == "normal":
                inner.copy_(torch.randn(n, generator=gen, device=gu.DEV) * 0.02)
            else:
                inner.fill_(fill)
            out.append((whole, inner))
        return out

    def run(together):
        state = torch.uint8 if q8 else torch.float32
        made = [tensors(torch.float32, "normal", 1), tensors(g_type, "normal", 2), tensors(state, 0, 3), tensors(state, 0, 4), tensors(torch.bfloat16, 0.0, 5)]
        w, g, m, v, low = ([i for _, i in x] for x in made)
        sm, sv = ([torch.ones(-(-n // 256), device=gu.DEV) for n in sizes] for _ in range(2))
        kind = lc.LC_BF16 if g_type == torch.bfloat16 else lc.LC_F32
        for step in (1, 2):
            for at in ([range(len(sizes))] if together else [[i] for i in range(len(sizes))]):
                pick = lambda a: [a[i] for i in at]
                if q8:
                    lc.adamw_step_q8(lc.AdamWQ8Args(pick(w), pick(g), pick(m), pick(sm), pick(v), pick(sv), w_lowp=pick(low), g_dtype=kind), 1e-3, 0.9, 0.99, 1e-8, 0.1, step, step)
                else:
                    lc.adamw_step(lc.AdamWArgs(pick(w), pick(g), pick(m), pick(v), w_lowp=pick(low), g_dtype=kind), 1e-3, 0.9, 0.99, 1e-8, 0.1, step)
        torch.cuda.synchronize()
        return [whole for x in made for whole, _ in x] + sm + sv, w

    got, w = run(True)
    want, _ = run(False)
    assert all(torch.equal(a, b) for a, b in zip(got, want))              # (what lies around the tensors among it)
    assert all(bool((x[:lead + offset] == 7).all()) and bool((x[-lead:] == 7).all()) for x in got[:5 * len(sizes)])
    assert all(t.isfinite().all() for t in w)
