"""GPU parity of the products over groups of rows against products in 64 bits.

Tolerances: a result is a sum of `depth` products.  Summed in fp32 in any order it is off by at most depth 2^-24 sum |a||b|; operands
in three 8-bit parts leave out less than 3 * 2^-24 of every product, and an instruction's own sums of 8 to 32 products add a few roundings
more: (depth + 8) 2^-24 sum |a||b| in all.  It is then rounded once: half a step of its type, or of the type's smallest number."""
import numpy as np
import pytest

from paper_2112_09335_amd import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def solver():
    from paper_2112_09335_amd import binding
    s = binding.Solver(0)                         # no graph, model or workspace
    yield s
    s.close()


def types():
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
LEAST = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}


def close(got, want, magnitude, depth, kind):
    """got against the 64-bit result, magnitude = sum |a||b| of every entry."""
    got = got.detach().cpu().double().numpy()
    loose = (depth + 8) * 2.0 ** -24 * magnitude
    room = loose + HALF[kind] * (np.abs(want) + loose) + LEAST[kind]
    far = np.abs(got - want) - room
    assert np.isfinite(got).all()
    assert (far <= 0).all(), (far.max(), np.unravel_index(far.argmax(), far.shape), (np.abs(got - want) / np.maximum(room, 1e-300)).max())


def draw(torch, seed, sizes, K, width, kind, transposed=False, before=0, behind=0, scale=1.0):
    """Rows of `sizes` groups between `before` and `behind` rows of no group, as CPU tensors of the type."""
    rng = np.random.default_rng(seed)
    t = types()[kind]
    n = before + int(sum(sizes)) + behind
    A = torch.from_numpy(rng.standard_normal((n, K)).astype(np.float32) * scale).to(t)
    B = torch.from_numpy(rng.standard_normal((len(sizes), width, K) if transposed else (len(sizes), K, width)).astype(np.float32)).to(t)
    ptr = torch.from_numpy((before + np.concatenate([[0], np.cumsum(sizes)])).astype(np.int64))
    return A, B, ptr


def want_nn(A, B, ptr, transposed):
    A, B, ptr = A.double().numpy(), B.double().numpy(), ptr.numpy()
    out = np.zeros((A.shape[0], B.shape[1 if transposed else 2]))
    size = np.zeros_like(out)
    for g in range(len(ptr) - 1):
        lo, hi = ptr[g], ptr[g + 1]
        Bg = B[g].T if transposed else B[g]
        out[lo:hi], size[lo:hi] = A[lo:hi] @ Bg, np.abs(A[lo:hi]) @ np.abs(Bg)
    return out, size


def want_tn(A, G, ptr):
    A, G, ptr = A.double().numpy(), G.double().numpy(), ptr.numpy()
    out = np.zeros((len(ptr) - 1, A.shape[1], G.shape[1]))
    size = np.zeros_like(out)
    for g in range(len(ptr) - 1):
        lo, hi = ptr[g], ptr[g + 1]
        out[g], size[g] = A[lo:hi].T @ G[lo:hi], np.abs(A[lo:hi]).T @ np.abs(G[lo:hi])
    return out, size


SHAPES = [
    # groups' sizes, K, C
    ([1], 1, 1), ([1], 64, 64), ([3], 5, 2), ([0, 1, 0], 33, 17), ([0, 0], 8, 8), ([1] * 70, 40, 24), ([5, 0, 130, 1, 64], 97, 301),
    ([63, 64, 65], 64, 64), ([127, 128, 129, 0, 1], 128, 128), ([255, 256, 257], 256, 256), ([300, 5, 0, 700], 512, 320),
    ([31, 2, 16, 15, 17, 8], 1000, 72), ([40, 33], 2048, 130), ([1000], 16, 3), ([2, 1, 0, 4], 1024, 512), ([600, 900], 7, 260),
    ([1500, 20], 136, 136), ([513], 520, 264), ([16, 16, 1, 0, 3], 2048, 1024),
]


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("sizes,K,width", SHAPES, ids=lambda v: str(v).replace(" ", "")[:24])
def test_product_over_groups(solver, kind, transposed, sizes, K, width):
    import torch
    A, B, ptr = draw(torch, K + width, sizes, K, width, kind, transposed)
    out = solver.op_transform_grouped(A.cuda(), B.cuda(), ptr.cuda(), transposed=transposed)
    assert out.dtype == A.dtype and tuple(out.shape) == (A.shape[0], width)
    close(out, *want_nn(A, B, ptr, transposed), K, kind)


def on_gpu_nn(torch, A, B, ptr, transposed):
    """want_nn with its products in 64 bits on the GPU: for sizes that fill it."""
    out = torch.zeros((A.shape[0], B.shape[1 if transposed else 2]), dtype=torch.float64, device="cuda")
    size = torch.zeros_like(out)
    for g in range(ptr.shape[0] - 1):
        lo, hi = int(ptr[g]), int(ptr[g + 1])
        Bg = (B[g].T if transposed else B[g]).double().cuda().contiguous()
        Ag = A[lo:hi].double().cuda()
        out[lo:hi], size[lo:hi] = Ag @ Bg, Ag.abs() @ Bg.abs()
    return out.cpu().numpy(), size.cpu().numpy()


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("sizes,K,width", [([9000, 0, 17001, 5, 14000], 136, 392), ([20000, 30, 20000], 520, 264), ([33000], 72, 512), ([11000, 9001], 200, 301),
                                           ([1200] * 12, 1032, 640)], ids=lambda v: str(v).replace(" ", "")[:24])
def test_product_over_groups_that_fills_the_chip(solver, kind, transposed, sizes, K, width):
    import torch
    A, B, ptr = draw(torch, K + width, sizes, K, width, kind, transposed)
    out = solver.op_transform_grouped(A.cuda(), B.cuda(), ptr.cuda(), transposed=transposed)
    close(out, *on_gpu_nn(torch, A, B, ptr, transposed), K, kind)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("sizes,K,width", [([4000, 9000, 0, 1, 5010, 8000, 4000], 97, 301), ([25000, 15000], 136, 128), ([40] * 70, 264, 200), ([40] * 70, 261, 201),
                                           ([2] * 64, 264, 640), ([2] * 64, 261, 645)], ids=lambda v: str(v).replace(" ", "")[:24])
def test_product_over_groups_in_every_size_of_tiles(solver, kind, transposed, sizes, K, width):
    """As above: 128 x 128 with unaligned rows and with few columns, 64 x 64 and 32 x 64 without sets that share the contraction."""
    test_product_over_groups_that_fills_the_chip(solver, kind, transposed, sizes, K, width)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("sizes,K,width", [([30000, 0, 41000, 7], 264, 392), ([60000], 520, 520), ([40000, 20001], 301, 200), ([700] * 40, 1024, 1032)],
                         ids=lambda v: str(v).replace(" ", "")[:24])
def test_weight_gradient_over_groups_that_fills_the_chip(solver, kind, sizes, K, width):
    import torch
    A, _, ptr = draw(torch, K + width, sizes, K, 1, kind)
    G, _, _ = draw(torch, K + width + 1, sizes, width, 1, kind, scale=2.0 ** -5)
    want = torch.zeros((len(sizes), K, width), dtype=torch.float64, device="cuda")
    size = torch.zeros_like(want)
    for g in range(len(sizes)):
        lo, hi = int(ptr[g]), int(ptr[g + 1])
        a, b = A[lo:hi].double().T.contiguous().cuda(), G[lo:hi].double().cuda()
        want[g], size[g] = a @ b, a.abs() @ b.abs()
    out = solver.op_wgrad_grouped(A.cuda(), G.cuda(), ptr.cuda())
    close(out, want.cpu().numpy(), size.cpu().numpy(), max(sizes), "f32")
    assert torch.equal(out, solver.op_wgrad_grouped(A.cuda(), G.cuda(), ptr.cuda()))


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("sizes,K,width", [([25000] * 8, 64, 64), ([60000], 521, 523)], ids=lambda v: str(v).replace(" ", "")[:24])
def test_weight_gradient_over_groups_in_every_size_of_tiles(solver, kind, sizes, K, width):
    """As above: 64 x 64 without sets that share the contraction, 128 x 256 with unaligned rows."""
    test_weight_gradient_over_groups_that_fills_the_chip(solver, kind, sizes, K, width)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("sizes,K,width", [([25000] * 8, 64, 64), ([60000], 521, 523), ([30000, 0, 41000, 7], 264, 392), ([700] * 40, 1024, 1032), ([40000, 20001], 301, 200)],
                         ids=lambda v: str(v).replace(" ", "")[:24])
def test_weight_gradient_of_16_bits_is_the_rounded_one(solver, kind, sizes, K, width):
    """The sums are the same (tested against 64 bits above), rounded once at the end."""
    import torch
    A, _, ptr = (x.cuda() for x in draw(torch, K, sizes, K, 1, kind))
    G = draw(torch, K + 1, sizes, width, 1, kind, scale=2.0 ** -5)[0].cuda()
    assert torch.equal(solver.op_wgrad_grouped(A, G, ptr, out_dtype=types()[kind]), solver.op_wgrad_grouped(A, G, ptr).to(types()[kind]))


@pytest.mark.parametrize("kind,out_kind", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f32"), ("f16", "f16")])
@pytest.mark.parametrize("sizes,K,width", SHAPES + [([20000, 3, 9000], 64, 48), ([70000], 24, 5), ([4096, 4097], 256, 256), ([40000], 130, 130)],
                         ids=lambda v: str(v).replace(" ", "")[:24])
def test_weight_gradient_over_groups(solver, kind, out_kind, sizes, K, width):
    import torch
    A, _, ptr = draw(torch, K + width, sizes, K, 1, kind)
    G, _, _ = draw(torch, K + width + 1, sizes, width, 1, kind, scale=2.0 ** -5)
    out = solver.op_wgrad_grouped(A.cuda(), G.cuda(), ptr.cuda(), out_dtype=types()[out_kind])
    assert out.dtype == types()[out_kind]
    close(out, *want_tn(A, G, ptr), max(sizes), out_kind)
    again = solver.op_wgrad_grouped(A.cuda(), G.cuda(), ptr.cuda(), out_dtype=types()[out_kind])
    assert torch.equal(out, again)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("K,width,step_a,step_o,at", [(64, 64, 64, 64, 0), (64, 64, 72, 80, 8), (64, 64, 65, 67, 1), (97, 301, 99, 303, 3), (256, 136, 256, 136, 1)])
def test_strides_offsets_and_rows_of_no_group(solver, kind, transposed, K, width, step_a, step_o, at):
    """A and out are parts of wider matrices, at any element; rows before the first group and behind the last are neither read (they hold no
    numbers) nor written, and neither is anything between the rows."""
    import torch
    sizes = [70, 0, 33, 1, 150]
    A, B, ptr = draw(torch, 5, sizes, K, width, kind, transposed, before=9, behind=40)
    n = A.shape[0]
    A[:9], A[-40:] = float("nan"), float("inf")
    wide = torch.full((n * step_a + at + 8,), float("nan"), dtype=A.dtype, device="cuda")
    Av = torch.as_strided(wide, (n, K), (step_a, 1), at)
    Av.copy_(A)
    held = torch.full((n * step_o + at + 8,), 7.0, dtype=A.dtype, device="cuda")
    out = torch.as_strided(held, (n, width), (step_o, 1), at)
    Bw = torch.zeros(B.numel() + at, dtype=B.dtype, device="cuda")[at:].view(B.shape)
    Bw.copy_(B)
    solver.op_transform_grouped(Av, Bw, ptr.cuda(), transposed=transposed, out=out)
    want, size = want_nn(A, B, ptr, transposed)
    close(out[9:-40], want[9:-40], size[9:-40], K, kind)
    mask = torch.ones_like(held, dtype=torch.bool)
    torch.as_strided(mask, (n, width), (step_o, 1), at)[9:-40] = False
    assert (held[mask] == 7.0).all()
    G, _, _ = draw(torch, 6, sizes, width, 1, kind, before=9, behind=40)
    G[:9], G[-40:] = float("inf"), float("nan")
    Gv = torch.as_strided(torch.full((n * step_o + at + 8,), float("nan"), dtype=A.dtype, device="cuda"), (n, width), (step_o, 1), at)
    Gv.copy_(G)
    dB = torch.full((len(sizes) * K * width + at,), 7.0, device="cuda")
    solver.op_wgrad_grouped(Av, Gv, ptr.cuda(), out=dB[at:].view(len(sizes), K, width))
    close(dB[at:].view(len(sizes), K, width), *want_tn(A, G, ptr), 150, "f32")
    assert (dB[:at] == 7.0).all()


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("K,width", [(64, 64), (97, 41), (256, 256), (1024, 128)])
def test_what_is_not_finite_stays_in_its_row_and_group(solver, kind, K, width):
    import torch
    sizes = [40, 3, 200, 17, 64]
    A, B, ptr = draw(torch, 8, sizes, K, width, kind)
    G, _, _ = draw(torch, 9, sizes, width, 1, kind)
    want, size = want_nn(A, B, ptr, False)
    dwant, dsize = want_tn(A, G, ptr)
    A[41, K - 1], A[250, 0], B[3, K // 2, 1] = float("nan"), float("inf"), float("-inf")
    out = solver.op_transform_grouped(A.cuda(), B.cuda(), ptr.cuda()).cpu()
    bad = ~torch.isfinite(out)
    lone = torch.zeros_like(bad)
    lone[41], lone[250], lone[243:260, 1] = True, True, True        # rows 243 .. 259 are group 3
    assert torch.equal(bad, lone)
    keep = ~(lone.any(1) | lone.all(1)).numpy()
    close(out[keep], want[keep], size[keep], K, kind)
    dB = solver.op_wgrad_grouped(A.cuda(), G.cuda(), ptr.cuda()).cpu()
    # row 41 is in group 1, row 250 in group 3: a row of dB each
    bad = ~torch.isfinite(dB)
    lone = torch.zeros_like(bad)
    lone[1, K - 1], lone[3, 0] = True, True
    assert torch.equal(bad, lone)
    for g in (0, 2, 4):
        close(dB[g], dwant[g], dsize[g], max(sizes), "f32")


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_many_groups(solver, kind):
    """More groups than one step of the search looks at, most of them empty, and runs of equal bounds across its steps."""
    import torch
    rng = np.random.default_rng(3)
    sizes = np.where(rng.random(5000) < 0.7, 0, rng.integers(0, 6, 5000))
    sizes[1000:1400] = 0
    sizes[4097] = 400
    A, B, ptr = draw(torch, 11, sizes.tolist(), 24, 16, kind)
    close(solver.op_transform_grouped(A.cuda(), B.cuda(), ptr.cuda()), *want_nn(A, B, ptr, False), 24, kind)
    G, _, _ = draw(torch, 12, sizes.tolist(), 16, 1, kind)
    close(solver.op_wgrad_grouped(A.cuda(), G.cuda(), ptr.cuda()), *want_tn(A, G, ptr), 400, "f32")


def test_bounds_past_the_rows_are_clamped(solver):
    """Bounds below zero and past n count as 0 and n; with descending ones the rows that two groups claim may hold either's product, and
    nothing outside is touched."""
    import torch
    A, B, _ = draw(torch, 13, [200], 64, 64, "f32")
    Bs = B.repeat(3, 1, 1)
    want, size = want_nn(A, Bs, torch.tensor([0, 60, 200, 200]), False)
    for ptr in ([-5, 60, 200, 900], [-(1 << 62), 60, 1 << 62, 1 << 62]):
        held = torch.full((202, 64), 3.0, device="cuda")
        solver.op_transform_grouped(A.cuda(), Bs.cuda(), torch.tensor(ptr).cuda(), out=held[1:201])
        close(held[1:201], want, size, 64, "f32")
        assert (held[0] == 3.0).all() and (held[201] == 3.0).all()
        dB = solver.op_wgrad_grouped(A.cuda(), A.cuda(), torch.tensor(ptr).cuda())
        close(dB, *want_tn(A, A, torch.tensor([0, 60, 200, 200])), 200, "f32")


@pytest.mark.parametrize("kind,K,width,n", [("f32", 64, 64, 5000), ("bf16", 256, 256, 5000), ("f32", 33, 70, 3000), ("bf16", 300, 24, 90)])
def test_descending_bounds_touch_nothing_outside(solver, kind, K, width, n):
    """What the rows and matrices hold is not specified then; the rows around out and what lies around the gradient and its scratch stay as they
    are, as do the operands."""
    import ctypes as C
    import torch
    t = types()[kind]
    rng = np.random.default_rng(54)
    A, D = torch.randn(n, K, device="cuda").to(t), torch.randn(n, width, device="cuda").to(t)
    lib, h = solver.lib, solver.h
    for trial in range(6):
        groups = (1, 2, 7, 64, 65, 300)[trial]
        bounds = rng.integers(-n, 2 * n, groups + 1)
        bounds[0], bounds[-1] = (n, 0) if trial % 2 else (bounds[0], bounds[-1])
        ptr = torch.from_numpy(np.sort(bounds)[::-1].copy() if trial < 2 else bounds).cuda()
        B = torch.randn(groups, K, width, device="cuda").to(t)
        A0, B0, D0 = A.clone(), B.clone(), D.clone()
        held = torch.full((n + 300, width), 7.0, dtype=t, device="cuda")
        solver.op_transform_grouped(A, B, ptr, out=held[150:150 + n])
        need = C.c_size_t()
        assert lib.cadmm_op_wgrad_grouped_scratch(h, n, K, width, groups, C.byref(need)) == 0
        around = 1 << 20
        scratch = torch.full((need.value + 2 * around,), 77, dtype=torch.uint8, device="cuda")
        at = (scratch.data_ptr() + around + 255) & ~255
        dB = torch.full((groups * K * width + 20000,), 7.0, device="cuda")
        solver._on_raw_stream()
        rc = lib.cadmm_op_wgrad_grouped(h, {"f32": 0, "bf16": 1}[kind], A.data_ptr(), n, K, K, D.data_ptr(), width, width, groups, ptr.data_ptr(), 0,
                                        dB.data_ptr() + 40000, at, need.value)
        assert rc == 0
        torch.cuda.synchronize()
        first = at - scratch.data_ptr()
        assert (held[:150] == 7).all() and (held[150 + n:] == 7).all()
        assert (dB[:10000] == 7).all() and (dB[10000 + groups * K * width:] == 7).all()
        assert (scratch[:first] == 77).all() and (scratch[first + need.value:] == 77).all()
        assert torch.equal(A, A0) and torch.equal(B, B0) and torch.equal(D, D0)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_offsets_past_32_bits(solver, kind):
    """Rows so far apart that an element's offset passes 2^31 and a byte's 2^32, and as many results."""
    import torch
    n, step = 40000, 60000
    A, B, ptr = draw(torch, 14, [1, 39990, 9], 32, 40, kind)
    pick = np.r_[0:5, 20000:20005, n - 12:n]
    big = torch.empty(n * step, dtype=A.dtype, device="cuda")
    Av = torch.as_strided(big, (n, 32), (step, 1))
    Av.copy_(A)
    out = torch.as_strided(big, (n, 40), (step, 1), 64)
    solver.op_transform_grouped(Av, B.cuda(), ptr.cuda(), out=out)
    want, size = want_nn(A, B, ptr, False)
    close(out[pick], want[pick], size[pick], 32, kind)
    dB = solver.op_wgrad_grouped(Av, out, ptr.cuda())
    close(dB, *want_tn(A, out.cpu(), ptr), 39990, "f32")


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_gradients_against_the_formulas_and_against_differences(solver, kind):
    """L = sum D * (A_g B_g): dA = D B_g^T, dB_g = A_g^T D, and L is linear in either operand, so that (L(B + E) - L(B - E)) / 2 is the
    directional derivative itself.  It is taken in 64 bits of products of the operator, whose roundings are counted."""
    import torch
    sizes, K, width = [50, 0, 81, 7], 72, 40
    A, B, ptr = draw(torch, 21, sizes, K, width, kind)
    D, _, _ = draw(torch, 22, sizes, width, 1, kind)
    run = lambda X, Y: solver.op_transform_grouped(X.cuda(), Y.cuda(), ptr.cuda()).cpu().double()  # noqa: E731
    dA = solver.op_transform_grouped(D.cuda(), B.cuda(), ptr.cuda(), transposed=True)
    dB = solver.op_wgrad_grouped(A.cuda(), D.cuda(), ptr.cuda())
    close(dA, *want_nn(D, B, ptr, True), width, kind)
    close(dB, *want_tn(A, D, ptr), max(sizes), "f32")
    rng = np.random.default_rng(23)
    for X, grad in ((A, dA), (B, dB)):
        # steps that the type holds exactly: powers of two of X's own step, with X rounded to leave room for them
        E = torch.from_numpy(rng.choice([-1.0, 1.0], size=tuple(X.shape))).to(X.dtype)
        near = (X * 4).round() / 4                       # X +- 1 is exact in every type
        up = run(near + E, B) if X is A else run(A, near + E)
        down = run(near - E, B) if X is A else run(A, near - E)
        size = torch.from_numpy((want_nn(near.abs() + 1, B, ptr, False) if X is A else want_nn(A, near.abs() + 1, ptr, False))[1])
        slope = float(((up - down) * D.double()).sum() / 2)
        room = float((size * D.double().abs()).sum()) * (HALF[kind] + (K + 8) * 2.0 ** -24)
        room += float((grad.cpu().double() * E.double()).abs().sum()) * (HALF[kind] + 100 * 2.0 ** -24)
        assert abs(slope - float((grad.cpu().double() * E.double()).sum())) <= room


def test_two_streams_and_a_captured_step(solver):
    """Forward, both gradients and the optimiser's step as a training step uses them: on a side stream, and captured and replayed with
    other work in between, against the same calls one after the other."""
    import torch
    sizes, K, width = [500, 0, 300, 77], 128, 96
    A, B, ptr = (x.cuda() for x in draw(torch, 31, sizes, K, width, "bf16"))
    D = torch.randn(A.shape[0], width, device="cuda").bfloat16()
    W0 = torch.randn(len(sizes), K, width, device="cuda")

    def step(W, M):
        out = solver.op_transform_grouped(A, W.bfloat16(), ptr)
        G = (out - D).bfloat16()
        dA = solver.op_transform_grouped(G, W.bfloat16(), ptr, transposed=True)
        dB = solver.op_wgrad_grouped(A, G, ptr)
        solver.op_muon_step(W, M, dB, lr=0.02, weight_decay=0.1)
        return out, dA, dB

    W, M = W0.clone(), torch.zeros_like(W0)
    seen = []
    for _ in range(4):
        out, dA, dB = step(W, M)
        seen.append([x.clone() for x in (out, dA, dB, W, M)])
    side = torch.cuda.Stream()
    Ws, Ms = W0.clone(), torch.zeros_like(W0)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for k in range(4):
            got = [*step(Ws, Ms), Ws, Ms]
            for x, y in zip(got, seen[k]):
                assert torch.equal(x, y)
    torch.cuda.synchronize()
    Wg, Mg = W0.clone(), torch.zeros_like(W0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(Wg, Mg)
    Wg.copy_(W0)
    Mg.zero_()
    for k in range(4):
        graph.replay()
        torch.cuda.synchronize()
        solver.op_wgrad_grouped(A, D, ptr)                          # the program's own work in between
        torch.cuda.synchronize()
        for x, y in zip([*got, Wg, Mg], seen[k]):
            assert torch.equal(x, y), k


def test_communities_of_a_graph_are_groups(solver):
    """comm_row_ptr of a solver's graph as the bounds, rows in the internal order."""
    import torch
    from paper_2112_09335_amd import binding
    w = synth.config(1)
    s = binding.Solver(0)
    try:
        s.build_graph(w.N, w.src, w.dst, w.M, w.comm)
        g = s.get_graph()
        ptr = torch.from_numpy(g["comm_row_ptr"])
        A, B, _ = draw(torch, 41, np.diff(g["comm_row_ptr"]).tolist(), 40, 24, "f32")
        out = s.op_transform_grouped(A.cuda(), B.cuda(), ptr.cuda())
        close(out, *want_nn(A, B, ptr, False), 40, "f32")
    finally:
        s.close()


def test_refusals_of_tensors(solver):
    import torch
    from paper_2112_09335_amd.binding import CadmmError
    A, B, ptr = (x.cuda() for x in draw(torch, 51, [5, 6], 8, 4, "f32"))
    bad = [
        (A.cpu(), B, ptr), (A, B.cpu(), ptr), (A, B, ptr.cpu()), (A, B, ptr.int()), (A, B.bfloat16(), ptr), (A.double(), B.double(), ptr),
        (A, B, ptr[:1]), (A, B[:1], ptr), (A, B[0], ptr), (A[:, :7], B, ptr), (A.T.contiguous().T, B, ptr), (A, B.transpose(1, 2), ptr),
        (A, B, ptr.repeat(2)[::2]), (A[:1].expand(11, 8), B, ptr),
    ]
    for a, b, p in bad:
        with pytest.raises(CadmmError):
            solver.op_transform_grouped(a, b, p)
    for out in (torch.empty(11, 5, device="cuda"), torch.empty(10, 4, device="cuda"), torch.empty(11, 4), torch.empty(11, 4, device="cuda").bfloat16()):
        with pytest.raises(CadmmError):
            solver.op_transform_grouped(A, B, ptr, out=out)
    G = torch.zeros(11, 4, device="cuda")
    for a, g, p, more in ((A, G[:10], ptr, {}), (A, G.half(), ptr, {}), (A, G, ptr[:1], {}), (A, G, ptr, dict(out_dtype=torch.float16)),
                          (A, G, ptr, dict(out=torch.empty(2, 8, 5, device="cuda"))), (A, G, ptr, dict(out=torch.empty(2, 4, 8, device="cuda").transpose(1, 2)))):
        with pytest.raises(CadmmError):
            solver.op_wgrad_grouped(a, g, p, **more)


def test_an_output_that_shares_elements_with_an_operand_is_refused(solver):
    """Its tiles would be written while others still read them.  Other columns of one buffer, and neighbours in memory, are apart."""
    import torch
    from paper_2112_09335_amd.binding import CadmmError
    n, K = 300, 64
    rng = np.random.default_rng(52)
    held = torch.from_numpy(rng.standard_normal((n + 70, 2 * K)).astype(np.float32)).cuda()
    before = held.clone()
    ptr = torch.tensor([0, 100, n], device="cuda")
    B = torch.randn(2, K, K, device="cuda")
    A = held[:n, :K]
    flat = held.view(-1)
    bad = [A, held[:n, 1:K + 1], held[:n, K - 1:2 * K - 1], held[1:n + 1, :K], held[40:n + 40, :K], flat[K:K + n * K].view(n, K),
           flat[:n * (K + 3)].view(n, K + 3)[:, :K], held[:1, :K].expand(n, K)]
    for out in bad:
        with pytest.raises(CadmmError):
            solver.op_transform_grouped(A, B, ptr, out=out)
    few = torch.tensor([0, 1, 2], device="cuda")
    with pytest.raises(CadmmError):
        solver.op_transform_grouped(A[:2], B, few, out=B[1, 5:7])
    with pytest.raises(CadmmError):
        solver.op_transform_grouped(A[:2, :3].contiguous(), B[:, :3, :3].contiguous(), few, out=few.view(torch.float32)[:6].view(2, 3))
    for out in (flat[:2 * K * K].view(2, K, K), flat[2 * K * (n - 1):2 * K * (n - 1) + 2 * K * K].view(2, K, K)):
        with pytest.raises(CadmmError):
            solver.op_wgrad_grouped(A, A.contiguous(), ptr, out=out)
        with pytest.raises(CadmmError):
            solver.op_wgrad_grouped(A.contiguous(), A, ptr, out=out)
    assert torch.equal(held, before)
    want = solver.op_transform_grouped(A, B, ptr)
    assert torch.equal(solver.op_transform_grouped(A, B, ptr, out=held[:n, K:]), want) and torch.equal(held[:, :K], before[:, :K])
    dB = solver.op_wgrad_grouped(A, A, ptr)
    at = flat[2 * K * (n - 1) + K:][:2 * K * K].view(2, K, K)                # right behind A's last row
    assert torch.equal(solver.op_wgrad_grouped(A, A, ptr, out=at), dB) and torch.equal(held[:n, :K], before[:n, :K])


@pytest.mark.parametrize("rows", [300, 40, 7])
def test_every_product_of_two_fp32_numbers(solver, rows):
    """Sums of one product: the three parts leave out less than 2^-24 (1 + 2^-8) of it, an instruction may be off by a step (2^-23) in adding
    the largest terms, and in adding those below 2^-7 of them by 2^-30 each: less than 4 * 2^-24 in all.  Numbers whose bits behind the eighth
    are all ones or just beyond a tie, random ones, and the largest of all against small ones."""
    import torch
    rng = np.random.default_rng(53)
    bits = np.array([0x3f80ffff, 0x3f807fff, 0x3f808001, 0x3f817f80, 0x3f80ff80, 0x3fffffff, 0x3f800000, 0x3f80807f, 0x3fc07f7f, 0x3f810001], np.uint32)
    x = np.concatenate([bits.view(np.float32), rng.uniform(1.0, 2.0, 290).astype(np.float32)])
    x *= np.exp2(rng.integers(-60, 60, 300)).astype(np.float32) * rng.choice([-1, 1], 300).astype(np.float32)
    y = rng.permutation(x)[:200] * np.float32(2.0 ** -3)
    largest = np.array([0x7f7fffff, 0x7f7f8000, 0x7f7f7fff, 0x7f7f8001, 0xff7fffff], np.uint32).view(np.float32)
    for a, b in ((x[:rows], y), (largest, np.concatenate([bits[:7].view(np.float32) * np.float32(2.0 ** -k) for k in (1, 40, 100)]))):
        want = np.outer(a.astype(np.float64), b.astype(np.float64))
        A, B = torch.from_numpy(a).view(-1, 1), torch.from_numpy(b)
        ptr = torch.tensor([0, len(a)])
        got = [solver.op_transform_grouped(A.cuda(), B.view(1, 1, -1).cuda(), ptr.cuda()),
               solver.op_transform_grouped(A.cuda(), B.view(1, -1, 1).cuda(), ptr.cuda(), transposed=True),
               solver.op_wgrad_grouped(A.view(1, -1).cuda(), B.view(1, -1).cuda(), torch.tensor([0, 1]).cuda())[0]]
        for g in got:
            far = np.abs(g.cpu().double().numpy() - want) / np.abs(want)
            assert far.max() < 4 * 2.0 ** -24, (far.max() * 2.0 ** 24, np.unravel_index(far.argmax(), far.shape))


@pytest.mark.parametrize("kind,small,large", [("f32", -100, 90), ("f32", -126, 100), ("f32", -140, 120), ("f32", -60, -60), ("bf16", -126, 100), ("bf16", -132, 110), ("f16", -15, 4),
                                              ("f16", -20, 8)])
@pytest.mark.parametrize("n,K,width", [(64, 64, 64), (5, 1, 40), (300, 256, 200), (9, 33, 5)])
def test_operands_near_the_least_numbers(solver, kind, small, large, n, K, width):
    """16-bit operands count as they are, subnormal ones too; the last part of an fp32 number is cut at 2^-133, bf16's least, which the
    other operand multiplies."""
    import torch
    rng = np.random.default_rng(55)
    A = torch.from_numpy(rng.standard_normal((n, K)) * 2.0 ** small).to(types()[kind])
    B = torch.from_numpy(rng.standard_normal((1, K, width)) * 2.0 ** large).to(types()[kind])
    ptr = torch.tensor([0, n])
    want, size = want_nn(A, B, ptr, False)
    cut = 2.0 ** -133 * 2.0 ** 24 / (K + 8)                   # (as close counts: times (K + 8) 2^-24)
    if kind == "f32":
        size = size + cut * (np.abs(B[0].double().numpy()).sum(0)[None, :] + A.double().abs().sum(1, keepdim=True).numpy())
    close(solver.op_transform_grouped(A.cuda(), B.cuda(), ptr.cuda()), want, size, K, kind)
    close(solver.op_transform_grouped(A.cuda(), B.transpose(1, 2).contiguous().cuda(), ptr.cuda(), transposed=True), want, size, K, kind)
    G = B[:, 0].expand(n, width).contiguous() * torch.from_numpy(rng.choice([-1.0, 1.0], (n, 1))).to(B.dtype)
    want, size = want_tn(A, G, ptr)
    if kind == "f32":
        cut = 2.0 ** -133 * 2.0 ** 24 / (n + 8)
        size = size + cut * (G.double().abs().sum(0).numpy()[None, None, :] + A.double().abs().sum(0).numpy()[None, :, None])
    close(solver.op_wgrad_grouped(A.cuda(), G.cuda(), ptr.cuda()), want, size, n, "f32")


def test_no_rows_at_all(solver):
    import torch
    ptr = torch.zeros(4, dtype=torch.int64, device="cuda")
    out = solver.op_transform_grouped(torch.empty(0, 16, device="cuda"), torch.zeros(3, 16, 8, device="cuda"), ptr)
    assert tuple(out.shape) == (0, 8)
    dB = solver.op_wgrad_grouped(torch.empty(0, 16, device="cuda"), torch.empty(0, 8, device="cuda"), ptr)
    assert (dB == 0).all() and tuple(dB.shape) == (3, 16, 8)
