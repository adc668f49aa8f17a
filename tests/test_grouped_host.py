"""Refusals of the products over groups of rows and of the orthogonalised updates, and the streams and devices they use: no GPU call."""
import ctypes as C
import os

import numpy as np
import pytest

from paper_2112_09335_amd import binding
from test_op_streams_host import recorder  # noqa: F401  (fixture)

OK, EINVAL, ENOMEM, EUNSUPPORTED = 0, -1, -3, -5
BUF = 0x100000                              # an address that is never looked at
MUON = (3.4445, -4.7750, 2.0315)


@pytest.fixture()
def host():
    s = binding.Solver(device=-1)
    yield s
    s.close()


def transform(s, type=0, A=BUF, n=10, lda=8, K=8, B=BUF, width=4, transposed=0, groups=2, ptr=BUF, out=BUF, ldo=4):
    return s.lib.cadmm_op_transform_grouped(s.h, type, A, n, lda, K, B, width, transposed, groups, ptr, out, ldo)


def wgrad(s, type=0, A=BUF, n=10, lda=8, K=8, G=BUF, ldg=4, width=4, groups=2, ptr=BUF, out_type=0, out=BUF, scratch=BUF, bytes=1 << 40):
    return s.lib.cadmm_op_wgrad_grouped(s.h, type, A, n, lda, K, G, ldg, width, groups, ptr, out_type, out, scratch, bytes)


def ortho(s, type=0, G=BUF, batch=2, K=8, width=4, steps=5, coefficients=MUON, eps=1e-7, out=BUF, scratch=BUF, bytes=1 << 40):
    c = None if coefficients is None else (C.c_float * 3)(*coefficients)
    return s.lib.cadmm_op_orthogonalise(s.h, type, G, batch, K, width, steps, c, eps, out, scratch, bytes)


def muon(s, type=0, G=BUF, W=BUF + 0x10000, M=BUF + 0x20000, batch=2, K=8, width=4, lr=0.1, momentum=0.9, nesterov=1, decay=0.0, scale=1.0, steps=5,
         coefficients=MUON, eps=1e-7, scratch=BUF, bytes=1 << 40):
    c = None if coefficients is None else (C.c_float * 3)(*coefficients)
    return s.lib.cadmm_op_muon_step(s.h, type, G, W, M, batch, K, width, lr, momentum, nesterov, decay, scale, steps, c, eps, scratch, bytes)


@pytest.mark.parametrize("call", [transform, wgrad, ortho, muon])
def test_a_right_call_is_refused_for_want_of_a_device_only(host, call):
    assert call(host) == EUNSUPPORTED
    assert b"host-only" in host.lib.cadmm_last_error(host.h)


@pytest.mark.parametrize("wrong", [
    dict(A=None), dict(B=None), dict(out=None), dict(ptr=None), dict(n=-1), dict(K=0), dict(width=0), dict(groups=0), dict(type=3),
    dict(type=-1), dict(lda=7), dict(ldo=3), dict(A=BUF + 2), dict(type=1, B=BUF + 1), dict(out=BUF + 1), dict(ptr=BUF + 4),
    dict(K=65537, lda=65537), dict(width=65537, ldo=65537), dict(groups=(1 << 20) + 1), dict(n=(1 << 40) + 1), dict(lda=1 << 59),
])
def test_refusals_of_the_product_over_groups(host, wrong):
    assert transform(host, **wrong) == EINVAL


def test_an_output_that_overlaps_its_input_in_part_is_refused(host):
    size = 2 * 8 * 4 * 4
    assert ortho(host, out=BUF) == EUNSUPPORTED and ortho(host, out=BUF + size) == EUNSUPPORTED and ortho(host, G=BUF + size) == EUNSUPPORTED
    assert ortho(host, out=BUF + size - 4) == EINVAL and ortho(host, G=BUF + size - 4) == EINVAL


def test_a_product_of_no_rows_is_done(host):
    assert transform(host, n=0, A=None, out=None) in (OK, EUNSUPPORTED)


def test_a_product_of_too_many_tiles_is_not_supported(host):
    assert transform(host, n=1 << 40, lda=8, width=60, ldo=60) == EUNSUPPORTED
    assert wgrad(host, K=60000, lda=60000, width=60000, ldg=60000, groups=1 << 20) == EUNSUPPORTED
    assert ortho(host, K=32768, width=32768, batch=1000) == EUNSUPPORTED


@pytest.mark.parametrize("wrong,code", [
    (dict(A=None), EINVAL), (dict(G=None), EINVAL), (dict(out=None), EINVAL), (dict(ptr=None), EINVAL), (dict(n=-1), EINVAL), (dict(K=0), EINVAL),
    (dict(width=0), EINVAL), (dict(groups=0), EINVAL), (dict(type=3), EINVAL), (dict(type=1, out_type=2), EINVAL), (dict(out_type=1), EINVAL),
    (dict(lda=7), EINVAL), (dict(ldg=3), EINVAL), (dict(G=BUF + 2), EINVAL), (dict(type=2, A=BUF + 1), EINVAL), (dict(type=2, out_type=0, out=BUF + 2), EINVAL),
    (dict(ptr=BUF + 2), EINVAL),
])
def test_refusals_of_the_weight_gradient_over_groups(host, wrong, code):
    assert wgrad(host, **wrong) == code


def test_scratch_that_is_too_small_or_misaligned_is_refused(host):
    need = C.c_size_t()
    assert host.lib.cadmm_op_orthogonalise_scratch(host.h, 2, 8, 4, C.byref(need)) == OK and need.value > 0
    assert ortho(host, bytes=need.value - 1) == ENOMEM and muon(host, bytes=need.value - 1) == ENOMEM
    assert ortho(host, bytes=need.value) == EUNSUPPORTED
    assert ortho(host, scratch=BUF + 128) == EINVAL and muon(host, scratch=BUF + 16) == EINVAL
    args = dict(n=200000, K=256, lda=256, width=256, ldg=256, groups=2)
    assert host.lib.cadmm_op_wgrad_grouped_scratch(host.h, 200000, 256, 256, 2, C.byref(need)) == OK
    if need.value:
        assert wgrad(host, bytes=need.value - 1, **args) == ENOMEM
        assert wgrad(host, scratch=None, **args) == EINVAL and wgrad(host, scratch=BUF + 64, **args) == EINVAL
    assert wgrad(host, bytes=need.value, **args) == EUNSUPPORTED


@pytest.mark.parametrize("call", [ortho, muon])
@pytest.mark.parametrize("wrong,code", [
    (dict(G=None), EINVAL), (dict(scratch=None), EINVAL), (dict(coefficients=None), EINVAL), (dict(batch=0), EINVAL), (dict(K=0), EINVAL),
    (dict(width=-1), EINVAL), (dict(steps=0), EINVAL), (dict(steps=65), EINVAL), (dict(eps=-1e-9), EINVAL), (dict(eps=float("nan")), EINVAL),
    (dict(eps=float("inf")), EINVAL), (dict(type=4), EINVAL), (dict(type=1, G=BUF + 1), EINVAL), (dict(K=32769), EUNSUPPORTED),
    (dict(batch=65536), EUNSUPPORTED),
    (dict(coefficients=(float("nan"), 0, 0)), EINVAL), (dict(coefficients=(1, float("inf"), 0)), EINVAL),
    (dict(coefficients=(2000.0, 0, 0)), EINVAL), (dict(coefficients=(4.1, 0, 0)), EINVAL),       # 4.1^5 = 1158
    (dict(coefficients=(1.0, 3.0, 0.0)), EINVAL),                                          # 4, 196, ...
])
def test_refusals_of_the_orthogonalised_updates(host, call, wrong, code):
    assert call(host, **wrong) == code


@pytest.mark.parametrize("coefficients,steps", [((4.0, 0, 0), 5), ((1.5, -0.5, 0), 64), ((15 / 8, -10 / 8, 3 / 8), 64), (MUON, 64), ((0, 0, 0), 1)])
def test_coefficients_that_keep_singular_values_in_bounds_are_taken(host, coefficients, steps):
    assert ortho(host, coefficients=coefficients, steps=steps) == EUNSUPPORTED                   # (for want of a device)


@pytest.mark.parametrize("wrong", [dict(W=None), dict(M=None), dict(W=BUF + 0x10002), dict(M=BUF + 0x20001),
                                   dict(W=BUF + 0x20000), dict(G=BUF + 0x10000), dict(M=BUF + 252), dict(G=BUF + 0x20004),
                                   dict(lr=float("nan")), dict(momentum=float("inf")),
                                   dict(decay=float("nan")), dict(scale=float("inf"))])
def test_refusals_of_the_optimiser_step(host, wrong):
    assert muon(host, **wrong) == EINVAL


def test_new_calls_run_where_the_context_is_and_on_the_stream_they_are_told(recorder):  # noqa: F811
    """With another device current, on the null stream and on the caller's: launched with the context's device current, on that stream, and
    the caller's device is current again afterwards."""
    recorder("""
f32, sz = ctypes.c_float, ctypes.c_size_t
lib.cadmm_op_transform_grouped.argtypes = [vp, i32, vp, i64, i64, i32, vp, i32, i32, i32, vp, vp, i64]
lib.cadmm_op_wgrad_grouped.argtypes = [vp, i32, vp, i64, i64, i32, vp, i64, i32, i32, vp, i32, vp, vp, sz]
lib.cadmm_op_orthogonalise.argtypes = [vp, i32, vp, i32, i32, i32, i32, vp, f32, vp, vp, sz]
lib.cadmm_op_muon_step.argtypes = [vp, i32, vp, vp, vp, i32, i32, i32, f32, f32, i32, f32, f32, i32, vp, f32, vp, sz]
buf, co = 0x20000, (f32 * 3)(3.4445, -4.775, 2.0315)
CALLS = [
    lambda t: lib.cadmm_op_transform_grouped(h, t, buf, 1000, 64, 64, buf, 48, 0, 4, buf, buf, 48),
    lambda t: lib.cadmm_op_transform_grouped(h, t, buf, 5, 65, 65, buf, 48, 1, 4, buf, buf, 49),
    lambda t: lib.cadmm_op_wgrad_grouped(h, t, buf, 100000, 64, 64, buf, 48, 48, 4, buf, 0, buf, buf, 1 << 40),
    lambda t: lib.cadmm_op_orthogonalise(h, t, buf, 3, 64, 48, 5, co, 1e-7, buf, buf, 1 << 40),
    lambda t: lib.cadmm_op_orthogonalise(h, t, buf, 3, 640, 700, 2, co, 1e-7, buf, buf, 1 << 40),
    lambda t: lib.cadmm_op_muon_step(h, t, buf, 2 * buf, 3 * buf, 3, 64, 48, .1, .9, 1, 0., 1., 5, co, 1e-7, buf, 1 << 40),
]
where = ctypes.c_int()
for device in (0, 1):
    assert rec.hipSetDevice(device) == 0
    for stream in (None, A, OWN, None, B):
        for f in CALLS:
            for t in (0, 1, 2):
                rec.recorder_clear()
                assert lib.cadmm_op_stream(h, stream) == 0
                rc = f(t)
                log = [(w, int(a), int(b)) for w, a, b in (l.split() for l in rec.recorder_log().decode().splitlines())]
                launches = [x for x in log if x[0] == "launch"]
                assert rc == 0 and launches and all(x[1:] == (stream or 0, 0) for x in launches), (rc, log)
                assert not any(w == "record-elsewhere" for w, _, _ in log), log
                assert rec.hipGetDevice(ctypes.byref(where)) == 0 and where.value == device
""")


def most_of(coefficients):
    """The largest |x (a + b x^2 + c x^4)| on [0, 1], by looking at a million of them (flat around it: off by 1e-11 of a + |b| + |c|)."""
    a, b, c = (np.float64(np.float32(x)) for x in coefficients)
    x = np.linspace(0.0, 1.0, 1 << 20)
    return np.abs(x * (a + x * x * (b + c * x * x))).max()


@pytest.mark.parametrize("call", [ortho, muon])
@pytest.mark.parametrize("shape", [(3, -3, 1e-17), (3, -3, -1e-17), (3, -3, 1e-18), (3, -3, 1e-16), (3, -3, 0), (3, -3, 1e-9), (-3, 3, 1e-17), (3, -3, 1e-3), (1, 0, -1),
                                   (-1, 0, 1), (5, -20, 16), (0, 1, -1), (0, 1, 1e-20), (1, -1e-20, -1), (3, -4, 1.2), (1, 1, 1), (1e-3, -1, 1e-17)])
def test_growth_is_judged_by_the_largest_value_wherever_it_lies(host, call, shape):
    """One step, coefficients brought to where the largest value is just below or above 1024, whatever their sizes relative to each other."""
    for size, code in ((1023.0, EUNSUPPORTED), (1025.0, EINVAL)):            # (EUNSUPPORTED: for want of a device)
        k = size / most_of(shape)
        coefficients = tuple(k * x for x in shape)
        assert (most_of(coefficients) < 1024) == (code == EUNSUPPORTED)
        assert call(host, coefficients=coefficients, steps=1) == code, coefficients


def test_sets_of_rows_meet_where_they_share_a_byte():
    rng = np.random.default_rng(1)
    seen = [0, 0]
    for _ in range(20000):
        sets = []
        for _ in range(2):
            width = int(rng.integers(1, 6))
            sets.append((int(rng.integers(0, 40)), int(rng.integers(0, 7)), width + int(rng.choice([0, 0, 1, 3, 7, 11])), width))
        if rng.random() < 0.5:
            sets[1] = (sets[1][0], sets[1][1], max(sets[0][2], sets[1][3]), sets[1][3])      # rows equally far apart
        bytes_of = [{at + i * step + k for i in range(n) for k in range(width)} for at, n, step, width in sets]
        meet = bool(bytes_of[0] & bytes_of[1])
        assert binding._rows_meet(*sets) == meet and binding._rows_meet(*sets[::-1]) == meet, sets
        seen[meet] += 1
    assert min(seen) > 2000
    far = (1 << 46, 3 << 20, 100, 40)
    assert not binding._rows_meet(far, ((1 << 46) + 40, 3 << 20, 100, 60)) and binding._rows_meet(far, ((1 << 46) + 39, 3 << 20, 100, 60))
    assert binding._rows_meet(far, ((1 << 46) + 40, 3 << 20, 101, 60)) and not binding._rows_meet(far, ((1 << 46) + 40, 3 << 20, 200, 60))


def test_sizes_past_the_limits_give_the_codes_that_the_header_names(host):
    need = C.c_size_t()
    query = host.lib.cadmm_op_wgrad_grouped_scratch
    most = dict(n=1 << 40, K=1 << 16, width=1 << 16, groups=1 << 20)
    for size, stride in dict(n=None, K="lda", width="ldo", groups=None).items():
        past = most[size] + 1
        assert transform(host, **{size: past}, **({stride: past} if stride else {})) == EINVAL
        assert wgrad(host, **{size: past}, **({"ldg" if stride == "ldo" else stride: past} if stride else {})) == EINVAL
        sizes = {**dict(n=10, K=8, width=4, groups=2), size: past}
        assert query(host.h, sizes["n"], sizes["K"], sizes["width"], sizes["groups"], C.byref(need)) == EINVAL
        sizes[size] = most[size]
        assert query(host.h, sizes["n"], sizes["K"], sizes["width"], sizes["groups"], C.byref(need)) == OK
    text = " ".join(open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "cadmm.h")).read().replace(" * ", " ").split())
    assert "At most 65536 columns, 2^20 groups and 2^40 rows (CADMM_EINVAL beyond), and result tiles for 2^22 workgroups (CADMM_EUNSUPPORTED beyond)" in text


@pytest.mark.parametrize("wrong", [dict(lr=1e30, scale=1e30), dict(lr=-1e30, scale=1e30), dict(lr=1e30, decay=1e30), dict(lr=3e38, scale=1.2)])
def test_rates_past_the_largest_number_are_refused(host, wrong):
    """Infinite in fp32, they would make NaN of every weight whose update is zero."""
    assert muon(host, **wrong) == EINVAL
    assert muon(host, **{**wrong, "lr": 1e-30}) == EUNSUPPORTED                # (for want of a device)
