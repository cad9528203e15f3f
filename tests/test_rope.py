"""RMS norm and rotation of queries and keys (pf_rope_init, pf_qk_norm_rope): frequencies and refusals on the CPU, results on the
GPU against the formula in 64 bits."""
import ctypes
import math
import os

import pytest
import torch

from paper_2605_13111_amd import binding as B
from paper_2605_13111_amd import synth

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libpf.so not built")
DEV = "cuda:0"


def _pairs(rot, axes):
    n = rot // 2
    return [n] if axes == 1 else [n - 2 * (n // 3), n // 3, n // 3] if axes == 3 else [n - n // 2, n // 2]


# ---- frequencies ------------------------------------------------------------------------------------------------------

def test_frequencies_of_one_and_three_axes():
    r = B.make_rope(128, base=10000.0)
    for i in range(64):
        assert math.isclose(r.turns[i], 10000.0 ** (-i / 64) / (2 * math.pi), rel_tol=1e-14)
    r = B.make_rope(128, axis_pairs=[22, 21, 21], interleaved=True, base=500.0)
    at = 0
    for n in (22, 21, 21):
        for m in range(n):
            assert math.isclose(r.turns[at], 500.0 ** (-m / n) / (2 * math.pi), rel_tol=1e-14)
            at += 1
    assert (r.rot_dim, r.n_axes, r.interleaved, r.magnitude) == (128, 3, 1, 1.0)


def test_scaled_frequencies():
    plain, lin = B.make_rope(64), B.make_rope(64, scaling="linear", factor=4.0, magnitude=1.25)
    assert lin.magnitude == 1.25 and all(math.isclose(lin.turns[i], plain.turns[i] / 4, rel_tol=1e-14) for i in range(32))
    s = B.make_rope(64, scaling="by_wavelength", factor=8.0, original_positions=4096, slow_turns=1.0, fast_turns=32.0)
    seen = set()
    for i in range(32):
        often = plain.turns[i] * 4096
        if often >= 32:
            want = 1.0
            seen.add("fast")
        elif often <= 1:
            want = 1 / 8
            seen.add("slow")
        else:
            keep = (often - 1) / 31
            want = keep + (1 - keep) / 8
            seen.add("ramp")
        assert math.isclose(s.turns[i], plain.turns[i] * want, rel_tol=1e-12)
    assert seen == {"fast", "slow", "ramp"}


@pytest.mark.parametrize("kw", [
    dict(rot_dim=136), dict(rot_dim=12), dict(rot_dim=-8), dict(axis_pairs=[64, 1]), dict(axis_pairs=[16, 16, 16, 16]), dict(axis_pairs=[]),
    dict(axis_pairs=[65, -1]), dict(base=0.0), dict(base=float("nan")), dict(scaling="linear", factor=0.5), dict(scaling="linear", factor=float("nan")),
    dict(scaling="by_wavelength", factor=2.0), dict(scaling="by_wavelength", factor=2.0, original_positions=100, slow_turns=4, fast_turns=4),
    dict(magnitude=float("inf")),
])
def test_frequencies_refused(kw):
    with pytest.raises(B.PfError) as e:
        B.make_rope(128, **kw)
    assert e.value.status == B.PF_ERR_INVALID_ARG


def test_head_sizes_refused():
    with pytest.raises(B.PfError) as e:
        B.make_rope(96)
    assert e.value.status == B.PF_ERR_UNSUPPORTED


def test_calls_refused_without_a_device():
    """Every refusal comes before anything is enqueued, so fake addresses do."""
    L, rope = B.lib(), B.make_rope(128)
    pos, fake = ctypes.c_void_p(0x1000), 0x10000

    def rows(x=fake, out=fake, weight=0, heads=4, reserved=0, xl=(512, 128), ol=(512, 128)):
        return B.pf_rope_rows(x, out, weight, heads, reserved, B.pf_chunk_layout(*xl), B.pf_chunk_layout(*ol))

    def call(q=None, k=None, n=10, eps=1e-6, r=rope, p=pos):
        q, k = rows() if q is None else q, rows() if k is None else k
        return L.pf_qk_norm_rope(ctypes.byref(r) if r is not None else None, n, p, ctypes.byref(q), ctypes.byref(k), eps, None)

    empty = B.pf_rope_rows()
    bad = B.PF_ERR_INVALID_ARG
    assert call(n=0) == B.PF_OK                                   # nothing to do, nothing touched
    assert call(n=-1) == bad and call(n=1 << 26) == bad and call(n=(1 << 26) + 1) == bad
    assert call(r=None) == bad and call(p=None) == bad and call(p=ctypes.c_void_p(0x1002)) == bad
    assert L.pf_qk_norm_rope(ctypes.byref(rope), 10, pos, None, ctypes.byref(rows()), 1e-6, None) == bad
    assert call(q=empty, k=empty) == bad
    for t in (rows(x=0), rows(out=0), rows(x=fake + 8), rows(out=fake + 2), rows(weight=fake + 8), rows(heads=-1), rows(heads=1025), rows(reserved=1),
              rows(xl=(512, 127)), rows(xl=(500, 128)), rows(ol=(256, 128)), rows(xl=(128, 0)), rows(heads=0)):
        assert call(q=t) == bad and call(k=t) == bad
    assert call(eps=-1.0) == bad and call(eps=float("nan")) == bad and call(eps=float("inf")) == bad
    assert call(q=rows(weight=fake), eps=0.0) == bad              # a weight without a norm
    odd = B.make_rope(128)
    odd.axis_pairs[0] = 63
    assert call(r=odd) == bad
    odd = B.make_rope(128)
    odd.head_dim = 96
    assert call(r=odd) == B.PF_ERR_UNSUPPORTED


def test_the_most_tokens_of_a_call():
    """A launch has fewer than 2^32 threads: four tokens to a workgroup of 256, fewer than 2^24 workgroups.  The refusal comes before anything
    is enqueued, so fake addresses do."""
    L, rope = B.lib(), B.make_rope(64)
    one = B.pf_rope_rows(0x10000, 0x10000, 0, 1, 0, B.pf_chunk_layout(64, 64 << 26), B.pf_chunk_layout(64, 64 << 26))
    for n in ((1 << 26) - 3, (1 << 26) - 2, (1 << 26) - 1):
        assert L.pf_qk_norm_rope(ctypes.byref(rope), n, 0x1000, ctypes.byref(one), ctypes.byref(B.pf_rope_rows()), 1e-6, None) == B.PF_ERR_INVALID_ARG


def test_no_tokens_need_no_memory():
    """Tensors without a token have no address; a call on them does nothing.  What is wrong without them is refused all the same."""
    L, rope, D = B.lib(), B.make_rope(128), 128

    def call(q, k, p=0, n=0):
        return L.pf_qk_norm_rope(ctypes.byref(rope), n, p, q, k, 1e-6, None)

    x = torch.empty((0, 4, D), dtype=torch.bfloat16).transpose(0, 1)
    rows = B._rope_rows(D, 0, x.get_device(), x, torch.empty_like(x), None)
    assert call(rows, rows) == B.PF_OK
    packed = B.pf_rope_rows(0, 0, 0, 4, 0, B.pf_chunk_layout(0, 0), B.pf_chunk_layout(0, 0))
    assert call(ctypes.byref(packed), ctypes.byref(B.pf_rope_rows())) == B.PF_OK
    assert call(rows, rows, n=1) == B.PF_ERR_INVALID_ARG and call(rows, rows, p=0x1000, n=1) == B.PF_ERR_INVALID_ARG
    packed.x = 0x1008
    assert call(ctypes.byref(packed), rows) == B.PF_ERR_INVALID_ARG


@pytest.mark.parametrize("which", ["x", "out"])
def test_views_that_repeat_one_row_are_refused(which):
    """A row expanded over heads and tokens has strides of zero, which the library's structs take for packed tensors."""
    D, dev = 64, torch.empty(0).get_device()
    good, bad = torch.zeros((3, 5, D), dtype=torch.bfloat16), torch.zeros(D, dtype=torch.bfloat16).expand(3, 5, D)
    B._rope_rows(D, 5, dev, good, good, None)
    with pytest.raises(AssertionError):
        B._rope_rows(D, 5, dev, bad if which == "x" else good, bad if which == "out" else good, None)
    L, rope = B.lib(), B.make_rope(D)
    for strided in (good[:1].expand(3, 5, D), good[:, :1].expand(3, 5, D)):   # one of the strides zero: refused by the library
        rows = B._rope_rows(D, 5, dev, *((strided, good) if which == "x" else (good, strided)), None)
        assert L.pf_qk_norm_rope(ctypes.byref(rope), 5, 0x1000, rows, ctypes.byref(B.pf_rope_rows()), 1e-6, None) == B.PF_ERR_INVALID_ARG


# ---- results ----------------------------------------------------------------------------------------------------------

def _formula(x, w, positions, rope, eps):
    """[heads, tokens, D] in 64 bits and the size of what is added up for each value."""
    y = x.double().cpu()
    if eps > 0:
        y = y / torch.sqrt(y.pow(2).mean(-1, keepdim=True) + eps)
        if w is not None:
            y = y * w.double().cpu()
    out, size = y.clone(), y.abs()
    at = 0
    for a in range(rope.n_axes):
        for _ in range(rope.axis_pairs[a]):
            i, j = (2 * at, 2 * at + 1) if rope.interleaved else (at, at + rope.rot_dim // 2)
            # the angle modulo one turn: exact products of 53 bits and 31 are not needed, 64-bit rounding leaves 1e-7 of a turn at 2^30
            t = positions[a].double().cpu() * rope.turns[at]
            t = (t - t.round()) * (2 * math.pi)
            m = rope.magnitude
            out[..., i], out[..., j] = m * (y[..., i] * t.cos() - y[..., j] * t.sin()), m * (y[..., i] * t.sin() + y[..., j] * t.cos())
            size[..., i] = size[..., j] = m * (y[..., i].abs() + y[..., j].abs())
            at += 1
    return out, size


def _check(got, x, w, positions, rope, eps):
    """One rounding to bf16 (2^-8 relative at most); in front of it fp32: the norm's sum, root, quotient and two products (8 roundings of
    2^-24 at most, each a factor on the value), the two products and the sum of the rotation, and a sine and cosine within 2e-6."""
    want, size = _formula(x, w, positions, rope, eps)
    err = (got.double().cpu() - want).abs()
    bound = 2.0 ** -8 * want.abs() + size * (2e-6 + 12 * 2.0 ** -24) * (1 + 2.0 ** -8) + 1e-38
    assert torch.isfinite(got).all()
    assert (err <= bound).all(), "off by %.3g where %.3g is allowed" % (float((err - bound).max()), float(bound[(err - bound) == (err - bound).max()][0]))


@pytest.mark.gpu
@pytest.mark.parametrize("D,rot,interleaved,axes", [
    (128, 128, False, 1), (128, 128, True, 3), (128, 64, False, 3), (128, 72, True, 1), (128, 8, False, 1), (128, 120, False, 2), (64, 64, True, 1),
    (64, 64, False, 3), (64, 40, False, 1), (64, 8, True, 1), (128, 0, False, 1), (64, 0, True, 1),
])
@pytest.mark.parametrize("tokens,hq,hk,eps,model", [(1, 1, 1, 1e-6, True), (7, 5, 2, 1e-5, False), (130, 12, 12, 0.0, True), (65, 32, 8, 1e-6, True),
                                                     (3, 40, 0, 1e-6, False), (33, 0, 3, 1e-6, True)])
def test_against_the_formula(D, rot, interleaved, axes, tokens, hq, hk, eps, model):
    rope = B.make_rope(D, rot, interleaved=interleaved, axis_pairs=_pairs(rot, axes) if rot else [0] * axes, magnitude=1.1)
    g = torch.Generator().manual_seed(tokens * 1000 + rot)
    positions = torch.stack([torch.randint(-50, 5000, (tokens,), generator=g) for _ in range(axes)]).to(torch.int32).to(DEV)

    def tensor(h, seed):
        if h == 0:
            return None, None
        if model:                                                 # rows of a wider buffer, with a gap behind every token
            x = synth.randn_bf16((tokens, h + 2, D), seed, device=DEV)[:, 1:h + 1].transpose(0, 1)
            o = torch.full((tokens, h, D), float("nan"), dtype=torch.bfloat16, device=DEV).transpose(0, 1)
        else:
            x = synth.randn_bf16((h, tokens, D), seed, device=DEV)
            o = torch.full_like(x, float("nan"))
        return x, o

    (q, qo), (k, ko) = tensor(hq, 5), tensor(hk, 6)
    qw, kw = ((1 + 0.3 * synth.randn_bf16((D,), 7 + i).float()).to(torch.bfloat16).to(DEV) if h and eps else None for i, h in enumerate((hq, hk)))
    q0, k0 = (None if t is None else t.clone() for t in (q, k))
    B.pf_qk_norm_rope(rope, positions, q, qo, k, ko, q_weight=qw, k_weight=kw, eps=eps)
    torch.cuda.synchronize()
    for x, x0, o, w in ((q, q0, qo, qw), (k, k0, ko, kw)):
        if x is not None:
            assert torch.equal(x, x0)
            _check(o, x, w, positions, rope, eps)


@pytest.mark.gpu
def test_far_positions_and_stretched_contexts():
    D, n = 128, 64
    positions = torch.tensor([[0, 1, -1, 2 ** 30, -2 ** 30, 2 ** 31 - 1, -2 ** 31, 131071] * 8], dtype=torch.int32, device=DEV)
    for rope in (B.make_rope(D), B.make_rope(D, scaling="by_wavelength", factor=8.0, original_positions=8192), B.make_rope(D, base=1e6, scaling="linear", factor=3.0)):
        q, o = synth.randn_bf16((3, n, D), 1, device=DEV), torch.empty((3, n, D), dtype=torch.bfloat16, device=DEV)
        B.pf_qk_norm_rope(rope, positions, q, o, eps=1e-6)
        torch.cuda.synchronize()
        _check(o, q, None, positions, rope, 1e-6)


@pytest.mark.gpu
def test_in_place_equals_out_of_place_and_the_rest_of_the_buffer_stays():
    D, n, H = 128, 77, 6
    rope = B.make_rope(D, axis_pairs=[22, 21, 21], interleaved=True)
    positions = torch.arange(3 * n, dtype=torch.int32, device=DEV).view(3, n)
    wide = synth.randn_bf16((n + 3, 3 * H, D), 3, device=DEV)     # q, k and v of a fused projection; three rows behind the last token
    before = wide.clone()
    q, k = wide[:n, :H].transpose(0, 1), wide[:n, H:2 * H].transpose(0, 1)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    B.pf_qk_norm_rope(rope, positions, q, qo, k, ko, eps=1e-6)
    B.pf_qk_norm_rope(rope, positions, q, q, k, k, eps=1e-6)
    torch.cuda.synchronize()
    assert torch.equal(q, qo) and torch.equal(k, ko)
    assert torch.equal(wide[:, 2 * H:], before[:, 2 * H:]) and torch.equal(wide[n:], before[n:])


@pytest.mark.gpu
def test_host_tensors_are_refused():
    rope, pos = B.make_rope(64), torch.zeros((1, 3), dtype=torch.int32, device=DEV)
    q, w = synth.randn_bf16((2, 3, 64), 1, device=DEV), synth.randn_bf16((64,), 2, device=DEV)
    good = [pos, q, q.clone(), q.clone(), q.clone(), w, w]
    B.pf_qk_norm_rope(rope, *good, eps=1e-6)
    for i in range(7):
        with pytest.raises(AssertionError):
            B.pf_qk_norm_rope(rope, *(t.cpu() if j == i else t for j, t in enumerate(good)), eps=1e-6)
    torch.cuda.synchronize()


@pytest.mark.gpu
def test_zero_rows_and_rows_that_are_not_finite():
    """A row of zeros stays zero; a NaN or an infinity stays in its own row."""
    D = 64
    rope = B.make_rope(D)
    positions = torch.arange(5, dtype=torch.int32, device=DEV)[None]
    q = synth.randn_bf16((4, 5, D), 9, device=DEV)
    q[1, 2] = 0
    q[2, 3, 7] = float("nan")
    q[3, 4, 8] = float("inf")
    o = torch.empty_like(q)
    B.pf_qk_norm_rope(rope, positions, q, o, eps=1e-6)
    torch.cuda.synchronize()
    assert (o[1, 2] == 0).all() and torch.isnan(o[2, 3]).all()
    bad = torch.zeros((4, 5), dtype=torch.bool, device=DEV)
    bad[2, 3] = bad[3, 4] = True
    assert torch.isfinite(o[~bad]).all()


@pytest.mark.gpu
def test_another_stream_and_a_captured_graph():
    D, n = 128, 40
    rope = B.make_rope(D)
    positions = torch.arange(n, dtype=torch.int32, device=DEV)[None]
    q, o, want = synth.randn_bf16((4, n, D), 1, device=DEV), torch.empty((4, n, D), dtype=torch.bfloat16, device=DEV), torch.empty((4, n, D), dtype=torch.bfloat16, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.pf_qk_norm_rope(rope, positions, q, o, eps=1e-6)
    torch.cuda.current_stream().wait_stream(side)
    graph, go = torch.cuda.CUDAGraph(), torch.empty_like(o)
    with torch.cuda.graph(graph):
        B.pf_qk_norm_rope(rope, positions, q, go, eps=1e-6)
    for seed in (1, 2, 3):
        q.copy_(synth.randn_bf16((4, n, D), seed, device=DEV))
        positions.add_(seed)
        graph.replay()
        B.pf_qk_norm_rope(rope, positions, q, want, eps=1e-6)
        torch.cuda.synchronize()
        assert torch.equal(go, want)
        if seed == 1:
            _check(o, q, None, positions - 1, rope, 1e-6)


@pytest.mark.gpu
@pytest.mark.parametrize("D,rot,interleaved", [(128, 64, False), (128, 8, True), (64, 0, False), (64, 32, True), (64, 8, False)])
def test_channels_that_are_not_turned_keep_their_bits(D, rot, interleaved):
    """Without a norm the channels behind rot_dim come out as they went in, zeros' signs among them, whatever stands beside them."""
    rope = B.make_rope(D, rot, interleaved=interleaved, magnitude=1.5)
    q = synth.randn_bf16((3, 6, D), 4, device=DEV)
    q[0, :, rot::2], q[1, :, rot + 1::3], q[2, :, rot:] = float("inf"), float("nan"), -0.0
    q[2, :, rot + 3::4] = -1.0
    o = torch.zeros_like(q)
    B.pf_qk_norm_rope(rope, torch.arange(6, dtype=torch.int32, device=DEV)[None], q, o)
    torch.cuda.synchronize()
    a, b = (t[..., rot:].contiguous().view(torch.int16) for t in (q, o))
    assert torch.equal(a, b)
