"""Attention of packed sequences, alone and behind a shared prefix (pf_packed_plan, pf_packed_attn_fwd): refusals on the CPU, results on
the GPU against the definition in 64 bits."""
import ctypes
import math
import os

import pytest
import torch

from paper_2605_13111_amd import binding as B
from paper_2605_13111_amd import synth

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libpf.so not built")
DEV = "cuda:0"


def _cu(lengths):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return out


# ---- refusals ---------------------------------------------------------------------------------------------------------

def _struct(cu_q=(0, 5, 9), cu_k=(0, 5, 9), heads=4, kv=2, D=128, block=1, prefix=0, reserved=0, work=0x1000, work_bytes=1 << 20, seqs=None):
    a, b = (ctypes.c_int32 * len(cu_q))(*cu_q), (ctypes.c_int32 * len(cu_k))(*cu_k)
    I = ctypes.POINTER(ctypes.c_int32)
    s = B.pf_packed(len(cu_q) - 1 if seqs is None else seqs, heads, kv, D, block, prefix, reserved, 0, 0, -1, -1, 0, ctypes.cast(a, I), ctypes.cast(b, I), work, work_bytes)
    s._keep = (a, b)
    return s


BAD = [dict(cu_q=(1, 5, 9)), dict(cu_k=(1, 5, 9)), dict(cu_q=(0, 5, 4)), dict(cu_k=(0, 5, 4)), dict(heads=0), dict(kv=0), dict(kv=3), dict(heads=1026, kv=2),
       dict(block=-1), dict(prefix=-1), dict(prefix=(1 << 24) + 1), dict(reserved=1), dict(seqs=0), dict(seqs=(1 << 20) + 1), dict(cu_q=(0, 1, (1 << 24) + 1)),
       dict(cu_k=(0, 1, (1 << 30) + 1)), dict(cu_q=(0, 1, 1 << 22), heads=512)]


@pytest.mark.parametrize("kw", BAD)
def test_batches_refused(kw):
    s, L = _struct(**kw), B.lib()
    assert L.pf_packed_work_bytes(ctypes.byref(s)) == 0 and L.pf_packed_workspace_bytes(ctypes.byref(s)) == 0
    assert L.pf_packed_plan(ctypes.byref(s), None) == B.PF_ERR_INVALID_ARG
    fake = ctypes.c_void_p(0x10000)
    assert L.pf_packed_attn_fwd(ctypes.byref(s), fake, None, fake, fake, None, None, None, None, fake, None, 0.0, None, 0, None) == B.PF_ERR_INVALID_ARG


def test_plans_refused():
    L = B.lib()
    assert L.pf_packed_plan(None, None) == B.PF_ERR_INVALID_ARG and L.pf_packed_work_bytes(None) == 0
    assert L.pf_packed_plan(ctypes.byref(_struct(D=96)), None) == B.PF_ERR_UNSUPPORTED
    assert L.pf_packed_plan(ctypes.byref(_struct(work=0)), None) == B.PF_ERR_INVALID_ARG
    assert L.pf_packed_plan(ctypes.byref(_struct(work=0x1008)), None) == B.PF_ERR_INVALID_ARG
    s = _struct()
    need = L.pf_packed_work_bytes(ctypes.byref(s))
    assert need > 0
    s.work_bytes = need - 1
    assert L.pf_packed_plan(ctypes.byref(s), None) == B.PF_ERR_CAPACITY
    with pytest.raises(B.PfError) as e:
        B.Packed([0, 4], [0, 4], 4, 4, 96, device="cpu")
    assert e.value.status == B.PF_ERR_UNSUPPORTED


def _checksum(s):
    """64-bit FNV-1a over the words that a plan depends on."""
    h = 1469598103934665603
    words = [s.n_seqs, s.n_heads, s.n_kv_heads, s.head_dim, s.block, s.prefix_tokens, s.n_items, s.n_planes, s.kernel]
    for i in range(1, s.n_seqs + 1):
        words += [s.cu_q[i], s.cu_k[i]]
    for w in words:
        h = ((h ^ (w & 0xffffffff)) * 1099511628211) % 2 ** 64
    return h


def test_calls_refused_without_a_device():
    """A struct filled in as a plan would (no plan is uploaded: every refusal comes before anything is enqueued)."""
    L, bad, fake = B.lib(), B.PF_ERR_INVALID_ARG, 0x10000

    def call(s, q=fake, k=fake, v=fake, out=fake, kp=0, vp=0, ql=(512, 128), kl=(256, 128), pl=None, ol=None, scale=0.0, ws=0, ws_bytes=0):
        lay = lambda x: None if x is None else ctypes.byref(B.pf_chunk_layout(*x))
        return L.pf_packed_attn_fwd(ctypes.byref(s), q, lay(ql), k, v, lay(kl), kp, vp, lay(pl), out, lay(ql if ol is None else ol), scale, ws, ws_bytes, None)

    def planned(planes=0, **kw):
        s = _struct(**kw)
        s.n_items, s.n_planes, s.total_q, s.total_k = 4, planes, s._keep[0][len(s._keep[0]) - 1], s._keep[1][len(s._keep[1]) - 1]
        s.planned_for = _checksum(s)
        return s

    assert call(_struct()) == bad                                 # never planned
    empty = planned(cu_q=(0, 0, 0))
    assert call(empty, q=0, out=0) == B.PF_OK                     # no query, nothing enqueued
    s = planned()
    for kw in (dict(q=0), dict(k=0), dict(v=0), dict(out=0), dict(q=fake + 8), dict(k=fake + 2), dict(v=fake + 8), dict(out=fake + 8), dict(ql=(512, 127)),
               dict(ql=(256, 128)), dict(ol=(512, 120)), dict(ol=(384, 128)), dict(kl=(128, 128)), dict(ws=0x10008), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf"))):
        assert call(s, **kw) == bad, kw
    s = planned()
    s.total_k = 8                                                 # planned for other lengths
    assert call(s) == bad
    s = planned(work_bytes=64)                                    # four items do not fit
    assert call(s) == bad
    s = planned(work=0)
    assert call(s) == bad
    for field, x in (("n_heads", 2), ("n_kv_heads", 1), ("head_dim", 64), ("block", 2), ("prefix_tokens", 3), ("n_items", 3), ("n_planes", 1), ("kernel", 1)):
        s = planned()
        setattr(s, field, x)                                      # planned for something else
        assert call(s, kp=fake, vp=fake, ws=0x20000, ws_bytes=1 << 30) == bad, field
        assert L.pf_packed_workspace_bytes(ctypes.byref(s)) == 0
    s = planned()
    s._keep[0][1] = s._keep[1][1] = 6                             # other lengths of the same sum, written where the old ones were
    assert call(s) == bad
    assert call(planned(), kp=fake) == bad and call(planned(), vp=fake) == bad   # a prefix of no tokens
    assert L.pf_packed_workspace_bytes(ctypes.byref(_struct())) == 0
    s = planned(planes=2, prefix=10)
    need = 2 * 9 * 4 * (128 * 4 + 8)
    assert L.pf_packed_workspace_bytes(ctypes.byref(s)) >= need
    assert call(s, ws=0x20000, ws_bytes=need) == bad              # no prefix tensors
    assert call(s, kp=fake, vp=fake, pl=(256, 128)) == bad        # no workspace
    assert call(s, kp=fake, vp=fake, pl=(256, 128), ws=0x20000, ws_bytes=need - 1) == bad
    assert call(s, kp=fake, vp=fake, pl=(128, 128), ws=0x20000, ws_bytes=need) == bad


def test_a_buffer_that_was_not_planned_in_is_refused():
    """The plan stands in `work`: another buffer in its place, aligned and large enough, holds none.  Everything else is refused where it
    does stand there, too."""
    L, fake = B.lib(), 0x10000

    def call(work=0x1000, q=fake, k=fake, v=fake, out=fake, kp=0, ql=(512, 128), kl=(512, 128), ol=(512, 128), scale=0.0, ws=0, ws_bytes=0, planes=0):
        s = _struct(kv=4)
        s.n_items, s.n_planes, s.total_q, s.total_k = 4, planes, 9, 9
        s.planned_for, s.planned_in = _checksum(s), 0x1000
        s.work = work
        ql, kl, ol = (ctypes.byref(B.pf_chunk_layout(*x)) for x in (ql, kl, ol))
        return L.pf_packed_attn_fwd(ctypes.byref(s), q, ql, k, v, kl, kp, None, None, out, ol, scale, ws, ws_bytes, None)

    for kw in (dict(work=0x2000), dict(q=0), dict(k=0), dict(v=0), dict(out=0), dict(q=fake + 8), dict(k=fake + 2), dict(out=fake + 8), dict(kp=fake), dict(ql=(512, 127)),
               dict(ql=(256, 128)), dict(ol=(384, 128)), dict(kl=(128, 128)), dict(ws=0x10008), dict(scale=-1.0), dict(scale=float("nan")), dict(planes=2),
               dict(planes=2, ws=0x20000, ws_bytes=2 * 9 * 4 * (128 * 4 + 8) - 1)):
        assert call(**kw) == B.PF_ERR_INVALID_ARG, kw


def test_batches_of_too_many_items_are_refused():
    """8 heads of 2^20 sequences: a launch of 2^23 workgroups would have too many threads."""
    n = 1 << 20
    s, L = _struct(cu_q=tuple(range(n + 1)), cu_k=tuple(range(n + 1)), heads=8, kv=8), B.lib()
    assert L.pf_packed_work_bytes(ctypes.byref(s)) == 0
    assert L.pf_packed_plan(ctypes.byref(s), None) == B.PF_ERR_UNSUPPORTED


def test_tensors_of_another_device_are_refused():
    """Host memory instead of device memory never reaches a kernel."""
    with pytest.raises((AssertionError, RuntimeError)):
        B.pf_packed_plan(B.Packed([0, 4], [0, 4], 2, 2, 64, device="cpu"))


def test_totals_follow_the_lengths():
    """Lengths that are written over in place are the batch's lengths, for a caller who sizes tensors by them too."""
    packed = B.Packed([0, 4, 9], [0, 5, 12], 2, 2, 64, device="cpu")
    assert (packed.total_q, packed.total_k) == (9, 12)
    packed.cu_k[1], packed.cu_k[2] = 6, 14
    packed.cu_q[2] = 8
    assert (packed.total_q, packed.total_k) == (8, 14)


@pytest.mark.parametrize("kw", [dict(cu_q=[0, 2 ** 32 + 5]), dict(cu_k=[0, 2 ** 32 + 5]), dict(block=2 ** 32), dict(prefix_tokens=2 ** 32), dict(n_heads=2 ** 32 + 2)])
def test_numbers_beyond_32_bits_are_refused(kw):
    """Cut down to the struct's 32 bits, each of these would be another batch: fewer tokens, no mask, no prefix."""
    args = dict(cu_q=[0, 5], cu_k=[0, 5], n_heads=2, n_kv_heads=2, head_dim=64)
    B.Packed(**args, device="cpu")
    with pytest.raises(B.PfError) as e:
        B.Packed(**{**args, **kw}, device="cpu")
    assert e.value.status == B.PF_ERR_INVALID_ARG


# ---- results ----------------------------------------------------------------------------------------------------------

def _definition(q, k, v, cu_q, cu_k, block, kp=None, vp=None, scale=None):
    """q [H, tq, D], k / v [KV, tk, D], kp / vp [KV, P, D] -> out [H, tq, D] in 64 bits and the error that the kernel's arithmetic may have:
      every weight rounded to bf16 (2^-8 of what it multiplies) and the result too (2^-8 of itself);
      a score off by (D + 4) 2^-24 of the sum of its products' sizes, plus 2^-20 for the exponent's argument and the power, which
      moves a weight by that factor, numerator and sum alike; n additions of 2^-24 each."""
    H, tq, D = q.shape
    G, scale = H // k.shape[0], D ** -0.5 if scale is None else scale
    out, tol = torch.zeros((H, tq, D), dtype=torch.float64, device=q.device), torch.zeros((H, tq, D), dtype=torch.float64, device=q.device)
    for s in range(len(cu_q) - 1):
        q0, q1, k0, k1 = cu_q[s], cu_q[s + 1], cu_k[s], cu_k[s + 1]
        for h in range(H):
            K, V, P = k[h // G, k0:k1].double(), v[h // G, k0:k1].double(), 0
            if kp is not None:
                P = kp.shape[1]
                K, V = torch.cat([kp[h // G].double(), K]), torch.cat([vp[h // G].double(), V])
            if q1 == q0 or K.shape[0] == 0:
                continue
            x = q[h, q0:q1].double() @ K.T * scale
            seen = torch.ones(x.shape, dtype=torch.bool, device=q.device)
            if block:
                place = torch.arange(q1 - q0, device=q.device) + (k1 - k0) - (q1 - q0)
                j = torch.arange(K.shape[0], device=q.device) - P
                seen = (j[None] < 0) | (torch.div(j[None], block, rounding_mode="floor") <= torch.div(place[:, None], block, rounding_mode="floor"))
            x = torch.where(seen, x, -math.inf)
            some = seen.any(1, keepdim=True)
            w = torch.where(some, torch.softmax(x, 1), 0.0)
            V0 = torch.where(seen.any(0)[:, None], V, 0.0)
            out[h, q0:q1] = w @ V0
            size = torch.where(seen, (q[h, q0:q1].double().abs() @ K.abs().T) * scale, 0.0).amax(1, keepdim=True)
            d = size * (D + 4) * 2.0 ** -24 + 2.0 ** -20
            A = w @ V0.abs()
            tol[h, q0:q1] = 2.0 ** -8 * out[h, q0:q1].abs() + A * (1 + 2.0 ** -8) * (2.0 ** -8 + 2 * d + K.shape[0] * 2.0 ** -24) + 1e-38
    return out, tol


def _tensors(H, KV, D, tq, tk, P, seed, model, spare=0, gain=1.0):
    def make(h, n, s):
        n += spare
        if model:
            return synth.randn_bf16((n, h, D), s, device=DEV).transpose(0, 1)
        return synth.randn_bf16((h, n, D), s, device=DEV)
    q, k, v = make(H, tq, seed) * gain, make(KV, tk, seed + 1), make(KV, tk, seed + 2)
    spare = 0
    kp, vp = (make(KV, P, seed + 3), make(KV, P, seed + 4)) if P else (None, None)
    return q, k, v, kp, vp


def _run(cu_q, cu_k, q, k, v, block, kp=None, vp=None, scale=0.0):
    packed = B.Packed(cu_q, cu_k, q.shape[0], k.shape[0], q.shape[2], block=block, prefix_tokens=0 if kp is None else kp.shape[1], device=DEV)
    B.pf_packed_plan(packed)
    # what an earlier use left in the workspace must not matter
    ws = torch.full((B.pf_packed_workspace_bytes(packed),), 255, dtype=torch.uint8, device=DEV)
    out = torch.full_like(q, float("nan"))
    B.pf_packed_attn_fwd(packed, q, k, v, out, ws, kp, vp, softmax_scale=scale)
    again = torch.full_like(q, float("nan"))
    B.pf_packed_attn_fwd(packed, q, k, v, again, ws, kp, vp, softmax_scale=scale)
    torch.cuda.synchronize()
    n = cu_q[-1]
    assert torch.equal(out[:, :n].contiguous().view(torch.int16), again[:, :n].contiguous().view(torch.int16))
    return out


def _case(cu_q, cu_k, H, KV, D, block, P, seed=1, model=True, gain=1.0, scale=None, spare=0):
    q, k, v, kp, vp = _tensors(H, KV, D, cu_q[-1], cu_k[-1], P, seed, model, spare, gain)
    out = _run(cu_q, cu_k, q, k, v, block, kp, vp, 0.0 if scale is None else scale)
    want, tol = _definition(q, k, v, cu_q, cu_k, block, kp, vp, scale)
    n = cu_q[-1]
    assert torch.isfinite(out[:, :n]).all()
    over = (out[:, :n].double() - want[:, :n]).abs() - tol[:, :n]
    assert over.max() <= 0 if over.numel() else True, "off by %.3g more than allowed" % float(over.max())
    return out, want


LENGTHS = {
    "one": ([1], [1]), "token": ([1], [777]), "tile": ([64], [64]), "odd": ([65, 1, 130], [65, 1, 130]), "empties": ([0, 5, 3, 0, 1], [5, 5, 0, 0, 129]),
    "long_queries": ([200, 7], [100, 3]), "late": ([3, 129, 33], [400, 257, 1000]), "steps": ([1] * 9, [1, 2, 63, 64, 65, 500, 0, 7, 128]),
}


@pytest.mark.gpu
@pytest.mark.parametrize("name", sorted(LENGTHS))
@pytest.mark.parametrize("H,KV,D", [(3, 3, 128), (8, 2, 128), (5, 1, 64), (4, 4, 64)])
@pytest.mark.parametrize("block,P", [(0, 0), (1, 0), (48, 0), (1, 70), (100, 1), (0, 256)])
def test_against_the_definition(name, H, KV, D, block, P):
    lq, lk = LENGTHS[name]
    _case(_cu(lq), _cu(lk), H, KV, D, block, P, model=(block + P) % 2 == 0)


@pytest.mark.gpu
@pytest.mark.parametrize("H,KV,D", [(4, 4, 128), (16, 2, 64), (24, 3, 128)])
@pytest.mark.parametrize("block,P", [(1, 0), (300, 0), (1, 1500), (0, 0)])
def test_longer_sequences(H, KV, D, block, P):
    lq = [1300, 513, 257, 1]
    _case(_cu(lq), _cu(lq), H, KV, D, block, P, seed=3)


@pytest.mark.gpu
@pytest.mark.parametrize("lq,lk,P,block", [
    ([1300, 513, 257, 1], None, 0, 1), ([1300, 513, 257, 1], None, 1500, 1), ([1000, 700], None, 0, 300), ([64, 900, 0, 255], [64, 2900, 70, 255], 0, 1),
    ([900, 900], [200, 700], 0, 1), ([901], [901], 130, 0), ([129, 300, 40], [1000, 1000, 1000], 64, 48), ([1200], [1200], 0, 2 ** 31 - 1)])
def test_launches_of_wide_items(lq, lk, P, block):
    """Enough work for items of 256 rows (head_dim 128): rows that end inside an item, rows that see nothing, a wave of a tile each with an end
    of its own, prefixes that end inside a tile."""
    lk = lq if lk is None else lk
    D = 128
    for KV, G in [(n, g) for g in (2, 5, 1) for n in range(8, 65, 4)]:   # the first numbers of heads that the planner takes wide items for
        packed = B.Packed(_cu(lq), _cu(lk), KV * G, KV, D, block=block, prefix_tokens=P, device=DEV)
        B.pf_packed_plan(packed)
        if packed.c.kernel == 1:
            break
    assert packed.c.kernel == 1, "the case must go by wide items"
    _case(_cu(lq), _cu(lk), KV * G, KV, D, block, P, seed=17)


@pytest.mark.gpu
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("seqs,P,H,KV", [(1, 0, 8, 1), (1, 9000, 4, 4), (40, 3333, 8, 2), (150, 129, 2, 2)])
def test_single_tokens_of_many_sequences(D, seqs, P, H, KV):
    lk = [1 + (i * 37) % 200 for i in range(seqs)] if seqs > 1 else [20000]
    _case(_cu([1] * seqs), _cu(lk), H, KV, D, 1, P, seed=5)


@pytest.mark.gpu
@pytest.mark.parametrize("gain,scale", [(60.0, None), (1.0, 3.0), (1.0, 1e-4), (30.0, 20.0), (1.0, 1e-30)])
@pytest.mark.parametrize("D", [64, 128])
def test_sharp_and_flat_softmax(gain, scale, D):
    """Scores far apart: the reference maximum moves many times; masked tiles in front of it."""
    _case(_cu([100, 300]), _cu([100, 300]), 4, 2, D, 1, 90, seed=7, gain=gain, scale=scale)


@pytest.mark.gpu
def test_host_tensors_are_refused():
    cu = [0, 7]
    q, k, v, kp, vp = _tensors(2, 2, 64, 7, 7, 5, 1, True)
    packed = B.Packed(cu, cu, 2, 2, 64, prefix_tokens=5, device=DEV)
    B.pf_packed_plan(packed)
    ws = torch.empty(B.pf_packed_workspace_bytes(packed), dtype=torch.uint8, device=DEV)
    good = [q, k, v, torch.empty_like(q), ws, kp, vp]
    B.pf_packed_attn_fwd(packed, *good)
    for i in range(7):
        with pytest.raises(AssertionError):
            B.pf_packed_attn_fwd(packed, *(t.cpu() if j == i else t for j, t in enumerate(good)))
    torch.cuda.synchronize()


@pytest.mark.gpu
def test_a_buffer_replaced_beside_the_struct_is_refused():
    """The struct holds an address; the tensor that it belongs to has to be the batch's still."""
    cu = [0, 7]
    q, k, v, _, _ = _tensors(2, 2, 64, 7, 7, 0, 1, True)
    packed = B.Packed(cu, cu, 2, 2, 64, device=DEV)
    B.pf_packed_plan(packed)
    ws, out, kept = torch.empty(B.pf_packed_workspace_bytes(packed), dtype=torch.uint8, device=DEV), torch.empty_like(q), packed.work
    packed.work = torch.zeros_like(kept)
    with pytest.raises(AssertionError):
        B.pf_packed_attn_fwd(packed, q, k, v, out, ws)
    with pytest.raises(AssertionError):
        B.pf_packed_plan(packed)
    packed.work = kept
    B.pf_packed_attn_fwd(packed, q, k, v, out, ws)
    assert torch.isfinite(out).all()


@pytest.mark.gpu
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("P", [0, 100])
def test_rows_behind_the_last_sequence(D, P):
    """Tensors longer than the batch: what lies behind may be anything and stays as it is."""
    cu = _cu([70, 33])
    q, k, v, kp, vp = _tensors(4, 2, D, 103, 103, P, 11, True, spare=40)
    kp, vp = (None, None) if P == 0 else (kp[:, :P], vp[:, :P])
    k[:, 103:], v[:, 103:] = float("nan"), float("inf")
    out = _run(cu, cu, q, k, v, 1, kp, vp)
    want, tol = _definition(q[:, :103], k[:, :103], v[:, :103], cu, cu, 1, kp, vp)
    assert ((out[:, :103].double() - want).abs() <= tol).all() and torch.isnan(out[:, 103:]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf"), -3.0e38])
@pytest.mark.parametrize("D", [64, 128])
def test_masked_keys_do_not_count(bad, D):
    """K of later tokens may hold anything: the rows that do not see them have the bits that they had."""
    cu = _cu([200])
    q, k, v, _, _ = _tensors(4, 4, D, 200, 200, 0, 13, False)
    out = _run(cu, cu, q, k, v, 1)
    k[:, 77:] = bad
    got = _run(cu, cu, q, k, v, 1)
    assert torch.equal(got[:, :77], out[:, :77])


def _wide(lq, lk, G, block, P=0):
    """The first number of key heads that the planner takes wide items for."""
    for KV in range(8, 65, 4):
        packed = B.Packed(_cu(lq), _cu(lk), KV * G, KV, 128, block=block, prefix_tokens=P, device=DEV)
        B.pf_packed_plan(packed)
        if packed.c.kernel == 1:
            return KV
    raise AssertionError("the case must go by wide items")


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [float("nan"), -float("inf"), -3.0e38])
def test_masked_keys_do_not_count_in_wide_items(bad):
    lq = [1200]
    KV, cu = _wide(lq, lq, 1, 1), _cu(lq)
    q, k, v, _, _ = _tensors(KV, KV, 128, 1200, 1200, 0, 13, True)
    out = _run(cu, cu, q, k, v, 1)
    k[:, 777:] = bad
    got = _run(cu, cu, q, k, v, 1)
    assert torch.equal(got[:, :777], out[:, :777])


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("D,n", [(64, 300), (128, 300), (128, 1200)])
def test_a_query_that_is_not_a_number_stays_alone(D, n, bad):
    """The other rows of its tile, and of the waves beside it, have the bits that they had."""
    KV, cu = (_wide([n], [n], 1, 1) if n == 1200 else 3), _cu([n])
    q, k, v, kp, vp = _tensors(KV, KV, D, n, n, 0 if n == 1200 else 70, 37, True)
    out = _run_bits(cu, q, k, v, kp, vp)
    q[1, 133] = bad
    got = _run_bits(cu, q, k, v, kp, vp)
    same = got == out
    assert torch.isnan(got[1, 133].view(torch.bfloat16)).all()
    same[1, 133] = True
    assert same.all()


def _run_bits(cu, q, k, v, kp, vp):
    packed = B.Packed(cu, cu, q.shape[0], k.shape[0], q.shape[2], block=1, prefix_tokens=0 if kp is None else kp.shape[1], device=DEV)
    B.pf_packed_plan(packed)
    ws, out = torch.zeros(B.pf_packed_workspace_bytes(packed), dtype=torch.uint8, device=DEV), torch.empty(q.shape, dtype=torch.bfloat16, device=DEV)
    B.pf_packed_attn_fwd(packed, q, k, v, out, ws, kp, vp)
    torch.cuda.synchronize()
    return out.view(torch.int16)


@pytest.mark.gpu
def test_rows_behind_the_last_sequence_of_wide_items():
    lq = [1100, 77]
    KV, cu, n = _wide(lq, lq, 2, 1), _cu(lq), 1177
    q, k, v, _, _ = _tensors(2 * KV, KV, 128, n, n, 0, 19, True, spare=300)
    k[:, n:], v[:, n:] = float("nan"), float("inf")
    out = _run(cu, cu, q, k, v, 1)
    want, tol = _definition(q[:, :n], k[:, :n], v[:, :n], cu, cu, 1)
    assert ((out[:, :n].double() - want).abs() <= tol).all() and torch.isnan(out[:, n:]).all()


@pytest.mark.gpu
def test_wide_items_beyond_32_bits():
    """Sequences behind one of 1 100 000 keys (and no query): they lie beyond 2^32 bytes of K and V."""
    lq, lk, D = [0, 1100, 77], [1100000, 1100, 77], 128
    KV = _wide(lq, lk, 2, 1)
    assert 1100000 * KV * D * 2 > 2 ** 32
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    k = torch.empty((sum(lk), KV, D), dtype=torch.bfloat16, device=DEV)
    v = torch.empty_like(k)
    for t in (k, v):
        for i in range(0, sum(lk), 50000):
            t[i:i + 50000] = torch.randn(t[i:i + 50000].shape, generator=g, device=DEV).to(torch.bfloat16)
    k, v = k.transpose(0, 1), v.transpose(0, 1)
    q = synth.randn_bf16((sum(lq), 2 * KV, D), 5, device=DEV).transpose(0, 1)
    out = _run(_cu(lq), _cu(lk), q, k, v, 1)
    want, tol = _definition(q, k, v, _cu(lq), _cu(lk), 1)
    assert ((out.double() - want).abs() <= tol).all()


@pytest.mark.gpu
@pytest.mark.parametrize("D", [64, 128])
def test_more_planes_than_a_wave_has_lanes(D):
    cu_q, cu_k = _cu([1]), _cu([40001])
    packed = B.Packed(cu_q, cu_k, 40, 1, D, block=1, device=DEV)
    B.pf_packed_plan(packed)
    assert packed.c.n_planes > 64, "the case must park many partial results"
    _case(cu_q, cu_k, 40, 1, D, 1, 0, seed=23)


@pytest.mark.gpu
@pytest.mark.parametrize("lq,lk,H,KV,P,parked", [
    ([88920, 1], [88920, 1], 24, 12, 2048, 1), ([30000] + [1] * 4, [30000] + [50] * 4, 32, 8, 4096, 4), ([2048] * 7 + [1], [2048] * 7 + [500000], 32, 8, 0, 1),
    ([2000] * 4 + [1] * 4, [2000] * 4 + [131072] * 4, 32, 8, 0, 4)])
def test_workspace_holds_the_rows_that_park(lq, lk, H, KV, P, parked):
    """Prompts whose rows have one item each, beside single tokens whose keys are split: partial results of the tokens only."""
    D = 128
    packed = B.Packed(_cu(lq), _cu(lk), H, KV, D, block=1, prefix_tokens=P, device=DEV)
    B.pf_packed_plan(packed)
    assert packed.c.n_planes > 1, "the case must park partial results"
    assert B.pf_packed_workspace_bytes(packed) <= parked * H * (packed.c.n_planes * (D * 4 + 8) + 4) + 512


@pytest.mark.gpu
@pytest.mark.parametrize("lq,lk,P", [([600] * 3 + [1] * 4, [600] * 3 + [50000] * 4, 0), ([700, 1, 900, 1, 1], [700, 9000, 900, 40, 8000], 500),
                                     ([1, 300, 1, 0, 2, 129], [7000, 300, 1, 50, 9000, 129], 0), ([1, 1, 2000, 3, 1], [100, 300, 2000, 90, 0], 6000)])
@pytest.mark.parametrize("H,KV,D", [(8, 2, 128), (8, 2, 64), (3, 3, 128)])
def test_prompts_beside_single_tokens_of_many_keys(lq, lk, P, H, KV, D):
    packed = B.Packed(_cu(lq), _cu(lk), H, KV, D, block=1, prefix_tokens=P, device=DEV)
    B.pf_packed_plan(packed)
    assert packed.c.n_planes > 1, "the case must park partial results"
    _case(_cu(lq), _cu(lk), H, KV, D, 1, P, seed=91)


def _dead(k, dead):
    """Keys with a score of minus infinity for queries whose first channel is positive."""
    k[:, dead, 0] = -float("inf")
    return k


@pytest.mark.gpu
@pytest.mark.parametrize("which", ["all", "own", "prefix", "first half"])
@pytest.mark.parametrize("lq,lk,H,KV,D,P,block", [
    ([70, 5, 9], [70, 5, 4], 4, 2, 64, 0, 1), ([300, 20], [300, 15], 3, 3, 128, 100, 1), ([1] * 4, [900, 3, 0, 64], 4, 2, 128, 700, 1), ([1], [5000], 4, 1, 64, 0, 1),
    ([1] * 40, [70] * 40, 8, 2, 64, 3000, 0), ([1], [20001], 40, 1, 128, 0, 1), ([1200], [1200], 0, 0, 128, 0, 1), ([1200], [1100], 0, 0, 128, 200, 300)])
def test_scores_of_minus_infinity(which, lq, lk, H, KV, D, P, block):
    """Keys whose score is minus infinity weigh nothing; a row that sees no other has no softmax (NaN), one that sees none at all is zero."""
    if H == 0:
        H = KV = _wide(lq, lk, 1, block, P)
    cu_q, cu_k = _cu(lq), _cu(lk)
    q, k, v, kp, vp = _tensors(H, KV, D, cu_q[-1], cu_k[-1], P, 97, True)
    q[..., 0] = q[..., 0].abs() + 0.5
    dead = torch.ones(cu_k[-1], dtype=torch.bool, device=DEV)
    if which == "prefix":
        dead[:] = False
    if which == "first half":
        for a, b in zip(cu_k, cu_k[1:]):
            dead[(a + b) // 2:b] = False
    dead_p = torch.full((P,), which in ("all", "prefix"), dtype=torch.bool, device=DEV)
    alive = k.clone(), None if kp is None else kp.clone()
    k = _dead(k, dead)
    kp = None if kp is None else _dead(kp, dead_p)
    out = _run(cu_q, cu_k, q, k, v, block, kp, vp).double()
    G = H // KV
    for s in range(len(lq)):
        place = torch.arange(lq[s], device=DEV) + lk[s] - lq[s]
        j = torch.arange(lk[s], device=DEV)
        seen = torch.ones((lq[s], lk[s]), dtype=torch.bool, device=DEV)
        if block:
            seen = torch.div(j[None], block, rounding_mode="floor") <= torch.div(place[:, None], block, rounding_mode="floor")
        seen = torch.cat([torch.ones((lq[s], P), dtype=torch.bool, device=DEV), seen], 1)
        live = seen & ~torch.cat([dead_p, dead[cu_k[s]:cu_k[s + 1]]])[None]
        none, lost = ~seen.any(1), seen.any(1) & ~live.any(1)
        for h in range(H):
            got = out[h, cu_q[s]:cu_q[s + 1]]
            assert (got[none] == 0).all() and torch.isnan(got[lost]).all()
            K, V = alive[0][h // G, cu_k[s]:cu_k[s + 1]].double(), v[h // G, cu_k[s]:cu_k[s + 1]].double()
            if P:
                K, V = torch.cat([alive[1][h // G].double(), K]), torch.cat([vp[h // G].double(), V])
            rest = live.any(1)
            if not rest.any():
                continue
            Q = q[h, cu_q[s]:cu_q[s + 1]].double()[rest]
            w = torch.softmax(torch.where(live[rest], Q @ K.T * D ** -0.5, -math.inf), 1)
            d = (Q.abs() @ K.abs().T).amax(1, keepdim=True) * D ** -0.5 * (D + 4) * 2.0 ** -24 + 2.0 ** -20   # as in _definition
            tol = 2.0 ** -8 * (w @ V).abs() + (w @ V.abs()) * (1 + 2.0 ** -8) * (2.0 ** -8 + 2 * d + K.shape[0] * 2.0 ** -24) + 1e-38
            assert ((got[rest] - w @ V).abs() <= tol).all()


def _tile_channels(cu_k, KV, D, P, device):
    """Values that say which tile of 64 keys they are from: key j of tile t (the prefix's tiles, then the sequence's own) has a value in channel t % D
    only.  A tile left out takes its share of one channel, whatever the length."""
    def values(tile):
        v = torch.zeros((tile.shape[0], KV, D), dtype=torch.bfloat16)
        v[torch.arange(tile.shape[0]), :, tile % D] = 1.0
        return v.to(device).transpose(0, 1)
    pre = (P + 63) // 64
    own = torch.cat([pre + torch.arange(b - a) // 64 for a, b in zip(cu_k, cu_k[1:])])
    return values(own), values(torch.arange(P) // 64) if P else None


LONG = [([1], [20000], 8, 1, 0), ([1], [40001], 40, 1, 0), ([1], [65536], 8, 8, 0), ([1] * 3, [9000, 130, 20001], 4, 4, 9000), ([1] * 40, [70] * 40, 8, 2, 20000),
        ([5, 1, 2], [30000, 9, 64], 2, 2, 5000), ([900, 1, 1], [900, 30000, 12000], 4, 2, 0)]


@pytest.mark.parametrize("D", [64, 128])
def test_a_lost_tile_would_be_seen(D):
    """The bound that results are held to is passed twice over by any one tile of 64 keys left out of the definition, at the longest of these lengths."""
    n = 65536
    g = torch.Generator().manual_seed(5)
    q, k = torch.randn((1, 1, D), generator=g).to(torch.bfloat16), torch.randn((1, n, D), generator=g).to(torch.bfloat16)
    v, _ = _tile_channels([0, n], 1, D, 0, "cpu")
    want, tol = _definition(q, k, v, [0, 1], [0, n], 1)
    w = torch.softmax(k[0].double() @ q[0, 0].double() * D ** -0.5, 0).view(-1, 64).sum(1)
    channel = torch.arange(n // 64) % D
    share = want[0, 0, channel]
    without = (share - w) / (1 - w)                               # the tile's channel once the tile is lost, the other weights' sum taken as all
    assert ((share - without) > 2 * tol[0, 0, channel]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("lq,lk,H,KV,P", LONG)
@pytest.mark.parametrize("D", [64, 128])
def test_every_tile_counts(lq, lk, H, KV, P, D):
    cu_q, cu_k = _cu(lq), _cu(lk)
    q, k, _, kp, _ = _tensors(H, KV, D, cu_q[-1], cu_k[-1], P, 57, True)
    v, vp = _tile_channels(cu_k, KV, D, P, DEV)
    out = _run(cu_q, cu_k, q, k, v, 1, kp, vp)
    want, tol = _definition(q, k, v, cu_q, cu_k, 1, kp, vp)
    assert torch.isfinite(out).all() and ((out.double() - want).abs() <= tol).all()


@pytest.mark.gpu
def test_every_tile_counts_in_wide_items():
    lq, D = [4801, 130], 128
    KV, cu = _wide(lq, lq, 1, 1), _cu(lq)
    q, k, _, _, _ = _tensors(KV, KV, D, cu[-1], cu[-1], 0, 57, True)
    v, _ = _tile_channels(cu, KV, D, 0, DEV)
    out = _run(cu, cu, q, k, v, 1)
    want, tol = _definition(q, k, v, cu, cu, 1)
    assert torch.isfinite(out).all() and ((out.double() - want).abs() <= tol).all()


@pytest.mark.gpu
def test_lengths_that_change_need_a_plan():
    """The lengths of a batch written over in place: refused until planned again, right afterwards."""
    packed = B.Packed(_cu([70, 30]), _cu([70, 30]), 4, 2, 64, block=1, device=DEV)
    q, k, v, _, _ = _tensors(4, 2, 64, 100, 100, 0, 29, True)
    out = torch.empty_like(q)
    B.pf_packed_plan(packed)
    ws = torch.empty(1 << 22, dtype=torch.uint8, device=DEV)
    B.pf_packed_attn_fwd(packed, q, k, v, out, ws)
    packed.cu_q[1] = packed.cu_k[1] = 20
    with pytest.raises(B.PfError):
        B.pf_packed_attn_fwd(packed, q, k, v, out, ws)
    B.pf_packed_plan(packed)
    assert B.pf_packed_workspace_bytes(packed) <= ws.numel()
    B.pf_packed_attn_fwd(packed, q, k, v, out, ws)
    want, tol = _definition(q, k, v, [0, 20, 100], [0, 20, 100], 1)
    assert ((out.double() - want).abs() <= tol).all()
    packed.cu_k[2] = 103                                          # three keys more than the tensors have
    B.pf_packed_plan(packed)
    with pytest.raises(AssertionError):
        B.pf_packed_attn_fwd(packed, q, k, v, out, ws)
    k, v = (torch.cat([t, t[:, :3]], 1) for t in (k, v))
    assert B.pf_packed_workspace_bytes(packed) <= ws.numel()
    B.pf_packed_attn_fwd(packed, q, k, v, out, ws)
    want, tol = _definition(q, k, v, [0, 20, 100], [0, 20, 103], 1)
    assert ((out.double() - want).abs() <= tol).all()


@pytest.mark.gpu
def test_another_buffer_needs_a_plan():
    cu = _cu([70, 30])
    packed = B.Packed(cu, cu, 4, 2, 64, block=1, device=DEV)
    q, k, v, _, _ = _tensors(4, 2, 64, 100, 100, 0, 29, True)
    out = torch.empty_like(q)
    B.pf_packed_plan(packed)
    ws = torch.empty(B.pf_packed_workspace_bytes(packed), dtype=torch.uint8, device=DEV)
    B.pf_packed_attn_fwd(packed, q, k, v, out, ws)
    want = out.clone()
    packed.work = torch.zeros_like(packed.work)
    packed.c.work = packed.work.data_ptr()
    with pytest.raises(B.PfError):
        B.pf_packed_attn_fwd(packed, q, k, v, out, ws)
    B.pf_packed_plan(packed)
    B.pf_packed_attn_fwd(packed, q, k, v, out.zero_(), ws)
    torch.cuda.synchronize()
    assert torch.equal(out, want)


PLANS = {  # lengths of queries, of keys, heads, key heads, head_dim, prefix: full, thin (joined by the last workgroup, or by a second launch), wide
    "full": ([300, 41], [300, 41], 4, 2, 64, 0), "arrival": ([1] * 4, [900] * 4, 4, 2, 128, 700), "joined": ([1] * 40, [70] * 40, 8, 2, 128, 3000),
    "wide": ([1200], [1200], 0, 0, 128, 0), "tiny": ([1], [1], 1, 1, 64, 0)}


def _planned(name, work=None):
    lq, lk, H, KV, D, P = PLANS[name]
    if name == "wide":
        H = KV = _wide(lq, lk, 1, 1)
    packed = B.Packed(_cu(lq), _cu(lk), H, KV, D, block=1, prefix_tokens=P, device=DEV)
    if work is not None:
        assert packed.c.work_bytes <= work.numel()
        packed.work = work
        packed.c.work, packed.c.work_bytes = work.data_ptr(), work.numel()
    q, k, v, kp, vp = _tensors(H, KV, D, sum(lq), sum(lk), P, 83, True)
    ws = torch.empty(1 << 27, dtype=torch.uint8, device=DEV)

    def call(out):
        B.pf_packed_attn_fwd(packed, q, k, v, out, ws, kp, vp)
    return packed, call, torch.zeros((sum(lq), H, D), dtype=torch.bfloat16, device=DEV).transpose(0, 1)


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["full", "arrival", "joined", "wide", "tiny"])
@pytest.mark.parametrize("other", ["full", "arrival", "wide", "tiny"])
def test_a_buffer_holds_its_last_plan_only(name, other):
    """Two batches that share the plan's buffer: a call under the plan that is not there any more, eager or in a graph captured while it was, says so in
    every row; planned again, the same graph is right again."""
    packed, call, out = _planned(name)
    B.pf_packed_plan(packed)
    assert B.pf_packed_workspace_bytes(packed) <= 1 << 27
    assert packed.c.kernel == int(name == "wide") and (packed.c.n_planes > 0) == (name in ("arrival", "joined"))
    call(out)
    want = out.clone()
    work = torch.zeros(1 << 22, dtype=torch.uint8, device=DEV)
    (packed, call, out), (second, call2, out2) = _planned(name, work), _planned(other, work)
    B.pf_packed_plan(packed)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    graph.replay()
    assert torch.equal(out, want)
    if other == name:                                             # the same batch: the same plan, whichever struct it was planned for last
        B.pf_packed_plan(second)
        graph.replay()
        assert torch.equal(out, want)
        call2(out2)
        assert torch.equal(out2, want)
        return
    for _ in range(2):
        B.pf_packed_plan(second)
        before = work.clone()
        call(out.zero_())
        assert torch.isnan(out).all()
        out.zero_()
        graph.replay()
        assert torch.isnan(out).all() and torch.equal(work, before)
        call2(out2)
        assert torch.isfinite(out2).all()
        B.pf_packed_plan(packed)
        graph.replay()
        assert torch.equal(out, want)
        call(out.zero_())
        assert torch.equal(out, want)


@pytest.mark.gpu
def test_a_plan_that_is_not_there_yet():
    """Captured, a plan reaches its buffer with the first replay."""
    packed, call, out = _planned("joined")
    packed.work.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.pf_packed_plan(packed)
    call(out)
    assert torch.isnan(out).all()
    graph.replay()
    call(out)
    assert torch.isfinite(out).all()


@pytest.mark.gpu
def test_gaps_between_rows_and_heads():
    """q, k and v as slices of one projection, the results as a slice of a wider buffer."""
    H, KV, D, n = 6, 3, 128, 150
    cu = _cu([100, 50])
    wide = synth.randn_bf16((n, H + 2 * KV + 1, D), 21, device=DEV)
    q, k, v = (wide[:, a:b].transpose(0, 1) for a, b in ((0, H), (H, H + KV), (H + KV, H + 2 * KV)))
    buf = torch.zeros((n, H + 2 * KV + 1, D), dtype=torch.bfloat16, device=DEV)
    packed = B.Packed(cu, cu, H, KV, D, block=1, device=DEV)
    B.pf_packed_plan(packed)
    ws = torch.empty(B.pf_packed_workspace_bytes(packed), dtype=torch.uint8, device=DEV)
    B.pf_packed_attn_fwd(packed, q, k, v, buf[:, :H].transpose(0, 1), ws)
    torch.cuda.synchronize()
    want, tol = _definition(q, k, v, cu, cu, 1)
    assert ((buf[:, :H].transpose(0, 1).double() - want).abs() <= tol).all() and (buf[:, H:] == 0).all()


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    """Keys of 64 heads by 300 000 tokens: 2.4e9 elements a tensor; the last sequence lies beyond 2^32 bytes."""
    KV, D, tk = 64, 128, 300000
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    k = torch.empty((tk, KV, D), dtype=torch.bfloat16, device=DEV)
    v = torch.empty_like(k)
    for t in (k, v):
        for i in range(0, tk, 50000):
            t[i:i + 50000] = torch.randn((50000, KV, D), generator=g, device=DEV).to(torch.bfloat16)
    k, v = k.transpose(0, 1), v.transpose(0, 1)
    cu_q, cu_k = _cu([1, 2, 40]), _cu([1000, 298000, 1000])
    q = synth.randn_bf16((43, KV, D), 5, device=DEV).transpose(0, 1)
    out = _run(cu_q, cu_k, q, k, v, 1)
    want, tol = _definition(q, k, v, cu_q, cu_k, 1)
    assert ((out.double() - want).abs() <= tol).all()


@pytest.mark.gpu
def test_streams_graphs_and_two_batches_at_once():
    H, KV, D = 8, 2, 128
    cu_a, cu_b = _cu([300, 41]), _cu([1] * 12)
    cu_bk = _cu([50 + i for i in range(12)])
    qa, ka, va, _, _ = _tensors(H, KV, D, cu_a[-1], cu_a[-1], 0, 31, True)
    qb, kb, vb, kp, vp = _tensors(H, KV, D, cu_b[-1], cu_bk[-1], 700, 41, True)
    want_a, want_b = _run(cu_a, cu_a, qa, ka, va, 1), _run(cu_b, cu_bk, qb, kb, vb, 1, kp, vp)
    pa, pb = B.Packed(cu_a, cu_a, H, KV, D, block=1, device=DEV), B.Packed(cu_b, cu_bk, H, KV, D, block=1, prefix_tokens=700, device=DEV)
    oa, ob = torch.empty_like(qa), torch.empty_like(qb)
    B.pf_packed_plan(pa)
    B.pf_packed_plan(pb)
    wa, wb = (torch.empty(B.pf_packed_workspace_bytes(p), dtype=torch.uint8, device=DEV) for p in (pa, pb))
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for s in (s1, s2):
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):                                            # side by side, each with a workspace of its own
        with torch.cuda.stream(s1):
            B.pf_packed_attn_fwd(pa, qa, ka, va, oa, wa)
        with torch.cuda.stream(s2):
            B.pf_packed_attn_fwd(pb, qb, kb, vb, ob, wb, kp, vp)
    torch.cuda.synchronize()
    assert torch.equal(oa, want_a) and torch.equal(ob, want_b)
    # plan and attention captured, replayed with other inputs, eager work between
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.pf_packed_plan(pb)
        B.pf_packed_attn_fwd(pb, qb, kb, vb, ob, wb, kp, vp)
    for seed in (51, 52, 53):
        qb.copy_(synth.randn_bf16((12, H, D), seed, device=DEV).transpose(0, 1))
        pb.work.zero_()
        graph.replay()
        got = ob.clone()
        want = _run(cu_b, cu_bk, qb, kb, vb, 1, kp, vp)
        assert torch.equal(got, want)


@pytest.mark.gpu
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("seqs,H,KV,P,keys", [(1, 8, 8, 0, 5000), (4, 8, 1, 3000, 70), (8, 4, 4, 700, 300), (32, 3, 3, 2000, 9), (33, 3, 3, 2000, 9),
                                                 (2, 8, 2, 2500, 64), (9, 2, 2, 2500, 64)])
def test_few_rows_split_over_many_workgroups(seqs, H, KV, P, keys, D):
    """Up to 8 rows a head are joined by the head's last workgroup, more by a second launch: launch after launch and replay after replay
    with the same bits, the plan's counters back at zero."""
    cu_q, cu_k = _cu([1] * seqs), _cu([keys + 3 * i for i in range(seqs)])
    q, k, v, kp, vp = _tensors(H, KV, D, cu_q[-1], cu_k[-1], P, 71, True)
    want, tol = _definition(q, k, v, cu_q, cu_k, 1, kp, vp)
    packed = B.Packed(cu_q, cu_k, H, KV, D, block=1, prefix_tokens=P, device=DEV)
    B.pf_packed_plan(packed)
    assert packed.c.n_planes > 1, "the case must park partial results"
    plan = packed.work.clone()
    ws = torch.full((B.pf_packed_workspace_bytes(packed),), 255, dtype=torch.uint8, device=DEV)
    out = torch.full_like(q, float("nan"))
    B.pf_packed_attn_fwd(packed, q, k, v, out, ws, kp, vp)
    torch.cuda.synchronize()
    assert ((out.double() - want).abs() <= tol).all()
    graph, again = torch.cuda.CUDAGraph(), torch.empty_like(q)
    with torch.cuda.graph(graph):
        B.pf_packed_attn_fwd(packed, q, k, v, again, ws, kp, vp)
    for i in range(20):
        again.fill_(float("nan"))
        ws.fill_(17 * i % 256)
        if i % 2:
            graph.replay()
        else:
            B.pf_packed_attn_fwd(packed, q, k, v, again, ws, kp, vp)
        assert torch.equal(again, out)
    assert torch.equal(packed.work, plan)


@pytest.mark.gpu
def test_a_prompt_taken_in_and_continued():
    """As they are used together: queries and keys of a whole prompt normalised and rotated, the prompt's attention causal by chunks, its
    keys and values taken into the ragged cache, the next chunk attended to through the cache -- and the same chunk attended to
    behind the prompt as a shared prefix, twice over."""
    H, D, tpf, chunk, frames = 3, 128, 40, 2, 6
    n, Lq = frames * tpf, chunk * tpf
    rope = B.make_rope(D, axis_pairs=[24, 20, 20], interleaved=True)
    raw = synth.randn_bf16((n + Lq, 3 * H, D), 61, device=DEV)
    t = torch.arange(n + Lq, device=DEV, dtype=torch.int32)
    pos = torch.stack([t // tpf, t % tpf // 8, t % 8]).contiguous()
    q, k, v = (raw[:, i * H:(i + 1) * H].transpose(0, 1) for i in range(3))
    B.pf_qk_norm_rope(rope, pos, q, q, k, k, eps=1e-6)
    # the prompt, and the prompt with the next chunk: the chunk is the last block
    cu = _cu([n + Lq])
    whole = _run(cu, cu, q, k, v, Lq)
    cu = _cu([n])
    prompt = _run(cu, cu, q[:, :n], k[:, :n], v[:, :n], Lq)
    assert torch.equal(prompt.contiguous(), whole[:, :n].contiguous())
    pool = B.Pool([synth.anchor_all(frames)] * H, tpf, D, device=DEV)
    B.pf_pool_reset(pool)
    B.pf_cache_append_strided(pool, k[:, :n].unflatten(1, (frames, tpf)), v[:, :n].unflatten(1, (frames, tpf)))
    index = B.Index(pool, Lq)
    B.pf_build_index(pool, index, Lq)
    out = torch.empty((Lq, H, D), dtype=torch.bfloat16, device=DEV).transpose(0, 1)
    ws = torch.empty(B.pf_attn_workspace_bytes(pool, Lq), dtype=torch.uint8, device=DEV)
    new = [x[:, n:].contiguous() for x in (q, k, v)]
    packed_out = torch.empty_like(new[0])
    B.pf_ragged_attn_fwd(pool, index, *new, packed_out, ws)
    torch.cuda.synchronize()
    want, tol = _definition(q, k, v, _cu([n + Lq]), _cu([n + Lq]), Lq)
    want, tol = want[:, n:], tol[:, n:]
    for got in (whole[:, n:], packed_out):
        assert ((got.double() - want).abs() <= tol).all()
    twice = [torch.cat([x, x], 1) for x in new]
    cu = _cu([Lq, Lq])
    both = _run(cu, cu, *twice, Lq, k[:, :n], v[:, :n])
    for got in (both[:, :Lq], both[:, Lq:]):
        assert ((got.double() - want).abs() <= tol).all()
