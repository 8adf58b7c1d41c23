"""Group-scaled rows without a GPU: the reference used by the GPU tests, what the C ABI refuses
before any HIP call, and what the Python binding refuses before any call."""
import numpy as np
import pytest
import torch

import group_reference as ref
import paper_1809_10572_amd as samd
from paper_1809_10572_amd import Fmt, GroupRows

OK, EINVAL, EALIGN, EUNSUP = 0, -1, -2, -3
P, ODD1, ODD2 = 0x10000, 0x10001, 0x10002   # fake device addresses: nothing may be dereferenced
S4, U4, S8 = Fmt(4, True), Fmt(4, False), Fmt(8, True)
F32, F16 = 0, 1


# ---- the reference --------------------------------------------------------------------------------

@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("signed", [True, False])
def test_rule_is_off_by_half_a_step(bits, signed):
    x = (np.random.default_rng(bits).standard_normal((40, 200)) * 3).astype(np.float32)
    x[3] = np.abs(x[3])
    q, scale, zero = ref.quantize(x, bits, signed, 64)
    back = ref.values(q, scale, zero, 64)
    at = np.arange(200) // 64
    # signed: half a step; unsigned: half a step of the value and half of the zero point
    assert (np.abs(back - x) <= scale[:, at] * (0.5 if signed else 1.0) * (1 + 1e-5)).all()
    assert q.min() >= (-(1 << bits - 1) + 1 if signed else 0) and q.max() <= (1 << bits - signed) - 1


def test_reference_unpack_reads_the_fields():
    w = np.array([[0x76543210, 0xFEDCBA98]], dtype=np.uint32)
    assert ref.unpack(w, 16, 4, False).tolist() == [list(range(16))]
    assert ref.unpack(w, 13, 4, True).tolist() == [[0, 1, 2, 3, 4, 5, 6, 7, -8, -7, -6, -5, -4]]
    assert ref.unpack(w, 5, 8, True).tolist() == [[0x10, 0x32, 0x54, 0x76, 0x98 - 256]]
    assert ref.spare_bits(w, 13, 4).tolist() == [0xFED] and ref.spare_bits(w, 5, 8).tolist() == [0xFEDCBA]


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_reference_slopes_by_differences(act):
    g = np.linspace(-9, 9, 1001)
    e = 1e-5
    numeric = (ref.activation(g + e, act)[0] - ref.activation(g - e, act)[0]) / (2 * e)
    assert np.abs(numeric - ref.activation(g, act)[1]).max() < 1e-8


# ---- the C ABI ------------------------------------------------------------------------------------

def matmul(x=P, type=F32, ldx=64, q=P, scale=P, zero=None, wf=S4, group=32, T=2, M=3, K=64, y=P, ldy=3):
    return samd.lib().samd_group_matmul(x, type, ldx, q, scale, zero, wf, group, T, M, K, y, ldy, None)


def grad(dy=P, type=F32, lddy=3, q=P, scale=P, zero=None, dy2=None, q2=None, scale2=None, zero2=None, wf=S4, group=32, T=2,
         M=3, K=64, dx=P, lddx=64):
    return samd.lib().samd_group_matmul_grad(dy, type, lddy, q, scale, zero, dy2, q2, scale2, zero2, wf, group, T, M, K, dx,
                                             lddx, None)


def gated(x=P, type=F32, ldx=64, qg=P, sg=P, zg=None, qu=P, su=P, zu=None, wf=S4, group=32, act=0, T=2, M=3, K=64, h=P, ldh=3,
          g8=None, gs=None, u8=None, us=None):
    return samd.lib().samd_group_gated(x, type, ldx, qg, sg, zg, qu, su, zu, wf, group, act, T, M, K, h, ldh, g8, gs, u8, us,
                                       None)


def gated_grad(dh=P, type=F32, lddh=3, g8=P, gs=P, u8=P, us=P, group=32, act=0, T=2, M=3, dg=P, du=P, ldd=3):
    return samd.lib().samd_group_gated_grad(dh, type, lddh, g8, gs, u8, us, group, act, T, M, dg, du, ldd, None)


def quantize(src=P, type=F32, rows=2, cols=64, ld=64, f=S4, group=32, q=P, scale=P, zero=None):
    return samd.lib().samd_group_quantize(src, type, rows, cols, ld, f, group, q, scale, zero, None)


def dequantize(q=P, scale=P, zero=None, rows=2, cols=64, f=S4, group=32, dst=P, type=F32, ld=64):
    return samd.lib().samd_group_dequantize(q, scale, zero, rows, cols, f, group, dst, type, ld, None)


@pytest.mark.parametrize("call", [matmul, grad, gated])
def test_products_refuse(call):
    assert call(type=3) == EINVAL and call(type=-1) == EINVAL
    assert call(group=16) == EUNSUP and call(group=256) == EUNSUP and call(group=0) == EUNSUP
    for bits in (1, 2, 3, 5, 8):
        assert call(wf=Fmt(bits, True)) == EUNSUP
    raw = Fmt(4, True)
    raw.is_signed = 2
    assert call(wf=raw) == EINVAL
    for size in ("T", "M", "K"):
        assert call(**{size: -1}) == EINVAL and call(**{size: 1 << 31}) == EINVAL
    assert b"2^31 - 1" in samd.lib().samd_last_error()
    assert call(wf=U4) == EINVAL                     # unsigned without zero points
    wide = (1 << 25) + 1
    assert call(K=wide, **({"lddx": wide} if call is grad else {"ldx": wide})) == EUNSUP
    assert call(T=0) == OK                           # nothing to do


def test_matmul_refuses():
    assert matmul(x=None) == EINVAL and matmul(y=None) == EINVAL and matmul(q=None) == EINVAL and matmul(scale=None) == EINVAL
    assert matmul(x=ODD2) == EALIGN and matmul(y=ODD2) == EALIGN and matmul(x=ODD1, type=F16) == EALIGN
    assert matmul(q=ODD2) == EALIGN and matmul(scale=ODD2) == EALIGN
    assert matmul(ldx=63) == EINVAL and matmul(ldy=2) == EINVAL and matmul(ldx=1 << 62) == EINVAL
    assert matmul(K=0) == EINVAL and matmul(M=0) == OK
    assert matmul(zero=P) == EINVAL                  # signed with zero points


def test_grad_refuses_a_sum_over_too_many_rows():
    many = (1 << 25) + 1
    assert grad(M=many, lddy=many) == EUNSUP
    assert b"M = 33554433" in samd.lib().samd_last_error()


def test_grad_refuses():
    assert grad(dy=None) == EINVAL and grad(dx=None) == EINVAL and grad(q=None) == EINVAL
    assert grad(dy=ODD2) == EALIGN and grad(dx=ODD2) == EALIGN
    assert grad(lddy=2) == EINVAL and grad(lddx=63) == EINVAL
    assert grad(M=0) == EINVAL and grad(K=0) == OK
    # a second pair comes whole or not at all
    assert grad(dy2=P) == EINVAL and grad(q2=P) == EINVAL and grad(dy2=P, q2=P) == EINVAL
    assert grad(dy2=P, q2=P, scale2=P, zero2=P) == EINVAL
    assert grad(dy2=ODD2, q2=P, scale2=P) == EALIGN and grad(dy2=P, q2=ODD1, scale2=P) == EALIGN


@pytest.mark.parametrize("type", [F32, F16])
@pytest.mark.parametrize("T", [1, 2, 16, 40, (1 << 31) - 1])
def test_results_of_too_many_workgroups_are_refused(type, T):
    """Launches of 2^32 threads and more are refused before they are made."""
    big = (1 << 31) - 1 if T <= 40 else 1 << 20
    assert matmul(type=type, T=T, M=big, ldy=big) == EUNSUP
    assert gated(type=type, T=T, M=big, ldh=big) == EUNSUP
    assert b"2^32 threads" in samd.lib().samd_last_error()
    if T > 40:
        assert grad(type=type, T=T, K=big, lddx=big) == EUNSUP


def test_gated_refuses():
    assert gated(act=2) == EINVAL and gated(act=-1) == EINVAL
    assert gated(qu=None) == EINVAL and gated(su=None) == EINVAL and gated(zu=P) == EINVAL and gated(qg=ODD1) == EALIGN
    assert gated(K=0) == EINVAL and gated(M=0) == OK and gated(h=None) == EINVAL and gated(ldh=2) == EINVAL
    whole = dict(g8=P, gs=P, u8=P, us=P)
    for part in whole:
        assert gated(**{**whole, part: None}) == EINVAL and gated(**{**whole, part: ODD2}) == EALIGN


def test_gated_grad_refuses():
    assert gated_grad(act=2) == EINVAL and gated_grad(group=48) == EUNSUP and gated_grad(type=7) == EINVAL
    for part in ("dh", "g8", "gs", "u8", "us", "dg", "du"):
        assert gated_grad(**{part: None}) == EINVAL and gated_grad(**{part: ODD2}) == EALIGN
    assert gated_grad(lddh=2) == EINVAL and gated_grad(ldd=2) == EINVAL and gated_grad(T=-1) == EINVAL
    assert gated_grad(T=0) == OK and gated_grad(M=0) == OK


@pytest.mark.parametrize("call", [quantize, dequantize])
def test_quantize_and_dequantize_refuse(call):
    for bits in (1, 2, 3, 5, 6, 7):
        assert call(f=Fmt(bits, True)) == EUNSUP
    assert call(f=Fmt(9, True)) == EINVAL and call(group=8) == EUNSUP and call(type=3) == EINVAL
    assert call(rows=-1) == EINVAL and call(cols=1 << 31) == EINVAL
    assert call(ld=63) == EINVAL and call(q=None) == EINVAL and call(scale=None) == EINVAL
    assert call(f=U4) == EINVAL and call(f=S8, zero=P) == EINVAL
    assert call(q=ODD1) == EALIGN and call(scale=ODD2) == EALIGN
    matrix = "src" if call is quantize else "dst"
    assert call(**{matrix: None}) == EINVAL and call(**{matrix: ODD2}) == EALIGN
    assert call(rows=0) == OK and call(cols=0) == OK


# ---- the binding ----------------------------------------------------------------------------------

class Recorder:
    def __init__(self, real):
        self.real, self.calls = real, []

    def __getattr__(self, name):
        if name in ("samd_row_words", "samd_status_str", "samd_last_error"):
            return getattr(self.real, name)

        def call(*args):
            self.calls.append((name, args))
            return samd.SAMD_OK
        return call


@pytest.fixture
def fake(monkeypatch):
    """CPU tensors taken for device tensors, unless they are marked as the host's."""
    rec, host = Recorder(samd.lib()), set()
    monkeypatch.setattr(samd, "lib", lambda: rec)
    monkeypatch.setattr(samd, "_on_gpu", lambda x: x.untyped_storage().data_ptr() not in host)
    monkeypatch.setattr(samd, "_stream", lambda x: 0)
    return rec, lambda x: host.add(x.untyped_storage().data_ptr()) or x


def rows(n, cols, bits=4, group=32, signed=True):
    groups = -(-cols // group)
    return GroupRows(torch.zeros(n, -(-cols * bits // 32), dtype=torch.int32), torch.zeros(n, groups),
                     None if signed else torch.zeros(n, groups, dtype=torch.uint8), cols, bits, group)


def test_binding_refuses(fake):
    rec, host = fake
    x, w = torch.zeros(3, 70), rows(5, 70)
    dy = torch.zeros(3, 5)
    g, u = rows(3, 5, 8), rows(3, 5, 8)
    bad = [
        lambda: samd.group_matmul(host(torch.zeros(3, 70)), w),
        lambda: samd.group_matmul(x.double(), w),
        lambda: samd.group_matmul(torch.zeros(70, 3).t(), w),                       # columns apart
        lambda: samd.group_matmul(torch.zeros(1, 70).expand(3, 70), w),             # rows on top of each other
        lambda: samd.group_matmul(torch.zeros(3, 64), w),                           # another K
        lambda: samd.group_matmul(torch.tensor(1.0), w),
        lambda: samd.group_matmul(x, rows(5, 70, 8)),                               # 8-bit weights
        lambda: samd.group_matmul(x, w._replace(q=w.q[:, :8].contiguous())),        # short rows
        lambda: samd.group_matmul(x, w._replace(scale=torch.zeros(5, 2))),          # short scales
        lambda: samd.group_matmul(x, w._replace(scale=w.scale.half())),
        lambda: samd.group_matmul(x, w._replace(zero=torch.zeros(5, 2, dtype=torch.uint8))),
        lambda: samd.group_matmul(x, w._replace(zero=torch.zeros(5, 3, dtype=torch.int32))),
        lambda: samd.group_matmul(x, w._replace(q=host(torch.zeros(5, 9, dtype=torch.int32)))),
        lambda: samd.group_matmul(x, w._replace(group=48)),
        lambda: samd.group_matmul(x, w, out=torch.zeros(3, 4)),
        lambda: samd.group_matmul(x, w, out=torch.zeros(2, 5)),
        lambda: samd.group_matmul(x, w, out=torch.zeros(3, 5).half()),
        lambda: samd.group_matmul_grad(dy, rows(4, 70)),
        lambda: samd.group_matmul_grad(dy, w, dy),
        lambda: samd.group_matmul_grad(dy, w, None, w),
        lambda: samd.group_matmul_grad(dy, w, torch.zeros(3, 5).half(), w),
        lambda: samd.group_matmul_grad(dy, w, torch.zeros(3, 9)[:, :5], w),         # another row stride
        lambda: samd.group_matmul_grad(dy, w, dy, rows(5, 71)),
        lambda: samd.group_matmul_grad(dy, w, dy, rows(5, 70, group=64)),
        lambda: samd.group_matmul_grad(dy, w, dy, rows(5, 70, signed=False)),
        lambda: samd.group_gated(x, w, rows(6, 70)),
        lambda: samd.group_gated(x, w, rows(5, 70, signed=False)),
        lambda: samd.group_gated(x, w, w, act="tanh"),
        lambda: samd.group_gated_save(x, w, rows(5, 64)),
        lambda: samd.group_gated_grad(dy, g, rows(3, 6, 8)),
        lambda: samd.group_gated_grad(dy, g, rows(2, 5, 8)),
        lambda: samd.group_gated_grad(dy, rows(3, 5, 4), u),
        lambda: samd.group_gated_grad(dy, rows(3, 5, 8, signed=False), u),
        lambda: samd.group_gated_grad(dy, g, rows(3, 5, 8, group=64)),
        lambda: samd.group_gated_grad(dy, g, u, "relu"),
        lambda: samd.group_gated_grad(dy, g, u, out=(torch.zeros(3, 5), torch.zeros(3, 8)[:, :5])),
        lambda: samd.group_quantize(x, 3, True),
        lambda: samd.group_quantize(x, 4, True, 100),
        lambda: samd.group_quantize(x.int(), 4, True),
        lambda: samd.group_dequantize(w, torch.float64),
        lambda: samd.group_dequantize(w, out=torch.zeros(5, 69)),
        lambda: samd.group_dequantize(w, out=torch.zeros(4, 70)),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
        assert not rec.calls, i


def test_binding_marshals_what_it_is_given(fake):
    rec, _ = fake
    w, x = rows(5, 70, signed=False), torch.zeros(2, 4, 70, dtype=torch.bfloat16)
    y = samd.group_matmul(x, w)
    assert y.shape == (2, 4, 5) and y.dtype == x.dtype
    name, a = rec.calls.pop()
    assert name == "samd_group_matmul" and a[0] == x.data_ptr() and a[1:3] == (2, 70)
    assert a[3:6] == (w.q.data_ptr(), w.scale.data_ptr(), w.zero.data_ptr()) and repr(a[6]) == "Fmt(4, u)"
    assert a[7:] == (32, 8, 5, 70, y.data_ptr(), 5, 0)
    view = torch.zeros(9, 80)[2:5, 3:73]
    samd.group_matmul(view, rows(5, 70))
    assert rec.calls.pop()[1][2] == 80
    h, g, u = samd.group_gated_save(x, w, w, "gelu")
    a = rec.calls.pop()[1]
    assert g.q.shape == (2, 4, 2) and u.scale.shape == (2, 4, 1) and a[11] == 1
    assert a[17:21] == (g.q.data_ptr(), g.scale.data_ptr(), u.q.data_ptr(), u.scale.data_ptr())
    samd.group_gated(x, w, w)
    assert rec.calls.pop()[1][17:21] == (None,) * 4
    dg, du = samd.group_gated_grad(h, g, u, "gelu")
    assert dg.shape == h.shape and rec.calls.pop()[0] == "samd_group_gated_grad"
    dx = samd.group_matmul_grad(dg, w, du, w)
    a = rec.calls.pop()[1]
    assert dx.shape == x.shape and a[6] == du.data_ptr() and a[11:15] == (32, 8, 5, 70)
    r = samd.group_quantize(x, 8, False, 64)
    assert r.q.shape == (2, 4, 18) and r.zero.shape == r.scale.shape == (2, 4, 2) and rec.calls.pop()[1][2:5] == (8, 70, 70)
    assert samd.group_dequantize(r, torch.float16).shape == x.shape


# ---- the compiled kernels -------------------------------------------------------------------------

def test_kernels_use_no_scratch():
    """Every kernel on group-scaled rows keeps its arrays in registers (a lambda that the compiler does not
    inline puts them into scratch memory, which costs a product a hundredfold)."""
    import re

    from test_kernel_resources import _code_objects, _kernels
    samd.lib()
    with open(samd.LIB_PATH, "rb") as f:
        blob = f.read()
    seen = 0
    for k in (k for elf in _code_objects(blob) for k in _kernels(elf)):
        if not re.search(r"group_(quantize|dequantize|gated_grad|vector|narrow|gemm|grad)_kernel", k[".name"]):
            continue
        seen += 1
        assert k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, k[".name"]
    assert seen > 100
