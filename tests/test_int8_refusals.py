"""Arguments that the calls on int8 codes refuse, before anything is enqueued.  Nothing is launched here."""
import pytest
import torch

FAKE = 0x1000  # an aligned address that is never dereferenced: every call below fails validation first, or has nothing to do
NULL, SHAPE, ALIGN, OVERFLOW, UNSUPPORTED, WORKSPACE = 1, 2, 3, 4, 5, 6


@pytest.fixture(scope="module")
def lib():
    import paper_1609_07061_amd as q

    return q._lib


def _calls(f, good):
    """call(name=value, ...): the status with these arguments of `good` replaced."""
    names = list(good)

    def call(**change):
        assert set(change) <= set(names)
        return f(*[change.get(n, good[n]) for n in names])

    return call


def test_rms_norm_quant(lib):
    call = _calls(lib.qnn_rms_norm_quant, dict(x=FAKE, ldx=64, residual=FAKE, ldr=64, type=2, gamma=FAKE, gamma_type=2, eps=1e-5, rows=4, K=64, sum=FAKE, lds=64,
                                               codes=FAKE, ldc=64, scale=FAKE, stream=None))
    assert call(rows=0) == 0 and call(rows=0, x=None, codes=None) == 0
    assert call(rows=-1) == SHAPE and call(K=0) == SHAPE
    assert all(call(**{n: 63}) == SHAPE for n in ("ldx", "ldr", "lds", "ldc"))
    assert call(type=3) == SHAPE and call(type=-1) == SHAPE and call(gamma_type=1) == SHAPE
    assert call(eps=-1.0) == SHAPE and call(eps=float("nan")) == SHAPE and call(eps=float("inf")) == SHAPE
    assert all(call(**{n: None}) == NULL for n in ("x", "gamma", "codes", "scale"))
    assert all(call(**{n: FAKE + 1}) == ALIGN for n in ("x", "residual", "sum", "gamma")) and call(scale=FAKE + 2) == ALIGN
    assert call(gamma_type=0, gamma=FAKE + 2) == ALIGN
    assert b"rms_norm_quant" in lib.qnn_last_error()


def test_rms_norm_backward(lib):
    assert lib.qnn_rms_norm_backward_workspace_bytes(4, 64) == 4 * 64 * 4
    assert lib.qnn_rms_norm_backward_workspace_bytes(100000, 64) == 512 * 64 * 4
    assert lib.qnn_rms_norm_backward_workspace_bytes(0, 64) == 0 and lib.qnn_rms_norm_backward_workspace_bytes(4, 16385) == 0
    call = _calls(lib.qnn_rms_norm_backward, dict(grad=FAKE, ldg=64, h=FAKE, ldh=64, grad_sum=FAKE, ldz=64, type=0, gamma=FAKE, gamma_type=0, eps=1e-5, rows=4, K=64,
                                                  grad_h=FAKE, ldo=64, grad_gamma=FAKE, workspace=FAKE, bytes=4 * 64 * 4, stream=None))
    assert call(rows=0) == SHAPE and call(K=0) == SHAPE and call(type=3) == SHAPE and call(gamma_type=2) == SHAPE and call(eps=-1.0) == SHAPE
    assert all(call(**{n: 63}) == SHAPE for n in ("ldg", "ldh", "ldz", "ldo"))
    assert call(K=16385, ldg=16385, ldh=16385, ldz=16385, ldo=16385) == UNSUPPORTED
    assert all(call(**{n: None}) == NULL for n in ("grad", "h", "gamma", "grad_h", "grad_gamma"))
    assert all(call(**{n: FAKE + 2}) == ALIGN for n in ("grad", "h", "grad_sum", "gamma", "grad_h", "grad_gamma"))
    assert call(workspace=None) == WORKSPACE and call(workspace=FAKE + 128) == WORKSPACE and call(bytes=4 * 64 * 4 - 1) == WORKSPACE


def test_silu_gate(lib):
    call = _calls(lib.qnn_silu_gate_quant, dict(gate=FAKE, ldg=64, up=FAKE, ldu=64, type=1, rows=4, F=64, codes=FAKE, ldc=64, scale=FAKE, stream=None))
    assert call(rows=0) == 0
    assert call(rows=-1) == SHAPE and call(F=0) == SHAPE and call(type=7) == SHAPE
    assert all(call(**{n: 63}) == SHAPE for n in ("ldg", "ldu", "ldc"))
    assert all(call(**{n: None}) == NULL for n in ("gate", "up", "codes", "scale"))
    assert all(call(**{n: FAKE + 1}) == ALIGN for n in ("gate", "up", "scale"))
    call = _calls(lib.qnn_silu_gate_backward, dict(grad=FAKE, ldd=64, gate=FAKE, ldg=64, up=FAKE, ldu=64, type=2, rows=4, F=64, grad_gate=FAKE, lda=64, grad_up=FAKE,
                                                   ldb=64, stream=None))
    assert call(rows=0) == 0
    assert call(rows=-1) == SHAPE and call(F=0) == SHAPE and call(type=7) == SHAPE
    assert all(call(**{n: 63}) == SHAPE for n in ("ldd", "ldg", "ldu", "lda", "ldb"))
    pointers = ("grad", "gate", "up", "grad_gate", "grad_up")
    assert all(call(**{n: None}) == NULL for n in pointers) and all(call(**{n: FAKE + 1}) == ALIGN for n in pointers)


def test_int8_gemm(lib):
    call = _calls(lib.qnn_int8_gemm, dict(A=FAKE, lda=64, scaleA=FAKE, W=FAKE, ldw=64, scaleW=FAKE, bias=FAKE, out=FAKE, ldo=32, type=0, M=4, N=32, K=64, stream=None))
    assert call(M=0) == 0 and call(N=0) == 0
    assert call(M=-1) == SHAPE and call(N=-1) == SHAPE and call(K=0) == SHAPE and call(type=5) == SHAPE
    assert call(lda=63) == SHAPE and call(ldw=63) == SHAPE and call(ldo=31) == SHAPE
    assert call(K=131072, lda=131072, ldw=131072) == OVERFLOW
    assert b"int32" in lib.qnn_last_error()
    assert all(call(**{n: None}) == NULL for n in ("A", "scaleA", "W", "scaleW", "out"))
    assert all(call(**{n: FAKE + 2}) == ALIGN for n in ("scaleA", "scaleW", "bias", "out"))


def test_int8_moe(lib):
    need = lib.qnn_int8_moe_workspace_bytes(4, 2, 48)
    assert need >= 4 * 2 * (48 * 4 + 3 * 4 + 8)
    assert all(lib.qnn_int8_moe_workspace_bytes(*a) == 0 for a in ((0, 2, 48), (65, 2, 48), (4, 0, 48), (4, 9, 48), (4, 2, 0), (4, 2, 131072)))
    call = _calls(lib.qnn_int8_moe, dict(x=FAKE, ldx=64, sx=FAKE, logits=FAKE, ldl=8, tokens=4, experts=8, top=2, H=64, F=48, W1=FAKE, ld1=64, s1=FAKE, W2=FAKE, ld2=48, s2=FAKE,
                                         out=FAKE, ldo=64, type=0, ws=FAKE, bytes=need, stream=None))
    assert call(tokens=0) == 0
    assert all(call(**c) == SHAPE for c in (dict(tokens=-1), dict(experts=0), dict(top=0), dict(top=9), dict(H=0), dict(F=0), dict(type=3)))
    assert all(call(**c) == SHAPE for c in (dict(ldx=63), dict(ldl=7), dict(ld1=63), dict(ld2=47), dict(ldo=63)))
    assert call(tokens=65) == UNSUPPORTED and call(experts=257, ldl=300) == UNSUPPORTED and call(experts=16, ldl=16, top=9) == UNSUPPORTED
    assert call(H=131072, ldx=131072, ld1=131072, ldo=131072) == OVERFLOW and call(F=131072, ld2=131072) == OVERFLOW
    assert all(call(**{n: None}) == NULL for n in ("x", "sx", "logits", "W1", "s1", "W2", "s2", "out"))
    assert all(call(**{n: FAKE + 2}) == ALIGN for n in ("sx", "logits", "s1", "s2", "out"))
    assert call(ws=None) == WORKSPACE and call(ws=FAKE + 4) == WORKSPACE and call(bytes=need - 1) == WORKSPACE


def _binding_refuses(q, device):
    z = lambda *n, dtype=torch.float32: torch.zeros(*n, dtype=dtype, device=device)
    f, i, s, v, i8 = z(4, 64), z(4, 64, dtype=torch.int8), z(4), z(64), torch.int8
    cases = [
        (lambda: q.qnn_rms_norm_quant(f, v[:63], 1e-5), "gamma must be dense"),
        (lambda: q.qnn_rms_norm_quant(f, v, 1e-5, f[:3]), "residual must be"),
        (lambda: q.qnn_rms_norm_quant(f, v, 1e-5, f.half()), "residual must have dtype"),
        (lambda: q.qnn_rms_norm_quant(f, v, 1e-5, codes=f), "codes must have dtype"),
        (lambda: q.qnn_rms_norm_quant(f.double(), v, 1e-5), "float32, float16 or bfloat16"),
        (lambda: q.qnn_rms_norm_backward(f[:, :63], f, v, 1e-5), "grad must be"),
        (lambda: q.qnn_rms_norm_backward(f, f, v, 1e-5, grad_gamma=v.half()), "grad_gamma must have dtype"),
        (lambda: q.qnn_silu_gate_quant(f.t(), f.t()), "contiguous rows"),
        (lambda: q.qnn_silu_gate_quant(f, f, scale=s[:3]), "scale must be dense"),
        (lambda: q.qnn_silu_gate_backward(f, f, f[:, 1:]), "up must be"),
        (lambda: q.qnn_int8_gemm(i, s, i[:, :63], s), "codes"),
        (lambda: q.qnn_int8_gemm(i, s[:3], i, s), "scaleA must be dense"),
        (lambda: q.qnn_int8_gemm(i, s, i, s, out=z(4, 5)), "out must be"),
        (lambda: q.qnn_int8_gemm(i, s, f, s), "W must have dtype"),
        (lambda: q.qnn_int8_moe(i, s, f[:, :2], 1, z(2, 64, 64, dtype=i8), z(2, 64), z(2, 64, 31, dtype=i8), z(2, 64)), "W1 must be"),
        (lambda: q.qnn_int8_moe(i, s, f[:, :2], 1, z(2, 64, 64, dtype=i8), z(2, 63), z(2, 64, 32, dtype=i8), z(2, 64)), "scale1 must be dense"),
        (lambda: q.qnn_int8_moe(i, s, f[:, :2], 1, z(2, 70, 64, dtype=i8)[:, :64], z(2, 64), z(2, 64, 32, dtype=i8), z(2, 64)), "without a gap"),
        (lambda: q.qnn_int8_moe(i, s, f[:, :3], 1, z(2, 64, 64, dtype=i8), z(2, 64), z(2, 64, 32, dtype=i8), z(2, 64)), "logits must be"),
    ]
    for call, message in cases:
        with pytest.raises(ValueError, match=message if device == "cuda" else message + "|must be a GPU tensor"):
            call()


def test_binding_refuses(lib):
    """Shapes, types and places of tensors that the binding does not pass on."""
    import paper_1609_07061_amd as q

    _binding_refuses(q, "cpu")
    with pytest.raises(ValueError, match="must be a GPU tensor"):
        q.qnn_rms_norm_quant(torch.zeros(4, 64), torch.zeros(64), 1e-5)


@pytest.mark.gpu
def test_binding_refuses_on_the_gpu(lib):
    import paper_1609_07061_amd as q

    _binding_refuses(q, "cuda")
    with pytest.raises(q.QnnError) as e:  # (more tokens than a call takes)
        z = lambda *n, dtype=torch.float32: torch.zeros(*n, dtype=dtype, device="cuda")
        q.qnn_int8_moe(z(65, 64, dtype=torch.int8), z(65), z(65, 2), 1, z(2, 64, 64, dtype=torch.int8), z(2, 64), z(2, 64, 32, dtype=torch.int8), z(2, 64))
    assert e.value.status == UNSUPPORTED
