"""Arguments that the calls on heads and the paged cache refuse, before anything is enqueued.  Nothing is launched here."""
import ctypes as C

import pytest
import torch

from test_int8_refusals import FAKE, NULL, SHAPE, ALIGN, UNSUPPORTED, WORKSPACE, _calls

BIG = 0x100000  # 256-byte aligned, never dereferenced


@pytest.fixture(scope="module")
def q():
    import paper_1609_07061_amd as q

    return q


def _rotation(q, **change):
    v = dict(positions=FAKE, ld_positions=4, freq=FAKE, axis=FAKE, axes=3, pairs=32, neighbours=0)
    v.update(change)
    return C.byref(q._Rotation(*v.values()))


def _cache(q, **change):
    v = dict(k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE, pages=10, heads=2, page=16, D=64, table=FAKE, ld_table=5, width=5, starts=FAKE, lengths=FAKE, sequences=3)
    v.update(change)
    return C.byref(q._PagedCache(*v.values()))


ROTATIONS = [(dict(pairs=-8), SHAPE), (dict(pairs=4), SHAPE), (dict(pairs=40), SHAPE), (dict(axes=0), SHAPE), (dict(ld_positions=3), SHAPE), (dict(ld_positions=-1), SHAPE),
             (dict(positions=None), NULL), (dict(freq=None), NULL), (dict(positions=FAKE + 2), ALIGN), (dict(freq=FAKE + 4), ALIGN), (dict(axis=FAKE + 1), ALIGN)]
HEADS = [(dict(D=24), UNSUPPORTED), (dict(D=272), UNSUPPORTED), (dict(D=0), UNSUPPORTED), (dict(tokens=-1), SHAPE), (dict(heads_q=-1), SHAPE), (dict(heads_q=70000), SHAPE),
         (dict(type=3), SHAPE), (dict(gamma_type=1), SHAPE), (dict(eps=-1.0), SHAPE), (dict(eps=float("nan")), SHAPE), (dict(gamma_q=None), SHAPE), (dict(gamma_k=None), SHAPE),
         (dict(gamma_q=FAKE + 1), ALIGN)]


def test_qk_norm_rotate(q):
    good = dict(q=FAKE, ldq=256, sq=64, heads_q=4, k=FAKE, ldk=128, sk=64, heads_k=2, type=2, gamma_q=FAKE, gamma_k=FAKE, gamma_type=2, eps=1e-5, rotation=_rotation(q), tokens=4,
                D=64, q_out=FAKE, ldqo=256, sqo=64, k_out=FAKE, ldko=128, sko=64, stream=None)
    call = _calls(q._lib.qnn_qk_norm_rotate, good)
    assert call(tokens=0) == 0 and call(tokens=0, q=None) == 0
    for change, status in HEADS + [(dict(heads_q=0, heads_k=0), SHAPE), (dict(rotation=None), NULL)]:
        assert call(**change) == status, change
    for n in ("ldq", "ldqo"):
        assert call(**{n: 255}) == SHAPE, n
    for n in ("sq", "sk", "sqo", "sko"):
        assert call(**{n: 63}) == SHAPE, n
    assert all(call(**{n: None}) == NULL for n in ("q", "k", "q_out", "k_out"))
    assert all(call(**{n: FAKE + 1}) == ALIGN for n in ("q", "k", "q_out", "k_out"))
    for change, status in ROTATIONS:
        assert call(rotation=_rotation(q, **change)) == status, change
    assert b"qk_norm_rotate" in q._lib.qnn_last_error()


def test_qk_norm_rotate_backward(q):
    need = q.qnn_qk_norm_rotate_backward_workspace_bytes(4, 4, 2, 64)
    assert need >= 2 * 64 * 4 and q.qnn_qk_norm_rotate_backward_workspace_bytes(0, 4, 2, 64) == 0 and q.qnn_qk_norm_rotate_backward_workspace_bytes(4, 4, 2, 300) == 0
    assert q.qnn_qk_norm_rotate_backward_workspace_bytes(1 << 30, 32, 8, 256) <= 1024 * 256 * 4
    good = dict(gq=FAKE, ldgq=256, sgq=64, gk=FAKE, ldgk=128, sgk=64, q=FAKE, ldq=256, sq=64, heads_q=4, k=FAKE, ldk=128, sk=64, heads_k=2, type=2, gamma_q=FAKE, gamma_k=FAKE,
                gamma_type=2, eps=1e-5, rotation=_rotation(q), tokens=4, D=64, oq=FAKE, ldoq=256, soq=64, ok=FAKE, ldok=128, sok=64, sums_q=FAKE, sums_k=FAKE, ws=BIG, bytes=need,
                stream=None)
    call = _calls(q._lib.qnn_qk_norm_rotate_backward, good)
    assert call(tokens=0) == SHAPE and call(tokens=0, gamma_q=None, gamma_k=None) == 0
    for change, status in HEADS:
        assert call(**change) == status, change
    for n in ("ldgq", "ldq", "ldoq"):
        assert call(**{n: 255}) == SHAPE, n
    assert all(call(**{n: None}) == NULL for n in ("gq", "gk", "q", "k", "oq", "ok", "sums_q", "sums_k"))
    assert all(call(**{n: FAKE + 1}) == ALIGN for n in ("gq", "gk", "q", "k", "oq", "ok", "sums_q", "sums_k"))
    for change, status in ROTATIONS:
        assert call(rotation=_rotation(q, **change)) == status, change
    assert call(ws=None) == WORKSPACE and call(ws=BIG + 128) == WORKSPACE and call(bytes=need - 1) == WORKSPACE


CACHES = [(dict(pages=0), SHAPE), (dict(heads=0), SHAPE), (dict(page=0), SHAPE), (dict(sequences=-1), SHAPE), (dict(width=6), SHAPE), (dict(width=-1), SHAPE), (dict(D=40), UNSUPPORTED),
          (dict(D=0), UNSUPPORTED), (dict(D=512), UNSUPPORTED), (dict(pages=1 << 27), UNSUPPORTED), (dict(page=1 << 30), UNSUPPORTED), (dict(k=None), NULL), (dict(v=None), NULL), (dict(k_scale=None), NULL),
          (dict(v_scale=None), NULL), (dict(table=None), NULL), (dict(starts=None), NULL), (dict(lengths=None), NULL), (dict(k=FAKE + 8), ALIGN), (dict(v=FAKE + 1), ALIGN),
          (dict(k_scale=FAKE + 2), ALIGN), (dict(table=FAKE + 2), ALIGN), (dict(lengths=FAKE + 1), ALIGN)]


def test_cache_append(q):
    good = dict(cache=_cache(q), q=FAKE, ldq=256, sq=64, heads_q=4, k=FAKE, ldk=128, sk=64, v=FAKE, ldv=128, sv=64, type=2, gamma_q=FAKE, gamma_k=FAKE, gamma_type=2, eps=1e-5,
                rotation=_rotation(q), tokens=4, q_out=FAKE, ldqo=256, sqo=64, stream=None)
    call = _calls(q._lib.qnn_cache_append, good)
    assert call(tokens=0) == 0 and call(cache=_cache(q, sequences=0)) == 0
    for change, status in CACHES:
        assert call(cache=_cache(q, **change)) == status, change
    assert call(cache=None) == NULL
    for change, status in [c for c in HEADS if "D" not in c[0]]:
        assert call(**change) == status, change
    assert all(call(**{n: None}) == NULL for n in ("q", "k", "v", "q_out")) and all(call(**{n: FAKE + 1}) == ALIGN for n in ("q", "k", "v", "q_out"))
    assert all(call(**{n: 127}) == SHAPE for n in ("ldk", "ldv")) and all(call(**{n: 60}) == SHAPE for n in ("sq", "sk", "sv", "sqo"))
    for change, status in ROTATIONS:
        assert call(rotation=_rotation(q, **change)) == status, change
    assert call(heads_q=0, gamma_q=FAKE) == SHAPE  # (a weight for queries that are not there)


def test_cache_attention(q):
    need = q.qnn_cache_attention_workspace_bytes(4, 3, 8, 2, 64, 2, 5000)
    assert need > 0
    assert all(q.qnn_cache_attention_workspace_bytes(*a) == 0 for a in ((0, 3, 8, 2, 64, 2, 5000), (4, 0, 8, 2, 64, 2, 5000), (4, 3, 7, 2, 64, 2, 5000), (4, 3, 8, 2, 64, 0, 5000), (4, 3, 8, 2, 64, 2, 0)))
    good = dict(cache=_cache(q), q=FAKE, ldq=512, sq=64, heads_q=8, type=1, scale=0.125, cap=0.0, slopes=FAKE, tree=FAKE, tokens=4, most_new=2, longest=5000, out=FAKE, ldo=512, so=64,
                ws=BIG, bytes=need, stream=None)
    call = _calls(q._lib.qnn_cache_attention, good)
    assert call(tokens=0) == 0 and call(cache=_cache(q, sequences=0)) == 0
    for change, status in CACHES:
        assert call(cache=_cache(q, **change)) == status, change
    inf, nan = float("inf"), float("nan")
    for change, status in [(dict(cache=None), NULL), (dict(tokens=-1), SHAPE), (dict(heads_q=0), SHAPE), (dict(heads_q=9), SHAPE), (dict(heads_q=70000), SHAPE), (dict(most_new=0), SHAPE),
                           (dict(longest=0), SHAPE), (dict(type=4), SHAPE), (dict(cap=-1.0), SHAPE), (dict(cap=9e-31), SHAPE), (dict(cap=nan), SHAPE), (dict(cap=inf), SHAPE), (dict(scale=nan), SHAPE),
                           (dict(scale=inf), SHAPE), (dict(ldq=511), SHAPE), (dict(ldo=511), SHAPE), (dict(sq=63), SHAPE), (dict(so=-64), SHAPE), (dict(q=None), NULL), (dict(out=None), NULL),
                           (dict(q=FAKE + 1), ALIGN), (dict(out=FAKE + 1), ALIGN), (dict(slopes=FAKE + 2), ALIGN), (dict(tree=FAKE + 4), ALIGN), (dict(ws=None), WORKSPACE),
                           (dict(ws=BIG + 64), WORKSPACE), (dict(bytes=need - 1), WORKSPACE)]:
        assert call(**change) == status, change


def test_rows_quant(q):
    call = _calls(q._lib.qnn_rows_quant, dict(x=FAKE, ldx=64, type=2, rows=4, K=64, codes=FAKE, ldc=64, scale=FAKE, stream=None))
    assert call(rows=0, x=None) == 0
    assert all(call(**c) == SHAPE for c in (dict(rows=-1), dict(K=0), dict(type=3), dict(ldx=63), dict(ldc=63)))
    assert all(call(**{n: None}) == NULL for n in ("x", "codes", "scale")) and call(x=FAKE + 1) == ALIGN and call(scale=FAKE + 2) == ALIGN


def _binding_refuses(q, device):
    z = lambda *n, dtype=torch.float32: torch.zeros(*n, dtype=dtype, device=device)
    i32, f64 = torch.int32, torch.float64
    x, k, g, pos, freq = z(4, 8, 64), z(4, 2, 64), z(64), z(1, 4, dtype=i32), z(32, dtype=f64)
    cache, table, starts, lengths = q.qnn_new_cache(4, 2, 16, 64, device), z(3, 2, dtype=i32), z(4, dtype=i32), z(3, dtype=i32)
    paged = (cache, table, starts, lengths)
    cases = [
        (lambda: q.qnn_qk_norm_rotate(x[0], k, g, g, 1e-5, pos, freq), r"q must be \[tokens\]"),
        (lambda: q.qnn_qk_norm_rotate(x, k[:3], g, g, 1e-5, pos, freq), "k must be"),
        (lambda: q.qnn_qk_norm_rotate(x, k.half(), g, g, 1e-5, pos, freq), "k must have dtype"),
        (lambda: q.qnn_qk_norm_rotate(x.transpose(1, 2), k, g, g, 1e-5, pos, freq), "contiguous heads|must be"),
        (lambda: q.qnn_qk_norm_rotate(x, k, g[:63], g, 1e-5, pos, freq), "gamma_q must be dense"),
        (lambda: q.qnn_qk_norm_rotate(x, k, g, g.half(), 1e-5, pos, freq), "must have one type"),
        (lambda: q.qnn_qk_norm_rotate(x, k, g, g, 1e-5, pos[:, :3], freq), "positions must be"),
        (lambda: q.qnn_qk_norm_rotate(x, k, g, g, 1e-5, pos.long(), freq), "positions must have dtype"),
        (lambda: q.qnn_qk_norm_rotate(x, k, g, g, 1e-5, pos, freq.float()), "freq must have dtype"),
        (lambda: q.qnn_qk_norm_rotate(x, k, g, g, 1e-5, None, freq), "needs positions"),
        (lambda: q.qnn_qk_norm_rotate(x, k, g, g, 1e-5, pos, freq, z(31, dtype=i32)), "axis must be dense"),
        (lambda: q.qnn_qk_norm_rotate(x, k, g, g, 1e-5, pos, freq, q_out=x[:, :7]), "q_out must be"),
        (lambda: q.qnn_qk_norm_rotate(x.double(), k, g, g, 1e-5, pos, freq), "float32, float16 or bfloat16"),
        (lambda: q.qnn_qk_norm_rotate_backward(x[:, :7], k, x, k, g, g, 1e-5, pos, freq), "grad_q must be"),
        (lambda: q.qnn_qk_norm_rotate_backward(x, k, x, k, g, g, 1e-5, pos, freq, grad_gamma_k=g.half()), "grad_gamma_k must have dtype"),
        (lambda: q.qnn_cache_append(*paged, k, k[:, :1], g, 1e-5, pos, freq), "v must be"),
        (lambda: q.qnn_cache_append(*paged, x, x, g, 1e-5, pos, freq), "k must have 2 heads of 64"),
        (lambda: q.qnn_cache_append((cache[0][:, :, ::2], *cache[1:]), *paged[1:], k, k, g, 1e-5, pos, freq), "codes of the cache must be dense"),
        (lambda: q.qnn_cache_append((cache[0], cache[1][:3], *cache[2:]), *paged[1:], k, k, g, 1e-5, pos, freq), "scales of the cache's keys"),
        (lambda: q.qnn_cache_append(cache, table, starts[:3], lengths, k, k, g, 1e-5, pos, freq), "starts must be dense"),
        (lambda: q.qnn_cache_append(cache, table.long(), starts, lengths, k, k, g, 1e-5, pos, freq), "table must have dtype"),
        (lambda: q.qnn_cache_attention(x[:, :, :32], *paged), "q must have heads of 64"),
        (lambda: q.qnn_cache_attention(x, *paged, slopes=g[:7]), "slopes must be dense"),
        (lambda: q.qnn_cache_attention(x, *paged, tree=z(4, dtype=i32)), "tree must have dtype"),
        (lambda: q.qnn_cache_attention(x, *paged, out=x.half()), "out must have dtype"),
        (lambda: q.qnn_rows_quant(g), "2-D"),
        (lambda: q.qnn_rows_quant(x[0], scale=g), "scale must be dense"),
    ]
    for call, message in cases:
        with pytest.raises(ValueError, match=message if device == "cuda" else message + "|must be a GPU tensor"):
            call()


def test_binding_refuses(q):
    _binding_refuses(q, "cpu")
    with pytest.raises(ValueError, match="must be a GPU tensor"):
        q.qnn_rows_quant(torch.zeros(4, 64))


@pytest.mark.gpu
def test_binding_refuses_on_the_gpu(q):
    _binding_refuses(q, "cuda")
    with pytest.raises(q.QnnError) as e:  # heads that do not divide
        z = lambda *n, dtype=torch.int32: torch.zeros(*n, dtype=dtype, device="cuda")
        q.qnn_cache_attention(z(1, 3, 64, dtype=torch.float32), q.qnn_new_cache(1, 2, 16, 64), z(1, 1), z(2), z(1))
    assert e.value.status == SHAPE


def test_workspaces_of_absurd_sizes():
    """Numbers whose products pass 64 bits: an answer, and no fault."""
    import paper_1609_07061_amd as q

    big = (1 << 63) - 1
    for tokens in (1, 1 << 31, 1 << 40, big):
        for other in (1, 1 << 30, 1 << 32, 1 << 48, big):
            for heads in (1, 65535):
                assert q.qnn_cache_attention_workspace_bytes(tokens, other, 65535, heads, 256, big, big) >= 0
                assert q.qnn_cache_attention_workspace_bytes(other, tokens, 65535, heads, 16, other, tokens) >= 0
                assert q.qnn_qk_norm_rotate_backward_workspace_bytes(tokens, other, heads, 256) >= 0
