"""What the drafting operators answer before they touch a device, and the host's side of 4-bit weights.  No GPU needed."""
import ctypes as C

import pytest
import torch

from paper_2501_08090_amd import binding as B
from paper_2501_08090_amd.drafting import quantize4

INVALID, SHAPE = -1, -2
FAKE = 1 << 20  # an aligned address that is never read: every call here is refused first


def code_of(call, *args):
    rc = call(*args)
    assert rc == 0 or B.last_error() != ""
    return rc


def test_null_handles():
    lib = B.load()
    assert lib.chiron_kv_index_bytes(None) == 0 and lib.chiron_linear4_workspace_bytes(None, 5) == 0
    assert lib.chiron_kv_index_destroy(None) == 0 and lib.chiron_linear4_destroy(None) == 0
    out = C.c_void_p(5)
    assert code_of(lib.chiron_kv_index_create, None, C.c_void_p(FAKE), C.c_uint64(1), C.byref(out)) == INVALID and not out.value
    assert code_of(lib.chiron_kv_index_create, None, C.c_void_p(FAKE), C.c_uint64(1), None) == INVALID
    assert code_of(lib.chiron_kv_index_update, None, None, 0, 1, FAKE, 1, FAKE, FAKE, 1, 1, None) == INVALID
    assert code_of(lib.chiron_append_kv_rope, None, None, 0, None, FAKE, 1, FAKE, FAKE, 1, 1, None) == INVALID
    assert code_of(lib.chiron_op_select_pages, None, None, None, 0, FAKE, FAKE, None, FAKE, 1, 1, 0, 0, FAKE, FAKE, None) == INVALID
    assert code_of(lib.chiron_op_sparse_attention, None, None, 0, FAKE, FAKE, None, FAKE, 1, FAKE, FAKE, 1, FAKE, None) == INVALID
    assert code_of(lib.chiron_op_verify_drafts, None, 1, 1, 4, FAKE, FAKE, FAKE, FAKE, None) == INVALID
    assert code_of(lib.chiron_op_linear4, None, FAKE, 1, FAKE, 0, None, None) == INVALID


def draft_batch(**kw):
    b = B.DraftBatch()
    b.logits = b.draft_logits = b.tokens = b.uniforms = b.noise = FAKE
    b.logits_stride = b.draft_stride = 100
    for k, v in kw.items():
        setattr(b, k, v)
    return b


@pytest.mark.parametrize("kw,batch,drafts,vocab,out,work,want", (
    ({}, -1, 4, 100, FAKE, FAKE, INVALID),
    ({}, 1, -1, 100, FAKE, FAKE, INVALID),
    ({}, 1, 4, 0, FAKE, FAKE, INVALID),
    ({}, 1, 128, 100, FAKE, FAKE, SHAPE),
    ({}, 1, 4, 101, FAKE, FAKE, INVALID),                       # rows closer than a row is long
    (dict(draft_stride=99), 1, 4, 100, FAKE, FAKE, INVALID),
    (dict(logits=None), 1, 4, 100, FAKE, FAKE, INVALID),
    (dict(noise=None), 1, 4, 100, FAKE, FAKE, INVALID),
    (dict(tokens=None), 1, 4, 100, FAKE, FAKE, INVALID),
    (dict(uniforms=None), 1, 4, 100, FAKE, FAKE, INVALID),
    ({}, 1, 4, 100, None, FAKE, INVALID),
    ({}, 1, 4, 100, FAKE, None, INVALID),
    ({}, 1, 4, 100, FAKE, FAKE + 8, INVALID),
    ({}, 258, 127, 100, FAKE, FAKE, "too large"),
    (dict(logits=None, tokens=None), 0, 4, 100, None, None, 0),  # no request: nothing to do
))
def test_verify_refusals(kw, batch, drafts, vocab, out, work, want):
    b = draft_batch(**kw)
    rc = B.load().chiron_op_verify_drafts(C.addressof(b), batch, drafts, vocab, out, FAKE, FAKE, work, None)
    assert rc == want if want != "too large" else rc < 0 and "too many" in B.last_error()


def test_verify_workspace():
    bytes_of = B.load().chiron_verify_workspace_bytes
    assert bytes_of(1, 0, 1) > 0
    for bad in ((-1, 4, 100), (1, -1, 100), (1, 128, 100), (1, 4, 0)):
        assert bytes_of(*bad) == 0
    assert bytes_of(0, 4, 100) == 0
    for a, b in (((1, 4, 1000), (2, 4, 1000)), ((1, 4, 1000), (1, 5, 1000)), ((1, 4, 1000), (1, 4, 100000))):
        assert 0 < bytes_of(*a) < bytes_of(*b) and bytes_of(*a) % 16 == 0


@pytest.mark.parametrize("n,k,group,scales,want", (
    (0, 128, 128, FAKE, INVALID), (8, 0, 128, FAKE, INVALID), (8, 128, 16, FAKE, SHAPE), (8, 128, 256, FAKE, SHAPE), (8, 160, 64, FAKE, SHAPE),
    (8, 128, 0, FAKE, SHAPE), (8, 128, 128, None, INVALID), (8, 128, 128, FAKE + 1, INVALID), (8, 1 << 23, 128, FAKE, SHAPE),
    (0x7fffffff, 1 << 22, 128, FAKE, SHAPE)))
def test_linear4_create_refusals(n, k, group, scales, want):
    out = C.c_void_p(5)
    rc = B.load().chiron_linear4_create(C.c_void_p(FAKE), C.c_void_p(scales), None, C.c_int32(n), C.c_int32(k), C.c_int32(group), None, C.byref(out))
    assert rc == want and not out.value and B.last_error() != ""
    assert B.load().chiron_linear4_create(C.c_void_p(FAKE), C.c_void_p(FAKE), None, C.c_int32(8), C.c_int32(128), C.c_int32(128), None, None) == INVALID


@pytest.mark.parametrize("group", (32, 64, 128))
def test_quantize4(group):
    g = torch.Generator().manual_seed(group)
    w = torch.randn((9, 4 * group), generator=g) * torch.rand((9, 1), generator=g)
    w[2] = 0
    w[3, :group] = 0
    w4, s = quantize4(w, group)
    assert w4.shape == (9, 2 * group) and w4.dtype == torch.uint8 and s.shape == (9, 4) and s.dtype == torch.bfloat16
    q = torch.stack((w4 & 15, w4 >> 4), -1).view(9, 4, group).double() - 8
    x, step = w.double().view(9, 4, group), s.double()[..., None]
    # to the nearest step; the largest value is 7 steps but for the scale's rounding to 8 bits, at most 7 * 2^-9 of a step more
    assert ((x - q * step).abs() <= step * (0.5 + 7 * 2.0 ** -8)).all()
    assert (q[2] == 0).all() and (q[3, 0] == 0).all() and (s[2] == 0).all()
    assert (q.abs().amax(-1)[s != 0] == 7).all()
