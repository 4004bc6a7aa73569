"""The paged cache's C ABI without a GPU: symbols, struct sizes, and every refusal - found on the host before any HIP call (fake
pointers are never dereferenced because no launch happens).  Then the Python layer's own refusals."""
import ctypes
import os
import re
import subprocess

import pytest
import torch

from paper_2502_14882_amd import binding as cq
from paper_2502_14882_amd import paged

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000
ABI = ["cqp_append_kv", "cqp_attn", "cqp_attn_workspace_bytes", "cqp_rotate"]
by = ctypes.byref


def test_symbols():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "cq_paged.h")).read(), flags=re.S)
    assert sorted(set(re.findall(r"\b(cqp_[a-z_0-9]+)\s*\(", text))) == ABI
    out = subprocess.run(["nm", "-D", "--defined-only", cq.LIB_PATH], capture_output=True, text=True)
    if out.returncode != 0:
        pytest.skip("nm is not available")
    assert sorted({l.split()[-1] for l in out.stdout.splitlines() if l.split()[-1].startswith("cqp_")}) == ABI


def test_header_is_c_and_the_structs_have_its_sizes(tmp_path):
    src = tmp_path / "s.c"
    src.write_text('#include "cq_paged.h"\n#include <stdio.h>\nint main(void) { printf("%zu %zu %zu %zu", sizeof(cqp_heads_t), '
                   'sizeof(cqp_cache_t), sizeof(cqp_batch_t), sizeof(cqp_rope_t)); return 0; }\n')
    exe = str(tmp_path / "s")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    sizes = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    assert sizes == [ctypes.sizeof(c) for c in (paged.CqpHeads, paged.CqpCache, paged.CqpBatch, paged.CqpRope)]


def heads(n=2, token=None, head=None, data=FAKE, d=128, reserved=0):
    return paged.CqpHeads(data, n * d if token is None else token, d if head is None else head, n, reserved)


def rope(rot=128, axes=3, pairs=0, freq=FAKE, axis=0, reserved=0):
    return paged.CqpRope(rot, axes, pairs, reserved, freq, (ctypes.c_uint8 * 128)(*([axis] * 128)))


def cache(n_pages=10, page=64, hk=2, d=128, kc=FAKE, vc=FAKE, ks=FAKE, vs=FAKE):
    return paged.CqpCache(n_pages, page, hk, d, kc, vc, ks, vs)


def batch(b=2, max_pages=4, max_new=1, max_len=256, table=FAKE, lens=FAKE, starts=FAKE):
    return paged.CqpBatch(b, max_pages, max_new, max_len, table, lens, starts)


def rotate(r=rope(), pos=FAKE, n=4, d=128, dtype=0, backward=0, i=None, o=None, count=1):
    i, o = i or heads(), o or heads()
    return paged.lib().cqp_rotate(by(r) if r else None, pos, n, d, dtype, backward, by(i), by(o), count, None)


def test_rotate_refusals():
    assert rotate(n=0) == cq.CQ_OK                                   # empty: no launch
    assert rotate(r=None) == cq.CQ_ERR_NULL
    assert rotate(pos=None) == cq.CQ_ERR_NULL
    assert rotate(pos=FAKE + 2) == cq.CQ_ERR_ALIGN
    assert rotate(r=rope(freq=None)) == cq.CQ_ERR_NULL
    assert rotate(r=rope(freq=FAKE + 1)) == cq.CQ_ERR_ALIGN
    for rot in (0, 8, 24, 144, -16):
        assert rotate(r=rope(rot=rot)) == cq.CQ_ERR_SHAPE
    assert rotate(r=rope(axes=0)) == cq.CQ_ERR_SHAPE
    assert rotate(r=rope(axes=5)) == cq.CQ_ERR_SHAPE
    assert rotate(r=rope(axes=2, axis=2)) == cq.CQ_ERR_SHAPE
    assert b"axis_of[0]" in paged.lib().cq_last_error()
    assert rotate(r=rope(pairs=2)) == cq.CQ_ERR_UNSUPPORTED
    assert rotate(r=rope(reserved=1)) == cq.CQ_ERR_SHAPE
    assert rotate(n=-1) == cq.CQ_ERR_SHAPE
    for d in (0, 16, 100, 288):
        assert rotate(d=d) == cq.CQ_ERR_SHAPE
    assert rotate(dtype=2) == cq.CQ_ERR_UNSUPPORTED
    assert rotate(backward=2) == cq.CQ_ERR_UNSUPPORTED
    assert rotate(count=0) == cq.CQ_ERR_SHAPE
    assert rotate(count=3) == cq.CQ_ERR_SHAPE
    assert rotate(i=heads(data=None)) == cq.CQ_ERR_NULL
    assert rotate(i=heads(data=FAKE + 8)) == cq.CQ_ERR_ALIGN
    assert rotate(i=heads(token=260)) == cq.CQ_ERR_ALIGN
    assert rotate(i=heads(token=-256)) == cq.CQ_ERR_ALIGN
    assert rotate(i=heads(n=0)) == cq.CQ_ERR_SHAPE
    assert rotate(i=heads(reserved=1)) == cq.CQ_ERR_SHAPE
    assert rotate(o=heads(n=3)) == cq.CQ_ERR_SHAPE                   # another number of heads
    assert rotate(o=heads(head=64)) == cq.CQ_ERR_SHAPE               # rows of the result overlap
    assert rotate(o=heads(token=128)) == cq.CQ_ERR_SHAPE
    assert rotate(o=heads(token=0)) == cq.CQ_ERR_SHAPE
    assert rotate(o=heads(token=128, head=256)) == cq.CQ_ERR_SHAPE   # 4 tokens of 128 do not fit between heads 256 apart
    L = paged.lib()
    assert L.cqp_rotate(by(rope()), FAKE, 4, 128, 0, 0, None, by(heads()), 1, None) == cq.CQ_ERR_NULL
    assert L.cqp_rotate(by(rope()), FAKE, 4, 128, 0, 0, by(heads()), None, 1, None) == cq.CQ_ERR_NULL


def append(c=cache(), s=batch(), n=2, dtype=0, k=None, v=None, r=None, pos=None, qi=None, qo=None):
    k, v = k or heads(), v or heads()
    return paged.lib().cqp_append_kv(by(c) if c else None, by(s) if s else None, n, dtype, by(k), by(v), by(r) if r else None, pos,
                                     by(qi) if qi else None, by(qo) if qo else None, None)


def attend(c=cache(), s=batch(), n=2, dtype=0, q=None, o=None, lse=None, causal=1, scale=0.0, ws=FAKE, nbytes=1 << 40):
    q, o = q or heads(8), o or heads(8)
    return paged.lib().cqp_attn(by(c) if c else None, by(s) if s else None, n, dtype, by(q), by(o), lse, causal, scale, ws, nbytes, None)


@pytest.mark.parametrize("call", (append, attend))
def test_refusals_of_caches_and_batches(call):
    assert call(n=0) == cq.CQ_OK
    assert call(c=None) == cq.CQ_ERR_NULL
    assert call(s=None) == cq.CQ_ERR_NULL
    for kw in (dict(n_pages=0), dict(hk=0), dict(d=100), dict(d=288), dict(page=8), dict(page=48), dict(page=512), dict(page=0)):
        assert call(c=cache(**kw)) == cq.CQ_ERR_SHAPE, kw
    for kw in (dict(kc=None), dict(vc=None), dict(ks=None), dict(vs=None)):
        assert call(c=cache(**kw)) == cq.CQ_ERR_NULL, kw
    for kw in (dict(kc=FAKE + 8), dict(vc=FAKE + 8), dict(ks=FAKE + 2), dict(vs=FAKE + 1)):
        assert call(c=cache(**kw)) == cq.CQ_ERR_ALIGN, kw
    for kw in (dict(b=0), dict(max_pages=0), dict(max_new=0), dict(max_len=0), dict(max_len=2147483647, max_pages=1 << 30)):
        assert call(s=batch(**kw)) == cq.CQ_ERR_SHAPE, kw
    for kw in (dict(table=None), dict(lens=None), dict(starts=None)):
        assert call(s=batch(**kw)) == cq.CQ_ERR_NULL, kw
    for kw in (dict(table=FAKE + 2), dict(lens=FAKE + 1), dict(starts=FAKE + 2)):
        assert call(s=batch(**kw)) == cq.CQ_ERR_ALIGN, kw
    assert call(n=-1) == cq.CQ_ERR_SHAPE
    assert call(dtype=7) == cq.CQ_ERR_UNSUPPORTED


def test_append_refusals():
    assert append(k=heads(3)) == cq.CQ_ERR_SHAPE
    assert append(v=heads(1)) == cq.CQ_ERR_SHAPE
    assert append(v=heads(data=None)) == cq.CQ_ERR_NULL
    assert append(k=heads(head=100)) == cq.CQ_ERR_ALIGN
    assert append(pos=FAKE) == cq.CQ_ERR_NULL                        # positions without a rope
    assert append(r=rope()) == cq.CQ_ERR_NULL                        # a rope without positions
    assert append(r=rope(rot=256), pos=FAKE) == cq.CQ_ERR_SHAPE
    assert append(qi=heads(8), qo=heads(8)) == cq.CQ_ERR_NULL        # queries without a rope
    assert append(r=rope(), pos=FAKE, qi=heads(8)) == cq.CQ_ERR_NULL
    assert append(r=rope(), pos=FAKE, qi=heads(8), qo=heads(4)) == cq.CQ_ERR_SHAPE
    assert append(r=rope(), pos=FAKE, qi=heads(8), qo=heads(8, token=512)) == cq.CQ_ERR_SHAPE


def test_attention_refusals():
    need = paged.lib().cqp_attn_workspace_bytes(by(cache()), by(batch()), 2, 8)
    assert need > 0 and need % 256 == 0
    assert attend(q=heads(7), o=heads(7)) == cq.CQ_ERR_SHAPE
    assert attend(q=heads(8), o=heads(4)) == cq.CQ_ERR_SHAPE
    assert attend(o=heads(8, token=0)) == cq.CQ_ERR_SHAPE
    assert attend(lse=FAKE + 2) == cq.CQ_ERR_ALIGN
    assert attend(causal=2) == cq.CQ_ERR_UNSUPPORTED
    for scale in (-1.0, float("nan"), float("inf")):
        assert attend(scale=scale) == cq.CQ_ERR_SHAPE
    assert attend(ws=None) == cq.CQ_ERR_WORKSPACE
    assert attend(ws=FAKE + 64) == cq.CQ_ERR_WORKSPACE
    assert attend(nbytes=need - 1) == cq.CQ_ERR_WORKSPACE


def test_calls_too_large_for_a_launch():
    L = paged.lib()
    many = batch(b=1 << 22, max_new=4)
    assert L.cqp_attn_workspace_bytes(by(cache(hk=8)), by(many), 1 << 22, 8) == 0
    assert attend(c=cache(hk=8), s=many, n=1 << 22, q=heads(8), o=heads(8)) == cq.CQ_ERR_SHAPE
    assert b"too many" in L.cq_last_error()
    assert attend(s=batch(max_new=1 << 30), n=1 << 30, q=heads(8), o=heads(8)) == cq.CQ_ERR_SHAPE
    assert rotate(n=1 << 30, i=heads(64), o=heads(64)) == cq.CQ_ERR_SHAPE
    assert append(s=batch(b=1 << 27), n=1 << 27) == cq.CQ_ERR_SHAPE


def test_workspace_sizes():
    f = paged.lib().cqp_attn_workspace_bytes
    assert f(by(cache()), by(batch()), 2, 7) == 0
    assert f(by(cache()), by(batch()), -1, 8) == 0
    assert f(by(cache(page=10)), by(batch()), 2, 8) == 0
    assert f(by(cache()), by(batch(max_len=0)), 2, 8) == 0
    assert f(None, by(batch()), 2, 8) == 0 and f(by(cache()), None, 2, 8) == 0
    for kw in (dict(kc=None, vc=None, ks=None, vs=None),):           # a size query needs no tensors
        assert f(by(cache(**kw)), by(batch(table=None, lens=None, starts=None)), 2, 8) > 0
    short, long = (f(by(cache()), by(batch(b=1, max_pages=1 << 12, max_len=n)), 1, 8) for n in (64, 1 << 17))
    assert short == 256 < long < 8 << 20


def test_python_refusals():
    z = torch.zeros
    codes = lambda *s: z(s, dtype=torch.uint8)          # noqa: E731
    f32 = lambda *s: z(s)                               # noqa: E731
    i32 = lambda *s: z(s, dtype=torch.int32)            # noqa: E731
    good = paged.PagedCache(codes(4, 2, 16, 64), codes(4, 2, 64, 16), f32(4, 2), f32(4, 2))
    for bad in ((codes(4, 2, 16, 64), codes(4, 2, 16, 64), f32(4, 2), f32(4, 2)), (codes(4, 2, 16, 64), codes(4, 2, 64, 16), f32(4), f32(4, 2)),
                (f32(4, 2, 16, 64), codes(4, 2, 64, 16), f32(4, 2), f32(4, 2)), (codes(4, 2, 8, 64), codes(4, 2, 64, 8), f32(4, 2), f32(4, 2)),
                (codes(4, 2, 16, 128)[..., ::2], codes(4, 2, 64, 16), f32(4, 2), f32(4, 2)), (codes(16, 64), codes(64, 16), f32(4, 2), f32(4, 2))):
        with pytest.raises(ValueError):
            paged.PagedCache(*bad)
    step = paged.PagedBatch(i32(2, 3), i32(2), i32(3), 1, 48)
    for bad in ((i32(2), i32(2), i32(3)), (i32(2, 3), i32(3), i32(3)), (i32(2, 3), i32(2), i32(2)), (i32(2, 3).long(), i32(2), i32(3)),
                (i32(2, 6)[:, ::2], i32(2), i32(3))):
        with pytest.raises(ValueError):
            paged.PagedBatch(*bad, 1, 48)
    turn = paged.Rope(f32(32), [0] * 16 + [1] * 16)
    assert turn.n_axes == 2
    for bad in ((f32(32, 1),), (f32(32).double(),), (f32(32), [0] * 31), (f32(32), [4] * 32), (f32(129),)):
        with pytest.raises(ValueError):
            paged.Rope(*bad)
    h = lambda n, d=64, t=2: z((t, n, d), dtype=torch.float16)      # noqa: E731
    for bad in (lambda: paged.cqp_rotate(turn, i32(2, 2), []), lambda: paged.cqp_rotate(turn, i32(2, 3), h(4)),
                lambda: paged.cqp_rotate(turn, i32(3, 2), h(4)), lambda: paged.cqp_rotate(turn, i32(2, 2), h(4).float()),
                lambda: paged.cqp_rotate(turn, i32(2, 2), [h(4), h(2, 32)]), lambda: paged.cqp_rotate(turn, i32(2, 2), h(4), out=h(4, t=3)),
                lambda: paged.cqp_rotate(turn, i32(2, 2), h(4)),      # no GPU tensors
                lambda: paged.cqp_append_kv(good, step, h(2), h(2), turn), lambda: paged.cqp_append_kv(good, step, h(2), h(2), q=h(4)),
                lambda: paged.cqp_append_kv(good, step, h(2), h(2, t=3)), lambda: paged.cqp_append_kv(good, step, h(2), h(2).bfloat16()),
                lambda: paged.cqp_append_kv(good, step, h(2), h(2), q_out=h(4)), lambda: paged.cqp_append_kv(good, step, h(2, 128), h(2, 128)),
                lambda: paged.cqp_append_kv(good, step, z((2, 64, 2), dtype=torch.float16).transpose(1, 2), h(2)),
                lambda: paged.cqp_append_kv(good, step, h(2), h(2)),
                lambda: paged.cqp_attn(good, step, h(4, 128)), lambda: paged.cqp_attn(good, step, h(4)[0]), lambda: paged.cqp_attn(good, step, h(4), out=h(2)),
                lambda: paged.cqp_attn(good, step, h(4), lse=f32(2, 4).double()), lambda: paged.cqp_attn(good, step, h(4), out=h(4).bfloat16()),
                lambda: paged.cqp_attn(good, step, h(4))):
        with pytest.raises(ValueError):
            bad()
