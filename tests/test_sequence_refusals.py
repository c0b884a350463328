"""What the token-sequence entry points refuse (no GPU: nothing is launched when validation fails)."""
import ctypes

import pytest
import torch

from paper_2601_22275_amd import binding
from paper_2601_22275_amd.binding import Cache, RotaryPlan, Tokens

INVALID, UNSUPPORTED = -1, -2
INT = ctypes.c_void_p(1 << 12)  # never followed


def T(data=1 << 16, t=64, h=64):
    return ctypes.byref(Tokens(data, t, h))


def refuses(code, rc, text):
    assert rc == code, (rc, binding.lib().vmonarch_last_error())
    assert text in binding.lib().vmonarch_last_error().decode()


def attend(q=None, k=None, v=None, out=None, qs=INT, ks=INT, n=1, tq=8, tk=8, hq=4, hk=2, d=64, scale=1.0):
    return binding.lib().vmonarch_packed_attention(q or T(1 << 16), k or T(1 << 17), v or T(1 << 18), out or T(1 << 19), None, qs, ks, n, tq, tk, hq, hk, d,
                                                   scale, 1, None)


def test_packed_attention_refusals():
    refuses(INVALID, attend(hq=3), "no multiple")
    refuses(INVALID, attend(n=0), "out of range")
    refuses(INVALID, attend(d=0), "out of range")
    refuses(INVALID, attend(tq=-1), "out of range")
    refuses(UNSUPPORTED, attend(d=257), "exceeds 256")
    refuses(UNSUPPORTED, attend(tk=2 ** 31), "tokens")
    refuses(UNSUPPORTED, attend(tq=2 ** 30, hq=512, hk=1), "one launch")
    for s in (0.0, -1.0, float("nan"), float("inf")):
        refuses(INVALID, attend(scale=s), "scale")
    refuses(INVALID, attend(qs=None), "q_starts")
    refuses(INVALID, attend(ks=None), "k_starts")
    refuses(INVALID, attend(q=T(0)), "null q.data")
    refuses(INVALID, attend(k=T((1 << 17) + 1)), "not aligned")
    refuses(INVALID, attend(v=T(1 << 18, -64)), "negative strides of v")
    refuses(INVALID, attend(out=T(1 << 19, 0)), "stride of zero")
    refuses(INVALID, attend(out=T(1 << 19, 64, 0)), "stride of zero")
    refuses(INVALID, attend(out=T(1 << 16)), "must not be an input")
    assert attend(tq=0, q=T(0), out=T(0)) == 0  # nothing to do


def test_packed_attention_bwd_refusals():
    lib = binding.lib()

    def go(lse=INT, ws=None, size=0, **kw):
        x = {n: T((1 << 16) + (i << 12)) for i, n in enumerate(("q", "k", "v", "out", "d_out", "dq", "dk", "dv"))}
        x.update(kw)
        return lib.vmonarch_packed_attention_bwd_f32(x["q"], x["k"], x["v"], x["out"], x["d_out"], lse, x["dq"], x["dk"], x["dv"], INT, INT, 1, 8, 8, 4, 2, 64,
                                                     1.0, 1, ws, size, None)

    refuses(INVALID, go(lse=None), "null lse")
    refuses(INVALID, go(dq=T(1 << 16)), "dq must not be q")
    refuses(INVALID, go(dk=T((1 << 16) + (5 << 12))), "must not be")
    refuses(INVALID, go(ws=ctypes.c_void_p(256), size=0), "both")
    refuses(INVALID, go(ws=ctypes.c_void_p(100), size=4096), "256-byte")
    refuses(-3, go(ws=ctypes.c_void_p(256), size=16), "needed")
    refuses(INVALID, go(dv=T(1 << 20, 64, 0)), "stride of zero")
    size = lib.vmonarch_packed_attention_bwd_workspace_bytes
    assert size(1, 0, 8, 4, 2, 64) == 0 and size(1, 8, 8, 4, 3, 64) == 0 and size(0, 8, 8, 4, 2, 64) == 0
    assert size(1, 10, 8, 4, 2, 64) >= 320                       # two statistics per row
    assert size(1, 100000, 128, 4, 2, 64) > 2 * 100000 * 4 * 4   # and partial sums where rows are many and keys few


def cache(**kw):
    c = dict(k=1 << 20, v=1 << 21, k_page_stride=4096, k_token_stride=128, k_head_stride=64, v_page_stride=4096, v_token_stride=128, v_head_stride=64,
             n_pages=8, page_size=16, table=1 << 12, table_stride=4, table_width=4, lengths=1 << 13)
    c.update(kw)
    return ctypes.byref(Cache(*[c[f] for f, _ in Cache._fields_]))


def test_paged_refusals():
    lib = binding.lib()

    def read(c=None, hq=4, hk=2, out=None, ws=None, size=0):
        return lib.vmonarch_paged_attention(T(), c or cache(), out or T(1 << 19), INT, 1, 8, hq, hk, 64, 1.0, 1, ws, size, None)

    def write(c=None, plan=None, pos=None):
        return lib.vmonarch_paged_append(T(), T(1 << 18), c or cache(), INT, 1, 8, 2, 64, plan, pos, 8, None)

    for f in (read, write):
        refuses(INVALID, f(cache(k=None)), "cache.k")
        refuses(INVALID, f(cache(table=None)), "cache.table")
        refuses(INVALID, f(cache(lengths=None)), "cache.lengths")
        refuses(INVALID, f(cache(lengths=(1 << 13) + 2)), "not aligned")
        refuses(INVALID, f(cache(page_size=0)), "positive")
        refuses(INVALID, f(cache(n_pages=0)), "positive")
        refuses(INVALID, f(cache(v_token_stride=-1)), "negative strides of cache.v")
        refuses(INVALID, f(cache(k=(1 << 20) + 1)), "not aligned")
        refuses(UNSUPPORTED, f(cache(table_width=2 ** 20, page_size=2 ** 12)), "room")
    refuses(INVALID, read(hq=5), "no multiple")
    refuses(INVALID, read(out=T()), "must not be an input")
    refuses(INVALID, read(ws=ctypes.c_void_p(300), size=4096), "256-byte")
    refuses(INVALID, write(cache(k_token_stride=0)), "stride of zero")
    refuses(INVALID, write(pos=INT), "positions without a plan")
    refuses(INVALID, write(plan=ctypes.byref(binding.rotary_plan([8, 8]))), "needs positions")
    refuses(INVALID, write(plan=ctypes.byref(binding.rotary_plan([33]))), "turns 66 channels")


def test_rotary_refusals():
    lib = binding.lib()
    plan = binding.rotary_plan([16])

    def go(q=None, qo=None, k=None, ko=None, hk=0, tokens=8, d=64, pos=INT, p=plan):
        return lib.vmonarch_rotary(q or T(), qo or T(1 << 17), 4, k, ko, hk, tokens, d, pos, 8, ctypes.byref(p) if p else None, 0, None)

    refuses(INVALID, go(p=None), "null plan")
    refuses(INVALID, go(pos=None), "positions")
    refuses(INVALID, go(k=T()), "together")
    refuses(INVALID, go(d=30), "turns 32 channels")
    refuses(UNSUPPORTED, go(d=300), "exceeds 256")
    refuses(INVALID, go(qo=T(1 << 16, 128)), "in place")
    refuses(INVALID, go(qo=T(1 << 17, 0)), "stride of zero")
    refuses(INVALID, go(tokens=-1), "out of range")
    for field, value, text in (("layout", 2, "layout"), ("axes", 4, "axes"), ("struct_bytes", 8, "struct_bytes"), ("amplitude", float("nan"), "amplitude")):
        bad = binding.rotary_plan([16])
        setattr(bad, field, value)
        refuses(INVALID, go(p=bad), text)
    bad = binding.rotary_plan([16])
    bad.frequency[3] = float("inf")
    refuses(INVALID, go(p=bad), "frequency[3]")
    assert go(tokens=0, pos=None, q=T(0), qo=T(0)) == 0
    p = RotaryPlan()
    one = (ctypes.c_int * 1)(16)
    for args in ((2, 1e4, 1), (0, 0.0, 1), (0, float("inf"), 1), (0, 1e4, 0), (0, 1e4, 4)):
        assert lib.vmonarch_rotary_init(ctypes.byref(p), *args, one) == INVALID
    assert lib.vmonarch_rotary_init(ctypes.byref(p), 0, 1e4, 1, (ctypes.c_int * 1)(129)) == INVALID
    for args in ((0.0, 0.0, 0.0, 0.0), (2.0, -1.0, 0.0, 1.0), (2.0, 100.0, 1.0, 1.0), (float("nan"), 0.0, 0.0, 0.0)):
        assert lib.vmonarch_rotary_scale(ctypes.byref(plan), *args) == INVALID


def test_rotary_frequencies():
    import numpy as np

    from tests import sequence_oracle as S
    for kw in (dict(), dict(base=500.0), dict(factor=4.0), dict(factor=8.0, context=2048.0, low_turns=1.0, high_turns=32.0)):
        p = binding.rotary_plan([5, 3, 2], **kw)
        f = S.frequencies([5, 3, 2], kw.get("base", 1e4), kw.get("factor", 1.0), kw.get("context", 0.0), kw.get("low_turns", 0.0), kw.get("high_turns", 0.0))
        assert np.allclose(np.array(p.frequency[:10]), f, rtol=1e-14, atol=0)


def test_binding_refuses_what_is_not_a_device_tensor():
    x = torch.zeros(4, 2, 8)
    s = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(binding.VMonarchError):
        binding.packed_attention(x, x, x, s)
    with pytest.raises(binding.VMonarchError):
        binding.rotary(x, None, s, binding.rotary_plan([2]))


def test_counts_at_the_edge_of_32_bits():
    # kernels look some tiles past the last token, so the last 2^16 counts are refused too
    refuses(UNSUPPORTED, attend(tk=2 ** 31 - 65535), "tokens")
    refuses(UNSUPPORTED, attend(tq=2 ** 30 - 32767, hq=4, hk=2), "one launch")
    refuses(UNSUPPORTED, attend(n=2 ** 30), "sequences")
    lib = binding.lib()
    wide = cache(table_width=2 ** 20 - 31, page_size=2 ** 11)  # 2^31 - 63488
    refuses(UNSUPPORTED, lib.vmonarch_paged_attention(T(), wide, T(1 << 19), INT, 1, 8, 4, 2, 64, 1.0, 1, None, 0, None), "room")
    refuses(UNSUPPORTED, lib.vmonarch_paged_append(T(), T(1 << 18), wide, INT, 1, 8, 2, 64, None, None, 8, None), "room")
    plan = binding.rotary_plan([16])
    refuses(UNSUPPORTED, lib.vmonarch_rotary(T(), T(1 << 18), 1, None, None, 0, 2 ** 31 - 65535, 64, INT, 8, ctypes.byref(plan), 0, None), "tokens")


def test_packed_descriptors_are_the_structures():
    assert binding._pack_tokens(1 << 40, 3, 1 << 33) == bytes(Tokens(1 << 40, 3, 1 << 33))
    values = (1 << 40, 1 << 41, 1, 2, 3, 4, 5, 1 << 33, 6, 7, 1 << 42, 1 << 34, 8, 1 << 43)
    assert binding._pack_cache(*values) == bytes(Cache(*values))
