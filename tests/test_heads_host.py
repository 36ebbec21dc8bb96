"""Rows of heads and the 4-bit cache: what the library refuses before anything is launched, and the reference's own pins."""
import ctypes

import numpy as np
import pytest
import torch

import heads_reference as ref
from paper_2608_13426_b200 import binding
from paper_2608_13426_b200 import build as rmm_build

OK_WS = (ctypes.c_void_p(4096), 1 << 30)
BAD, ODD, WS = binding.RMM_ERR_INVALID_ARG, binding.RMM_ERR_UNSUPPORTED, binding.RMM_ERR_WORKSPACE


@pytest.fixture(scope="module")
def L():
    rmm_build.build()
    return binding.lib()


def heads(ptr=4096, dtype=0, B=2, H=4, L=3, D=128, stride=None):
    return binding.rmm_heads_t(ptr, dtype, B, H, L, D, (ctypes.c_int64 * 3)(*(stride or (H * L * D, L * D, D))))


def cache(**kw):
    c = dict(pool=4096, n_pages=8, page=64, Hkv=2, Dh=128, page_stride=2 * 4 * 2304, head_stride=4 * 2304, pages=4096, B=2, max_pages=4,
             pages_stride=4, lengths=4096, new_len=None)
    c.update(kw)
    return binding.rmm_kv4_t(*c.values())


def rope(**kw):
    c = dict(table=4096, table_rows=10, table_stride=128, rot=128, interleaved=0, weight_dtype=1, eps=1e-6, positions=None, pos_stride=(0, 0))
    c.update(kw)
    c["pos_stride"] = (ctypes.c_int64 * 2)(*c["pos_stride"])
    return binding.rmm_rope_t(*c.values())


def test_struct_layouts_match_header():
    assert ctypes.sizeof(binding.rmm_heads_t) == 8 + 8 + 4 * 8 + 3 * 8
    assert ctypes.sizeof(binding.rmm_rope_t) == 8 + 3 * 8 + 2 * 4 + 8 + 8 + 2 * 8
    assert ctypes.sizeof(binding.rmm_kv4_t) == 8 + 4 * 8 + 2 * 8 + 8 + 3 * 8 + 2 * 8


def test_norm_rope_refusals(L):
    def call(Q=heads(), K=heads(H=2), qw=None, kw=None, r=rope(), Qo=heads(), Ko=heads(H=2), ws=OK_WS):
        return L.rmm_qk_norm_rope(Q, K, qw, kw, r, Qo, Ko, *ws, None)

    for kw, code in [(dict(Q=None), BAD), (dict(Q=heads(ptr=None)), BAD), (dict(Q=heads(L=0)), BAD), (dict(Q=heads(dtype=2)), ODD),
                     (dict(Q=heads(stride=(-1, 1, 1))), ODD), (dict(Q=heads(ptr=4097)), ODD), (dict(Qo=heads(H=5)), BAD), (dict(Ko=None), BAD),
                     (dict(K=heads(H=2, L=4)), BAD), (dict(K=heads(H=2, dtype=1)), ODD), (dict(Ko=heads(H=2, dtype=1)), ODD),
                     (dict(qw=4096, r=None), BAD), (dict(r=rope(rot=0)), BAD), (dict(r=rope(rot=144)), BAD), (dict(r=rope(rot=40)), ODD),
                     (dict(r=rope(table_rows=0)), BAD), (dict(r=rope(table_stride=100)), BAD), (dict(r=rope(table=4098)), ODD),
                     (dict(qw=4096, r=rope(eps=-1.0)), BAD), (dict(qw=4096, r=rope(weight_dtype=2)), ODD), (dict(kw=4098), ODD),
                     (dict(r=rope(positions=4098)), ODD), (dict(r=rope(positions=4096, pos_stride=(-1, 1))), ODD),
                     (dict(Q=heads(D=260), Qo=heads(D=260), K=None, Ko=None), ODD), (dict(Q=heads(D=12), Qo=heads(D=12), K=None, Ko=None, r=None), ODD),
                     (dict(ws=(None, 1 << 20)), WS), (dict(ws=(ctypes.c_void_p(4100), 1 << 20)), WS), (dict(ws=(ctypes.c_void_p(4096), 4095)), WS)]:
        assert call(**kw) == code, kw


def test_cache_refusals(L):
    k, v, q, o = heads(H=2), heads(H=2), heads(), heads()
    for c, code in [(None, BAD), (cache(pool=None), BAD), (cache(pages=None), BAD), (cache(lengths=None), BAD), (cache(Dh=96), ODD),
                    (cache(B=3), BAD), (cache(n_pages=0), BAD), (cache(max_pages=0), BAD), (cache(page=48), ODD), (cache(page=8), ODD),
                    (cache(pool=4104), ODD), (cache(head_stride=4 * 2304 + 8), ODD), (cache(head_stride=3 * 2304), BAD), (cache(page_stride=2304), BAD),
                    (cache(pages_stride=-1), ODD), (cache(max_pages=1 << 40), ODD), (cache(lengths=4097), ODD), (cache(new_len=4098), ODD)]:
        assert L.rmm_kv4_append(k, v, c, None, None, None, None, *OK_WS, None) == code
        assert L.rmm_kv4_read(c, k, v, *OK_WS, None) == code
        assert L.rmm_kv4_attn(q, c, 1, 1.0, o, None, *OK_WS, None) == code
        assert L.rmm_kv4_attn_workspace_bytes(q, c) == 0
    c = cache()
    need = L.rmm_kv4_attn_workspace_bytes(q, c)
    assert need > 4096
    for args, code in [((heads(H=3), v, c, None, None, None, None), BAD), ((k, heads(H=2, dtype=1), c, None, None, None, None), ODD),
                       ((heads(H=3), heads(H=3), c, None, None, None, None), BAD), ((k, v, c, None, None, k, None), BAD),
                       ((k, v, c, None, None, heads(H=2, dtype=1), heads(H=2, dtype=1)), ODD), ((k, v, c, 4096, None, None, None), BAD),
                       ((k, v, c, None, rope(rot=24), None, None), ODD)]:
        assert L.rmm_kv4_append(*args, *OK_WS, None) == code
    assert L.rmm_kv4_append(k, v, c, None, None, None, None, ctypes.c_void_p(4096), 100, None) == WS
    assert L.rmm_kv4_read(c, heads(H=4), heads(H=4), *OK_WS, None) == BAD
    assert L.rmm_kv4_read(c, k, heads(H=2, dtype=1), *OK_WS, None) == ODD
    for args, code in [((heads(H=3), c, 1, 1.0, heads(H=3)), BAD), ((heads(D=64), c, 1, 1.0, heads(D=64)), BAD), ((heads(dtype=1), c, 1, 1.0, o), ODD),
                       ((q, c, 1, 1.0, heads(dtype=1)), ODD), ((q, c, 1, 0.0, o), BAD), ((q, c, 1, 1.5, o), BAD), ((q, c, 1, float("nan"), o), BAD),
                       ((heads(L=17), c, 1, 0.5, heads(L=17)), ODD), ((q, c, 1, 1.0, None), BAD)]:
        assert L.rmm_kv4_attn(*args, None, *OK_WS, None) == code
    assert L.rmm_kv4_attn(q, c, 1, 1.0, o, None, ctypes.c_void_p(4096), need - 1, None) == WS
    many = cache(B=1 << 20, max_pages=1 << 20)
    assert L.rmm_kv4_attn(heads(B=1 << 20), many, 1, 1.0, heads(B=1 << 20), None, *OK_WS, None) == ODD   # the blocks' axis passes 2^31


def test_outputs_that_overlap_are_refused(L):
    """An element that two rows write has no one value: an expanded output, rows that reach into the next, one array for two outputs."""
    there = 1 << 20
    for o in (heads(there, stride=(0, 384, 128)), heads(there, stride=(1536, 0, 128)), heads(there, stride=(1536, 384, 0)),
              heads(there, stride=(1536, 384, 120)), heads(there, stride=(1528, 384, 128)), heads(there, stride=(128, 512, 128))):
        assert L.rmm_qk_norm_rope(heads(), None, None, None, rope(), o, None, *OK_WS, None) == BAD
        assert L.rmm_kv4_attn(heads(), cache(), 1, 1.0, o, None, *OK_WS, None) == BAD
        c = cache(Hkv=4, page_stride=4 * 4 * 2304)
        assert L.rmm_kv4_read(c, o, heads(), *OK_WS, None) == BAD and L.rmm_kv4_read(c, heads(), o, *OK_WS, None) == BAD
        assert L.rmm_kv4_append(heads(), heads(), c, None, None, o, heads(), *OK_WS, None) == BAD
        assert L.rmm_kv4_append(heads(), heads(), c, None, None, heads(), o, *OK_WS, None) == BAD
    k = heads(H=2)
    assert L.rmm_qk_norm_rope(heads(), k, None, None, rope(), heads(there), heads(there, H=2), *OK_WS, None) == BAD
    assert L.rmm_kv4_read(cache(), k, k, *OK_WS, None) == BAD
    assert L.rmm_kv4_append(k, k, cache(), None, None, heads(there, H=2), heads(there, H=2), *OK_WS, None) == BAD
    # in place: another dtype, other strides
    assert L.rmm_qk_norm_rope(heads(), None, None, None, rope(), heads(dtype=1), None, *OK_WS, None) == BAD
    assert L.rmm_qk_norm_rope(heads(), None, None, None, rope(), heads(stride=(1536, 128, 512)), None, *OK_WS, None) == BAD
    assert L.rmm_kv4_attn(heads(), cache(), 1, 1.0, heads(there), ctypes.c_void_p(4098), *OK_WS, None) == ODD


def test_tensors_that_are_not_the_calls():
    q = torch.zeros(1, 2, 3, 64, dtype=torch.bfloat16)
    for f in (lambda: binding.rmm_qk_norm_rope(q), lambda: binding.rmm_qk_norm_rope(None), lambda: binding.rmm_kv4_append(q, q, None, None, None),
              lambda: binding.rmm_kv4_read(torch.zeros(2, 1, 1, 1152, dtype=torch.uint8), None, None), lambda: binding.rmm_kv4_read(None, None, None),
              lambda: binding.rmm_kv4_attn(q, None, None, None)):
        with pytest.raises(binding.RmmError) as e:
            f()
        assert e.value.code == BAD
    for args in [(4, 1, 128, 48), (4, 1, 96, 64), (4, 1, 128, 8)]:
        with pytest.raises(binding.RmmError) as e:
            binding.rmm_kv4_pool(*args, device="cpu")
        assert e.value.code == ODD
    assert binding.rmm_kv4_pool(3, 2, 64, 32, device="cpu").shape == (3, 2, 2, 1152)


def test_the_table_holds_cosines_then_sines():
    t = binding.rmm_rope_table(70000, 64, 500000.0)
    assert t.shape == (70000, 64) and t.dtype == torch.float32
    for p, j in [(0, 0), (1, 3), (69999, 0), (69999, 31)]:
        a = p * 500000.0 ** (-2 * j / 64)
        assert abs(t[p, j].item() - np.cos(a)) < 1e-7 and abs(t[p, 32 + j].item() - np.sin(a)) < 1e-7


def test_reference_pins():
    x = torch.tensor([[0.0, 15.0] + [7.5] * 62]).bfloat16()
    n, step, low = ref.quantise(x)
    assert step.item() == 1.0 and low.item() == 0.0 and n[0, :3].tolist() == [0, 15, 8]         # 7.5: halves to the even code
    assert torch.equal(ref.held(torch.full((1, 64), 3.25).bfloat16()), torch.full((1, 64), 3.25, dtype=torch.float64))
    y = torch.randn(50, 128, generator=torch.Generator().manual_seed(0)).bfloat16()
    n, step, low = ref.quantise(y)
    assert ((ref.held(y) - y.double()).abs() <= 0.53 * step.repeat_interleave(64, -1)).all()
    z, size = ref.norm_rope(torch.tensor([[3.0, 4.0] + [0.0] * 14]), None, ref.table(2, 16)[1:], True)
    c, s = np.cos(1.0), np.sin(1.0)
    assert np.allclose(z[0, :2], [3 * c - 4 * s, 4 * c + 3 * s]) and np.allclose(size[0, :2], [3 * c + 4 * s, 4 * c + 3 * s])
    z, _ = ref.norm_rope(torch.tensor([[3.0] + [0.0] * 7 + [4.0] + [0.0] * 7]), torch.full((16,), 2.0), ref.table(2, 16)[1:], eps=0.0)
    r = 2 / np.sqrt(25 / 16)
    assert np.allclose(z[0, [0, 8]], [r * (3 * c - 4 * s), r * (4 * c + 3 * s)])
    assert ref.to_bf16(torch.tensor([1 + 2.0 ** -8 + 2.0 ** -40], dtype=torch.float64)).item() == 1 + 2.0 ** -7
    assert ref.to_bf16(torch.tensor([1 + 2.0 ** -8], dtype=torch.float64)).item() == 1.0
