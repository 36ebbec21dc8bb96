"""The native marshalling of the calls on rows of heads and the 4-bit cache: as by Python, and what it leaves to Python."""
import pytest
import torch

import paper_2608_13426_b200 as rmm
from paper_2608_13426_b200 import binding

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.fixture(scope="module")
def native():
    n = binding._native()
    assert n is not None
    return n


@pytest.fixture(scope="module")
def ws():
    return torch.zeros(32 << 20, dtype=torch.uint8, device="cuda")     # a call that is given one goes through Python


@pytest.fixture
def state():
    g = torch.Generator(device="cuda").manual_seed(1)
    B, Hq, Hkv, L, D = 2, 8, 2, 3, 64
    both = torch.randn(B, L, Hq + 2 * Hkv, D, generator=g, device="cuda").to(BF16).transpose(1, 2)
    return dict(Q=both[:, :Hq], K=both[:, Hq:Hq + Hkv], V=both[:, Hq + Hkv:], w=torch.rand(D, device="cuda"), rope=rmm.rmm_rope_table(300, D, device="cuda"),
                pos=ints([[5, 6, 7], [200, 201, 202]]), pool=rmm.rmm_kv4_pool(40, Hkv, D, 16), pages=torch.randperm(40, device="cuda").int().view(2, 20),
                n=ints([8, 203]), new=ints([3, 2]))


@pytest.mark.parametrize("interleaved", [False, True])
def test_norm_rope(native, ws, state, interleaved):
    s = state
    for Q, K, qw, kw, rope, pos in [(s["Q"], s["K"], s["w"], s["w"], s["rope"], s["pos"]), (s["Q"], None, s["w"].bfloat16(), None, s["rope"], s["pos"][0]),
                                    (s["Q"].float(), s["K"].float(), None, s["w"], s["rope"][:, :32], None), (s["Q"], s["K"], None, None, None, None),
                                    (torch.nn.Parameter(s["Q"]), s["K"], torch.nn.Parameter(s["w"]), s["w"], s["rope"], s["pos"][:1])]:
        got = native.norm_rope(Q, K, qw, kw, rope, pos, 1e-6, interleaved)
        want = rmm.rmm_qk_norm_rope(Q, K, qw, kw, rope, pos, interleaved=interleaved, ws=ws)
        for a, b in zip(got if K is not None else (got,), want if K is not None else (want,)):
            assert torch.equal(a, b) and a.is_contiguous() and not a.requires_grad
        pub = rmm.rmm_qk_norm_rope(Q, K, qw, kw, rope, pos, interleaved=interleaved)
        assert torch.equal(pub[0] if K is not None else pub, want[0] if K is not None else want)
    assert rmm.rmm_status_read() == 0


def test_cache(native, ws, state):
    s = state
    other = s["pool"].clone()
    for new in (None, s["new"]):
        for held in (True, False):
            got = native.kv4_append(s["K"], s["V"], s["pool"], s["pages"], s["n"], new, s["w"], s["rope"], 1e-6, False, held)
            want = rmm.rmm_kv4_append(s["K"], s["V"], other, s["pages"], s["n"], new, s["w"], s["rope"], want_values=held, ws=ws)
            assert torch.equal(s["pool"], other)
            if held:
                assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
            else:
                assert got is False and want is None
                assert rmm.rmm_kv4_append(s["K"], s["V"], s["pool"], s["pages"], s["n"], new, s["w"], s["rope"]) is None
        for dt in (BF16, F32):
            got, want = native.kv4_read(s["pool"], s["pages"], s["n"], new, 3, dt), rmm.rmm_kv4_read(s["pool"], s["pages"], s["n"], new, 3, dt, ws=ws)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and got[0].dtype == dt
        for causal, rho_d in ((True, 1.0), (False, 0.5), (True, 1)):
            got = native.kv4_attn(s["Q"], s["pool"], s["pages"], s["n"], new, causal, rho_d)
            assert torch.equal(got, rmm.rmm_kv4_attn(s["Q"], s["pool"], s["pages"], s["n"], new, causal, rho_d, ws=ws))
            assert torch.equal(got, rmm.rmm_kv4_attn(s["Q"], s["pool"], s["pages"], s["n"], new, causal, rho_d))
    assert rmm.rmm_status_read() == 0


def test_what_is_not_plain_is_left_to_python_and_refused_the_same_way(native, ws, state):
    s = state
    Q, K, V, pool, pages, n = (s[x] for x in ("Q", "K", "V", "pool", "pages", "n"))
    for args in [(Q.half(), None, None, None, None, None), (Q, K.float(), None, None, None, None), (Q[0], None, None, None, None, None),
                 (Q, None, s["w"].double(), None, None, None), (Q, None, s["w"][:5], None, None, None), (Q, K, s["w"], s["w"].bfloat16(), None, None),
                 (Q, None, None, None, s["rope"].double(), None), (Q, None, None, None, s["rope"], s["pos"].long()), (Q, None, None, None, s["rope"], s["pos"][:, :2]),
                 (Q.cpu(), None, None, None, None, None), ("Q", None, None, None, None, None)]:
        assert native.norm_rope(*args, 1e-6, False) is None
        with pytest.raises((binding.RmmError, AttributeError)):
            rmm.rmm_qk_norm_rope(*args)
    for args in [(Q, pool.int(), pages, n, None), (Q, pool, pages.long(), n, None), (Q, pool, pages, n[:1], None), (Q, pool, pages, n, s["new"].long()),
                 (Q, pool[..., 1:], pages, n, None), (Q, pool.cpu(), pages, n, None), (Q[..., :32], pool, pages, n, None), (Q.float(), pool, pages, n, None)]:
        assert native.kv4_attn(*args, True, 1.0) is None
        with pytest.raises(binding.RmmError):
            rmm.rmm_kv4_attn(*args)
    assert native.kv4_attn(Q, pool, pages, n, None, 1, 1.0) is None and native.kv4_read(pool, pages, n, None, 1, torch.float16) is None
    assert native.kv4_read(pool, pages, n, None, 0, BF16) is None and native.norm_rope() is None and native.kv4_append(1) is None
    assert torch.equal(rmm.rmm_kv4_attn(Q, pool, pages, n, None, 1, 1.0), rmm.rmm_kv4_attn(Q, pool, pages, n, None, True, 1.0))
    got = []
    for more in ({}, {"ws": ws}):                              # refused by the library itself: one message
        with pytest.raises(binding.RmmError) as e:
            rmm.rmm_kv4_attn(Q, pool, pages, n, None, True, 1.5, **more)
        got.append((e.value.code, str(e.value)))
        with pytest.raises(binding.RmmError) as e:
            rmm.rmm_qk_norm_rope(Q, None, None, None, s["rope"][:, :40], **more)
        got.append((e.value.code, str(e.value)))
        with pytest.raises(binding.RmmError) as e:
            rmm.rmm_kv4_append(Q, Q, pool, pages, n, **more)
        got.append((e.value.code, str(e.value)))
    assert got[:3] == got[3:]
