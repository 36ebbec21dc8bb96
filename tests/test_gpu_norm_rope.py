"""Norm and rotation of query and key heads in one pass (norm_rope.cu)."""
import pytest
import torch

import heads_reference as ref
import paper_2608_13426_b200 as rmm
from paper_2608_13426_b200 import binding

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def inputs(B, Hq, Hkv, L, D, dtype, seed=0, layout="blhd"):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(B, L, Hq + Hkv, D, generator=g) * (1 + 3 * torch.randn(D, generator=g).abs())
    x = x.to(dtype)
    q, k = x[:, :, :Hq].transpose(1, 2), x[:, :, Hq:].transpose(1, 2)
    if layout == "bhld":
        q, k = q.contiguous(), k.contiguous()
    return q, k, 1 + 0.3 * torch.randn(D, generator=g), 1 + 0.3 * torch.randn(D, generator=g)


def on_gpu(x):
    """Same strides on the GPU."""
    base = torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device="cuda")
    return base.copy_(x)


def check(got, x, w, rows, interleaved, eps=1e-6):
    want, size = ref.norm_rope(x, w, rows, interleaved, eps)
    got = got.cpu()
    # the fp32 chain (heads.cuh), and the rounding to the output's type
    tol = 2.0 ** -20 * size * 1.01 + (2.0 ** -8 if got.dtype == BF16 else 2.0 ** -24) * want.abs()
    assert ((got.double() - want).abs() <= tol).all(), ((got.double() - want).abs() / tol.clamp(min=1e-300)).max()


@pytest.mark.parametrize("out", [None, BF16, F32])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B, Hq, Hkv, L, D, rot, interleaved, layout", [
    (1, 1, 1, 1, 128, 128, False, "blhd"),       # one row
    (2, 32, 8, 5, 128, 128, False, "blhd"),
    (3, 7, 3, 33, 80, 80, False, "bhld"),        # 10 of 16 lanes, heads that end inside a warp's turn
    (2, 5, 1, 17, 96, 32, True, "blhd"),         # a third of the columns, neighbouring pairs
    (1, 9, 2, 40, 256, 128, False, "blhd"),      # a row is a warp
    (2, 3, 3, 9, 64, 64, True, "bhld"),
    (1, 40, 8, 3, 8, 0, False, "blhd"),          # the smallest head
    (2, 4, 2, 6, 16, 16, False, "bhld"),
    (1, 2, 1, 70, 248, 240, False, "blhd"),      # half of 240 columns lies off the eights' pairs
])
def test_rows_match_64_bits(B, Hq, Hkv, L, D, rot, interleaved, layout, dtype, out):
    q, k, qw, kw = inputs(B, Hq, Hkv, L, D, dtype, seed=D + L, layout=layout)
    t = ref.table(200, rot) if rot else None
    pos = torch.randint(0, 200, (B, L), generator=torch.Generator().manual_seed(1)).int()
    Q, K = rmm.rmm_qk_norm_rope(on_gpu(q), on_gpu(k), qw.cuda(), kw.cuda(), None if t is None else t.cuda(), pos.cuda(), interleaved=interleaved, out_dtype=out)
    assert Q.dtype == K.dtype == (out or dtype)
    rows = None if t is None else t[pos.long()][:, None]
    check(Q, q, qw, rows, interleaved)
    check(K, k, kw, rows, interleaved)
    assert rmm.rmm_status_read() == 0


def test_parts_may_be_missing():
    q, k, qw, kw = inputs(2, 6, 2, 11, 128, BF16)
    t = ref.table(64, 128)
    rows = t[:11]
    Q = rmm.rmm_qk_norm_rope(on_gpu(q), None, qw.bfloat16().cuda(), None, t.cuda())        # queries only, positions 0 .. L - 1, bf16 weights
    check(Q, q, qw.bfloat16(), rows, False)
    Q, K = rmm.rmm_qk_norm_rope(on_gpu(q), on_gpu(k), None, kw.cuda(), t.cuda(), torch.arange(20, 31, dtype=torch.int32).cuda())
    check(Q, q, None, t[20:31], False)
    check(K, k, kw, t[20:31], False)
    Q, K = rmm.rmm_qk_norm_rope(on_gpu(q), on_gpu(k))                                        # neither: a copy
    assert torch.equal(Q.cpu(), q) and torch.equal(K.cpu(), k)
    Q = rmm.rmm_qk_norm_rope(on_gpu(q), q_weight=qw.cuda(), eps=0.5)
    check(Q, q, qw, None, False, eps=0.5)
    zero = torch.zeros(1, 2, 3, 64, dtype=BF16, device="cuda")
    assert torch.count_nonzero(rmm.rmm_qk_norm_rope(zero, q_weight=torch.ones(64, device="cuda"))) == 0
    assert rmm.rmm_status_read() == 0


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_in_place_and_odd_strides(dtype):
    q, k, qw, kw = inputs(2, 6, 2, 13, 64, dtype, seed=4)
    t = ref.table(40, 64)
    Q, K = rmm.rmm_qk_norm_rope(on_gpu(q), on_gpu(k), qw.cuda(), kw.cuda(), t.cuda())
    a, b = on_gpu(q), on_gpu(k)
    A, B = rmm.rmm_qk_norm_rope(a, b, qw.cuda(), kw.cuda(), t.cuda(), inplace=True)
    assert A is a and B is b and torch.equal(A, Q) and torch.equal(B, K)
    wide = torch.full((2, 13, 6, 67), 7.0, dtype=dtype, device="cuda")                       # rows off 16 bytes
    wide[..., 1:65] = q.transpose(1, 2).cuda()
    v = wide[..., 1:65].transpose(1, 2)
    assert torch.equal(rmm.rmm_qk_norm_rope(v, None, qw.cuda(), None, t.cuda()), Q)
    rmm.rmm_qk_norm_rope(v, None, qw.cuda(), None, t.cuda(), inplace=True)
    assert torch.equal(v, Q) and (wide[..., 0] == 7).all() and (wide[..., 65:] == 7).all()
    strided = torch.zeros(40, 80, device="cuda")[:, :64]                                      # a table inside a wider one
    strided.copy_(t)
    assert torch.equal(rmm.rmm_qk_norm_rope(on_gpu(q), None, qw.cuda(), None, strided), Q)
    one = on_gpu(q)[:, :1].expand(2, 6, 13, 64)                                               # a head shared by all
    got = rmm.rmm_qk_norm_rope(one, None, qw.cuda(), None, t.cuda())
    assert torch.equal(got, Q[:, :1].expand(2, 6, 13, 64))


def test_positions_outside_the_table_are_reported_and_skipped():
    q, _, qw, _ = inputs(1, 4, 1, 6, 64, BF16)
    t = ref.table(10, 64).cuda()
    a = on_gpu(q)
    pos = torch.tensor([[0, 9, 10, -1, 3, 1 << 30]], dtype=torch.int32).cuda()
    rmm.rmm_qk_norm_rope(a, None, qw.cuda(), None, t, pos, inplace=True)
    assert rmm.rmm_status_read() == binding.RMM_ERR_BOUNDS
    assert torch.equal(a[:, :, [2, 3, 5]].cpu(), q[:, :, [2, 3, 5]])
    check(a[:, :, [0, 1, 4]], q[:, :, [0, 1, 4]], qw, t.cpu()[[0, 9, 3]], False)
    assert rmm.rmm_status_read() == 0


def test_another_stream_and_a_captured_call():
    q, k, qw, kw = inputs(2, 8, 2, 3, 128, BF16)
    t, qd, kd, w1, w2 = ref.table(100, 128).cuda(), on_gpu(q), on_gpu(k), qw.cuda(), kw.cuda()
    pos = torch.full((2, 3), 5, dtype=torch.int32, device="cuda")
    want = rmm.rmm_qk_norm_rope(qd, kd, w1, w2, t, pos)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = rmm.rmm_qk_norm_rope(qd, kd, w1, w2, t, pos)
    s.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    ws = torch.zeros(8192, dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    binding.poison_outputs(False)
    try:
        with torch.cuda.graph(graph):
            out = rmm.rmm_qk_norm_rope(qd, kd, w1, w2, t, pos, ws=ws)
    finally:
        binding.poison_outputs(True)
    for p in (5, 60):
        pos.fill_(p)
        graph.replay()
        want = rmm.rmm_qk_norm_rope(qd, kd, w1, w2, t, pos)
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


def test_offsets_beyond_32_bits():
    """Sequences, heads and rows that lie more than 2^32 bytes apart."""
    far = (1 << 31) + 128
    memory = torch.empty(far + 4096, dtype=BF16, device="cuda")
    x = torch.randn(2, 2, 2, 64, generator=torch.Generator().manual_seed(3)).to(BF16)
    t = ref.table(2, 64).cuda()
    want = rmm.rmm_qk_norm_rope(x.cuda(), rope=t)
    for stride in ((far, 128, 64), (128, far, 64), (128, 64, far)):
        q = memory.as_strided((2, 2, 2, 64), stride + (1,))
        q.copy_(x)
        assert torch.equal(rmm.rmm_qk_norm_rope(q, rope=t), want)
        rmm.rmm_qk_norm_rope(q, rope=t, inplace=True)
        assert torch.equal(q, want)
    assert rmm.rmm_status_read() == 0


def test_written_memory_that_overlaps_is_refused():
    x = torch.zeros(1, 2, 3, 64, dtype=BF16, device="cuda")
    for call in (lambda: rmm.rmm_qk_norm_rope(x[:, :1].expand(1, 2, 3, 64), inplace=True), lambda: rmm.rmm_qk_norm_rope(x, x, inplace=True)):
        with pytest.raises(binding.RmmError) as e:
            call()
        assert e.value.code == binding.RMM_ERR_INVALID_ARG
    rmm.rmm_qk_norm_rope(x[:, :1].expand(1, 2, 3, 64))   # read only
    assert rmm.rmm_status_read() == 0


def test_refusals():
    q = torch.zeros(1, 2, 3, 64, dtype=BF16, device="cuda")
    w, t = torch.ones(64, device="cuda"), ref.table(8, 64).cuda()
    bad, odd = binding.RMM_ERR_INVALID_ARG, binding.RMM_ERR_UNSUPPORTED
    for args, kw, code in [((q[0],), {}, bad), ((q.cpu(),), {}, bad), ((q.half(),), {}, odd), ((q.transpose(2, 3),), {}, odd),
                           ((q[..., :60],), {}, odd), ((q, q[..., :32]), {}, bad), ((q, q.float()), {}, odd), ((q, None, w[:32]), {}, bad),
                           ((q, q, w, w.bfloat16()), {}, odd), ((q, None, w.cpu()), {}, bad), ((q, None, w, None, t[:, :40]), {}, odd),
                           ((q, None, w, None, t.double()), {}, bad), ((q, None, w, None, torch.ones(4, 80, device="cuda")), {}, bad),
                           ((q, None, w, None, t, torch.zeros(1, 3, dtype=torch.int64, device="cuda")), {}, bad),
                           ((q, None, w, None, t, torch.zeros(1, 4, dtype=torch.int32, device="cuda")), {}, bad),
                           ((q, None, w), {"eps": -1.0}, bad), ((q, None, w), {"eps": float("nan")}, bad),
                           ((q,), {"inplace": True, "out_dtype": F32}, bad), ((q,), {"out_dtype": torch.float16}, odd),
                           ((torch.zeros(1, 1, 1, 264, dtype=BF16, device="cuda"),), {}, odd),
                           ((q,), {"ws": torch.zeros(64, dtype=torch.uint8, device="cuda")}, binding.RMM_ERR_WORKSPACE)]:
        with pytest.raises(binding.RmmError) as e:
            rmm.rmm_qk_norm_rope(*args, **kw)
        assert e.value.code == code, (args[0].shape, kw, str(e.value))
