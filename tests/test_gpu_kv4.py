"""A paged cache held in 4 bits: what goes in, what comes out, and attention over it (kv4_cache.cu, kv4_attn.cu)."""
import math

import pytest
import torch

import heads_reference as ref
import paper_2608_13426_b200 as rmm
from paper_2608_13426_b200 import binding

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def gen(seed):
    return torch.Generator().manual_seed(seed)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def page_table(lengths, page, spare=2, seed=0):
    need = [max(1, -(-n // page)) for n in lengths]
    order = torch.randperm(sum(need) + spare, generator=gen(seed)).int()
    table = torch.full((len(lengths), max(need)), -7, dtype=torch.int32)   # entries behind a sequence's end are not read
    at = 0
    for b, n in enumerate(need):
        if lengths[b]:
            table[b, :n] = order[at:at + n]
        at += n
    return table, sum(need) + spare


def blocks_of(pool, table, b, n):
    """One sequence's blocks on the CPU: [Hkv, blocks, 18 D]"""
    page = pool.shape[2] * 16
    idx = table[b, :-(-n // page)].long()
    return pool.cpu()[idx].transpose(0, 1).flatten(1, 2)


def filled(lengths, Hkv, D, page, seed=0, k_scale=1.0, garbage=True):
    """A pool that holds random keys and values; unused places hold NaN steps and codes of ones.  (pool, table, held K and V by sequence)"""
    table, pages = page_table(lengths, page, seed=seed)
    pool = torch.full((pages, Hkv, page // 16, 18 * D), 255 if garbage else 0, dtype=torch.uint8, device="cuda")
    B, L = len(lengths), max(1, max(lengths))
    g = gen(seed + 1)
    K = (torch.randn(B, Hkv, L, D, generator=g) * k_scale + torch.randn(1, Hkv, 1, D, generator=g)).to(BF16)
    V = torch.randn(B, Hkv, L, D, generator=g).to(BF16)
    if max(lengths):
        rmm.rmm_kv4_append(K.cuda(), V.cuda(), pool, table.cuda(), ints(lengths), ints(lengths))
    return pool, table, K, V


# ---- append and read


def check_append(lengths, new, Hkv, D, page, L, dtype, norm, rot, interleaved, seed=0, rows_off=0, held=True):
    B = len(lengths)
    table, pages = page_table(lengths, page, seed=seed)
    pool = torch.full((pages, Hkv, page // 16, 18 * D), 0xA5, dtype=torch.uint8, device="cuda")
    before = pool.cpu().clone()
    g = gen(seed + 1)
    K = (torch.randn(B, L, Hkv, D + rows_off, generator=g) * (1 + 3 * torch.randn(D + rows_off, generator=g).abs())).to(dtype)[..., rows_off:]
    V = torch.randn(B, L, Hkv, D + rows_off, generator=g).to(dtype)[..., rows_off:]
    w = 1 + 0.3 * torch.randn(D, generator=g) if norm else None
    t = ref.table(max(lengths) + 1, rot) if rot else None

    def dev(x):
        return torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device="cuda").copy_(x).transpose(1, 2)

    got = rmm.rmm_kv4_append(dev(K), dev(V), pool, table.cuda(), ints(lengths), None if new is None else ints(new), None if w is None else w.cuda(),
                             None if t is None else t.cuda(), interleaved=interleaved, want_values=held)
    assert rmm.rmm_status_read() == 0 and (got is None) == (not held)
    written = torch.zeros(pages * Hkv * page // 16, 16, dtype=torch.bool)
    for b in range(B):
        n = L if new is None else new[b]
        first = lengths[b] - n
        z, _ = ref.norm_rope(K[b, :n].transpose(0, 1), w, t[first:first + n] if rot else None, interleaved)
        z = K[b, :n].transpose(0, 1) if w is None and t is None and dtype == BF16 else ref.to_bf16(z)
        v = V[b, :n].transpose(0, 1).to(BF16)
        if n:
            both = ref.unpack(blocks_of(pool, table, b, lengths[b]))
            for (codes, step, low), x in zip(both, (z, v)):
                wc, ws, wl = ref.quantise(x)
                part = slice(first, first + n)
                assert torch.equal(codes.flatten(1, 2)[:, part], wc)
                assert torch.equal(step.flatten(1, 2)[:, part], ws) and torch.equal(low.flatten(1, 2)[:, part], wl)
        if held:
            for o, x in zip(got, (z, v)):
                assert torch.equal(o[b, :, :n].cpu(), ref.held(x).float().to(BF16)) and torch.count_nonzero(o[b, :, n:]) == 0
        idx = table[b].long()
        for at in range(first, lengths[b]):
            for h in range(Hkv):
                written[(idx[at // page] * Hkv + h) * (page // 16) + at % page // 16, at % 16] = True
    # what was not appended stays as it was
    fresh, old = ref.unpack(pool.cpu().view(-1, 18 * D)), ref.unpack(before.view(-1, 18 * D))
    for x, y in zip(fresh, old):
        for a, b in zip(x, y):
            assert torch.equal(a[~written], b[~written])
    return pool, table


@pytest.mark.parametrize("lengths, new, Hkv, D, page, L, dtype, norm, rot, interleaved", [
    ([1], None, 1, 128, 16, 1, BF16, True, 128, False),                       # one token into an empty cache
    ([17, 33, 64, 1000], [1, 1, 1, 1], 2, 128, 64, 1, BF16, True, 128, False),  # a decode step
    ([40, 7, 100], [40, 0, 13], 3, 64, 16, 40, BF16, False, 64, False),       # ragged chunks, one sequence sits out
    ([300, 129], [250, 129], 2, 256, 32, 250, F32, True, 128, True),          # wide fp32 heads, neighbouring pairs
    ([130], None, 8, 128, 128, 130, F32, True, 128, False),                   # a block, a page and two tokens
    ([77, 78], [30, 31], 1, 128, 16, 31, BF16, False, 0, False),              # neither norm nor rotation
    ([77, 5], [33, 5], 2, 256, 16, 33, BF16, True, 0, False),                 # norm alone
    ([20], None, 40, 64, 16, 20, F32, False, 32, True),                       # many heads, half of the columns turn
    ([2050, 2049], [2050, 2000], 2, 128, 64, 2050, BF16, True, 128, False),   # a prompt
])
def test_the_codes_are_those_of_64_bits(lengths, new, Hkv, D, page, L, dtype, norm, rot, interleaved):
    check_append(lengths, new, Hkv, D, page, L, dtype, norm, rot, interleaved, seed=L)


def test_append_of_unaligned_rows_and_without_values():
    check_append([50, 9], [40, 9], 2, 128, 16, 40, BF16, True, 128, False, rows_off=3)
    check_append([50, 9], [40, 9], 2, 64, 16, 40, F32, True, 64, True, rows_off=1, held=False)


def test_steps_of_groups_that_are_constant_tiny_or_large():
    x = torch.zeros(1, 1, 6, 128)
    x[0, 0, 1] = 2.5                                        # no step: the least value is all
    x[0, 0, 2, :64], x[0, 0, 2, 64:] = -1e30, 1e30
    x[0, 0, 2, 3] = 1e30
    x[0, 0, 3] = torch.linspace(-1e-30, 1e-30, 128)
    x[0, 0, 4, 5] = 1.0                                     # all but one at the least value
    x[0, 0, 5] = torch.arange(128) % 31 / 2                 # halves of a step
    x = x.to(BF16)
    pool = rmm.rmm_kv4_pool(1, 1, 128, 16)
    got = rmm.rmm_kv4_append(x.cuda(), -x.cuda(), pool, ints([[0]]), ints([6]), want_values=True)
    assert torch.equal(got[0].cpu(), ref.held(x).float().to(BF16)) and torch.equal(got[1].cpu(), ref.held(-x).float().to(BF16))
    (ck, sk, _), (cv, sv, _) = ref.unpack(pool.cpu()[0])
    assert torch.equal(ck[0, 0, :6], ref.quantise(x)[0][0, 0]) and torch.equal(cv[0, 0, :6], ref.quantise(-x)[0][0, 0])
    assert rmm.rmm_status_read() == 0


@pytest.mark.parametrize("out", [BF16, F32])
@pytest.mark.parametrize("D, Hkv, page", [(64, 3, 16), (128, 2, 64), (256, 1, 32)])
def test_read_returns_what_is_held(D, Hkv, page, out):
    lengths = [70, 1, 0, 33, 16]
    pool, table, K, V = filled(lengths, Hkv, D, page, seed=D)
    k, v = rmm.rmm_kv4_read(pool, table.cuda(), ints(lengths), ints(lengths), rows=75, out_dtype=out)
    new = [5, 1, 0, 4, 6]
    k2, v2 = rmm.rmm_kv4_read(pool, table.cuda(), ints(lengths), ints(new), rows=6, out_dtype=out)
    for b, n in enumerate(lengths):
        for whole, last, x in ((k, k2, K), (v, v2, V)):
            want = ref.held(x[b, :, :n]).float().to(out)
            assert torch.equal(whole[b, :, :n].cpu(), want) and torch.count_nonzero(whole[b, :, n:]) == 0
            assert torch.equal(last[b, :, :new[b]].cpu(), want[:, n - new[b]:]) and torch.count_nonzero(last[b, :, new[b]:]) == 0
    assert rmm.rmm_status_read() == 0
    k3, _ = rmm.rmm_kv4_read(pool, table.cuda(), ints(lengths), rows=1, out_dtype=out)      # the last token of each; one has none
    assert rmm.rmm_status_read() == binding.RMM_ERR_BOUNDS
    assert torch.equal(k3[[0, 1, 3, 4]], torch.stack([k[b, :, n - 1:n] for b, n in enumerate(lengths) if n])) and torch.count_nonzero(k3[2]) == 0


# ---- attention


def check_attn(lengths, Hq, Hkv, D, page, L, new=None, causal=True, rho_d=1.0, seed=0, q_scale=1.0, k_scale=1.0, **kw):
    pool, table, K, V = filled(lengths, Hkv, D, page, seed, k_scale)
    Q = (torch.randn(len(lengths), L, Hq, D, generator=gen(seed + 5)) * q_scale).to(BF16).transpose(1, 2)
    q = Q.transpose(1, 2).cuda().transpose(1, 2)
    O, idx = rmm.rmm_kv4_attn(q, pool, table.cuda(), ints(lengths), None if new is None else ints(new), causal=causal, rho_d=rho_d, want_idx=True, **kw) \
        if L <= 16 else (rmm.rmm_kv4_attn(q, pool, table.cuda(), ints(lengths), None if new is None else ints(new), causal=causal, rho_d=rho_d, **kw), None)
    assert rmm.rmm_status_read(kw.get("ws")) == 0
    compare(O, idx, Q, K, V, lengths, [L] * len(lengths) if new is None else new, causal, rho_d)
    return O


def compare(O, idx, Q, K, V, lengths, new, causal, rho_d, only=None):
    B, Hq, L, D = Q.shape
    Hkv = K.shape[1]
    kd = rmm.rmm_keep_count(rho_d, D)
    O = O.double().cpu()
    for b, n in enumerate(lengths):
        for kv in range(Hkv):
            k, v = ref.held(K[b, kv, :n]), ref.held(V[b, kv, :n])
            codes, step, low = ref.quantise(V[b, kv, :n]) if n else (torch.zeros(0, D), torch.zeros(0, D // 64), torch.zeros(0, D // 64))
            for h in range(kv * Hq // Hkv, (kv + 1) * Hq // Hkv):
                if only is not None and (b, h) not in only:
                    continue
                want, tol = ref.attention(Q[b, h], k, v, codes.double(), step.double(), low.double(), new[b], causal, kd)
                err = (O[b, h] - want).abs()
                assert (err <= tol).all(), (b, h, (err / tol.clamp(min=1e-30)).max().item(), err.max().item())
                if idx is not None and new[b]:
                    assert torch.equal(idx[b, h].cpu().long(), ref.keep(Q[b, h, :new[b]], kd))


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("lengths, Hq, Hkv, page, L, new, causal, rho_d", [
    ([1], 1, 1, 16, 1, None, True, 1.0),                       # one key, one row
    ([15, 16, 17, 0, 33], 4, 2, 16, 1, None, True, 1.0),       # around a block; a sequence without tokens
    ([63, 64, 65, 128], 8, 1, 64, 1, None, True, 1.0),         # pages that end inside a tile; a full group of rows
    ([700], 12, 2, 32, 1, None, True, 0.5),                    # one job over many CTAs, six rows, half of the features
    ([300, 5, 90], 6, 2, 16, 5, None, True, 0.3),              # drafts; more rows than tokens
    ([300, 5, 90, 7], 4, 1, 16, 7, [7, 2, 0, 7], True, 0.7),   # padded drafts, one sequence without rows
    ([257, 31], 16, 1, 128, 3, None, False, 1.0),              # 48 rows on a kv head, every token seen
    ([120, 400], 2, 2, 16, 16, None, True, 0.5),               # the longest selected step
    ([150, 40], 4, 2, 16, 40, [40, 33], True, 1.0),            # a chunk
    ([4099], 2, 1, 64, 1, None, True, 1.0),                    # one job over all CTAs
])
def test_attention_matches_64_bits(lengths, Hq, Hkv, page, L, new, causal, rho_d, D):
    check_attn(lengths, Hq, Hkv, D, page, L, new, causal, rho_d, seed=D + L)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("lengths, Hq, Hkv, page, L, new, causal, rho_d", [
    ([15, 16, 17, 0, 33], 12, 1, 16, 1, None, True, 1.0),
    ([1], 9, 1, 16, 1, None, True, 1.0),
    ([300, 5, 90], 6, 2, 16, 5, None, True, 0.3),
    ([300, 5, 90, 7], 4, 1, 16, 7, [7, 2, 0, 7], True, 0.7),
    ([257, 31], 16, 1, 128, 3, None, False, 1.0),
    ([120, 400], 2, 2, 16, 16, None, True, 0.5),
    ([150, 40], 4, 2, 16, 40, [40, 33], True, 1.0),
    ([4099, 40], 10, 1, 64, 1, None, True, 0.5),
    ([9000], 16, 1, 64, 1, None, True, 1.0),
])
def test_tables_with_room_for_many_more_tokens(lengths, Hq, Hkv, page, L, new, causal, rho_d, D):
    """The room of a table decides how many rows read the keys at a time; its entries behind a sequence's end are not looked at."""
    pool, table, K, V = filled(lengths, Hkv, D, page, seed=D + L)
    wide = torch.full((len(lengths), (1 << 20) // page), -1, dtype=torch.int32)
    wide[:, :table.shape[1]] = table
    Q = torch.randn(len(lengths), Hq, L, D, generator=gen(7)).to(BF16)
    if new is not None:   # rows that are none may hold anything
        for b, n in enumerate(new):
            Q[b, :, n:] = torch.tensor([float("nan"), float("inf")]).repeat(D // 2).to(BF16)
    got = rmm.rmm_kv4_attn(Q.cuda(), pool, wide.cuda(), ints(lengths), None if new is None else ints(new), causal=causal, rho_d=rho_d)
    narrow = rmm.rmm_kv4_attn(Q.cuda(), pool, table.cuda(), ints(lengths), None if new is None else ints(new), causal=causal, rho_d=rho_d)
    assert rmm.rmm_status_read() == 0
    Q = torch.nan_to_num(Q.float(), 0.0, 0.0, 0.0).to(BF16)
    for O in (got, narrow):
        compare(O, None, Q, K, V, lengths, [L] * len(lengths) if new is None else new, causal, rho_d)


def test_many_short_and_some_long_sequences():
    """More sequences than a CTA has threads, most of them a few tokens long; jobs that lie inside a CTA and jobs that many share."""
    lengths = [(7 * i) % 40 for i in range(600)]
    lengths[5], lengths[300], lengths[599] = 1500, 0, 900
    check_attn(lengths, 2, 1, 64, 16, 1, seed=1)
    lengths = [(11 * i) % 50 for i in range(70)]
    lengths[69] = 3000
    check_attn(lengths, 8, 2, 128, 16, 3, new=[i % 4 for i in range(70)], rho_d=0.5, seed=2)


@pytest.mark.parametrize("pairs", [308, 328, 348, 629, 648, 668, 1250])
def test_one_job_over_many_blocks_of_the_grid(pairs):
    """Jobs cut into 16, 17, 18, 32, 33, 34 and more pieces, whose sums meet in one step or in two."""
    check_attn([pairs * 32 - 5], 3, 1, 64, 64, 1, seed=pairs)


@pytest.mark.parametrize("sequences", [36, 37, 38])
def test_pieces_that_fill_the_grid(sequences):
    """148 jobs of three pieces are as many as the blocks that 148 SMs hold, and no block is left for jobs that are not cut."""
    check_attn([1500] * sequences, 4, 4, 64, 64, 1, seed=3)
    check_attn([1500] * sequences + [3], 4, 4, 64, 64, 1, seed=4)


@pytest.mark.parametrize("L", [1, 16])
@pytest.mark.parametrize("pairs", [47, 96, 97, 224, 225, 240, 241, 247, 576, 577, 583, 1536, 1537, 1543, 2600, 2670, 3100])
def test_one_job_in_pieces_that_meet_once_or_twice(pairs, L):
    """Numbers of pieces around those where the way in which their sums meet changes; groups with one piece more than the others."""
    check_attn([pairs * 32 - 7], 1, 1, 64, 128, L, seed=pairs)


@pytest.mark.parametrize("q_scale, k_scale", [(30.0, 30.0), (1e-6, 1.0), (1e4, 1e-3), (1e-12, 1e12)])
def test_logits_of_any_size(q_scale, k_scale):
    check_attn([200, 77], 4, 2, 128, 16, 2, q_scale=q_scale, k_scale=k_scale, seed=3)


def test_growing_logits_move_the_reference():
    """Keys whose logits rise along the sequence: the reference is refreshed again and again; falling ones never again."""
    n, D = 900, 128
    for sign in (1.0, -1.0):
        K = (torch.randn(1, 1, n, D, generator=gen(1)) * 0.1 + sign * torch.linspace(-30, 30, n)[:, None]).to(BF16)
        V = (torch.randn(1, 1, n, D, generator=gen(2)) * torch.logspace(-6, 4, n)[:, None]).to(BF16)
        Q = torch.ones(1, 3, 1, D).to(BF16) * torch.tensor([1.0, 0.3, -1.0])[None, :, None, None].to(BF16)
        pool, table = rmm.rmm_kv4_pool(60, 1, D, 16), torch.randperm(57, generator=gen(3)).int()[None]
        rmm.rmm_kv4_append(K.cuda(), V.cuda(), pool, table.cuda(), ints([n]))
        O, idx = rmm.rmm_kv4_attn(Q.cuda(), pool, table.cuda(), ints([n]), want_idx=True)
        compare(O, idx, Q, K, V, [n], [1], True, 1.0)


def test_values_of_uneven_steps_and_none():
    """Steps from none (constant groups) over 2^-60 to 2^30 in one row's tokens."""
    n, D = 160, 64
    K = torch.randn(1, 2, n, D, generator=gen(1)).to(BF16)
    V = torch.randn(1, 2, n, D, generator=gen(2))
    V[:, 0] *= torch.tensor([2.0 ** -60, 1.0, 2.0 ** 30, 0.0])[torch.arange(n) % 4][:, None]
    V[:, 1] = 3.0
    V = V.to(BF16)
    Q = torch.randn(1, 4, 1, D, generator=gen(3)).to(BF16)
    pool, table = rmm.rmm_kv4_pool(10, 2, D, 16), torch.arange(10).int()[None]
    rmm.rmm_kv4_append(K.cuda(), V.cuda(), pool, table.cuda(), ints([n]))
    O = rmm.rmm_kv4_attn(Q.cuda(), pool, table.cuda(), ints([n]))
    compare(O, None, Q, K, V, [n], [1], True, 1.0)
    assert torch.equal(O[0, 2:].cpu(), torch.full((2, 1, D), 3.0).to(BF16))
    tiny = (V.float() * 2.0 ** -40).to(BF16)
    rmm.rmm_kv4_append(K.cuda(), tiny.cuda(), pool, table.cuda(), ints([n]))
    compare(rmm.rmm_kv4_attn(Q.cuda(), pool, table.cuda(), ints([n])), None, Q, K, tiny, [n], [1], True, 1.0)


def test_equal_feature_scores_go_to_the_lower_index():
    pool, table, K, V = filled([100], 1, 64, 16, seed=2)
    Q = torch.randn(1, 2, 1, 64, generator=gen(1)).sign().to(BF16)
    O, idx = rmm.rmm_kv4_attn(Q.cuda(), pool, table.cuda(), ints([100]), rho_d=0.5, want_idx=True)
    assert torch.equal(idx.cpu(), torch.arange(32, dtype=torch.int32).expand(1, 2, 32))
    compare(O, idx, Q, K, V, [100], [1], True, 0.5)


def test_pools_and_tables_of_other_strides():
    """A layer of a pool that holds several, a table inside a wider one, Q and its heads in any order."""
    lengths, D = [90, 33], 128
    pool, table, K, V = filled(lengths, 2, D, 32, seed=4)
    Q = torch.randn(2, 4, 3, D, generator=gen(1)).to(BF16)
    want = rmm.rmm_kv4_attn(Q.cuda(), pool, table.cuda(), ints(lengths))
    layers = torch.full((pool.shape[0], 3, 2, 2, 18 * D), 255, dtype=torch.uint8, device="cuda")
    layers[:, 1] = pool
    wide = torch.full((2, table.shape[1] + 5), -1, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = table.cuda()
    view = layers[:, 1]
    got = rmm.rmm_kv4_attn(Q.cuda(), view, wide[:, :table.shape[1]], ints(lengths))
    assert torch.equal(got, want)
    heads_first = pool.transpose(0, 1).contiguous().transpose(0, 1)
    odd = torch.zeros(2, 4, 3, D + 3, dtype=BF16, device="cuda")
    odd[..., 3:] = Q.cuda()
    assert torch.equal(rmm.rmm_kv4_attn(odd[..., 3:], heads_first, wide, ints(lengths)), want)
    k, v = rmm.rmm_kv4_read(view, wide, ints(lengths), ints(lengths), rows=90)
    k0, v0 = rmm.rmm_kv4_read(pool, table.cuda(), ints(lengths), ints(lengths), rows=90)
    assert torch.equal(k, k0) and torch.equal(v, v0)
    rmm.rmm_kv4_append(K.cuda(), V.cuda(), view, wide, ints(lengths), ints(lengths))
    assert (layers[:, [0, 2]] == 255).all() and torch.equal(rmm.rmm_kv4_attn(Q.cuda(), view, wide, ints(lengths)), want)
    shared = torch.stack([table[0], table[0]]).cuda()                          # two sequences on one prefix
    both = rmm.rmm_kv4_attn(Q[:1].expand(2, 4, 3, D).cuda(), pool, shared, ints([90, 90]))
    assert torch.equal(both[0], both[1])
    assert rmm.rmm_status_read() == 0


@pytest.mark.parametrize("page", [16, 64])
def test_a_pool_beyond_32_bits(page):
    """The first and the last pages of a pool of 5 GB: page numbers times bytes pass 2^32."""
    lengths, D, Hkv = [200, 77], 128, 2
    size = Hkv * page // 16 * 18 * D
    pages = 5 * (1 << 30) // size
    need = [-(-n // page) for n in lengths]
    table = torch.full((2, max(need)), -1, dtype=torch.int32)
    table[0, :need[0]] = pages - 1 - torch.arange(need[0])
    table[1, :need[1]] = torch.arange(need[1])
    big = torch.empty(pages, Hkv, page // 16, 18 * D, dtype=torch.uint8, device="cuda")
    big[table[0, :need[0]].long().cuda()] = 255
    big[:need[1]] = 255
    small, order, K, V = filled(lengths, Hkv, D, page, seed=6)
    rmm.rmm_kv4_append(K.cuda(), V.cuda(), big, table.cuda(), ints(lengths), ints(lengths))
    for b, n in enumerate(need):
        assert torch.equal(big[table[b, :n].long().cuda()], small[order[b, :n].long().cuda()])
    Q = torch.randn(2, 4, 2, D, generator=gen(1)).to(BF16).cuda()
    assert torch.equal(rmm.rmm_kv4_attn(Q, big, table.cuda(), ints(lengths)), rmm.rmm_kv4_attn(Q, small, order.cuda(), ints(lengths)))
    for x, y in zip(rmm.rmm_kv4_read(big, table.cuda(), ints(lengths), ints(lengths), rows=200),
                    rmm.rmm_kv4_read(small, order.cuda(), ints(lengths), ints(lengths), rows=200)):
        assert torch.equal(x, y)
    assert rmm.rmm_status_read() == 0


def test_what_lies_outside_is_reported():
    """Pages that are none of the pool's, lengths and rows beyond the table: reported, skipped, nothing else is touched."""
    lengths, D = [40, 40], 64
    pool, table, K, V = filled(lengths, 1, D, 16, seed=6)
    Q = torch.randn(2, 2, 1, D, generator=gen(1)).to(BF16)
    want = rmm.rmm_kv4_attn(Q.cuda(), pool, table.cuda(), ints(lengths))
    for bad in (-1, pool.shape[0], 1 << 30, -(1 << 31)):
        t = table.clone()
        t[1, 1] = bad
        O = rmm.rmm_kv4_attn(Q.cuda(), pool, t.cuda(), ints(lengths))
        assert rmm.rmm_status_read() == binding.RMM_ERR_BOUNDS and torch.equal(O[0], want[0])
        keep = [i for i in range(40) if not 16 <= i < 32]                       # the tokens of the other pages
        assert torch.isfinite(O[1].float()).all()
        compare(O[1:], None, Q[1:], K[1:, :, keep], V[1:, :, keep], [len(keep)], [1], True, 1.0)
        k, _ = rmm.rmm_kv4_read(pool, t.cuda(), ints(lengths), ints(lengths), rows=40)
        assert rmm.rmm_status_read() == binding.RMM_ERR_BOUNDS and torch.count_nonzero(k[1, :, 16:32]) == 0 and torch.count_nonzero(k[1, :, 32:]) > 0
        other = pool.clone()
        rmm.rmm_kv4_append(K.cuda(), V.cuda(), other, t.cuda(), ints(lengths), ints(lengths))
        assert rmm.rmm_status_read() == binding.RMM_ERR_BOUNDS and torch.equal(other, pool)
    for n in ([1000, 40], [-5, 40], [1 << 30, 40]):
        O = rmm.rmm_kv4_attn(Q.cuda(), pool, table.cuda(), ints(n))
        assert rmm.rmm_status_read() == binding.RMM_ERR_BOUNDS and torch.equal(O[1], want[1])
    for rows in ([5, 1], [-1, 1]):
        O = rmm.rmm_kv4_attn(Q.cuda(), pool, table.cuda(), ints(lengths), ints(rows))
        assert rmm.rmm_status_read() == binding.RMM_ERR_BOUNDS and torch.equal(O[1], want[1])
    before = pool.clone()
    x = torch.randn(2, 1, 4, D, dtype=BF16, device="cuda")
    rmm.rmm_kv4_append(x, x, pool, table.cuda(), ints([2, 40]), ints([4, 0]))    # more rows than tokens: two have no place
    assert rmm.rmm_status_read() == binding.RMM_ERR_BOUNDS
    k, _ = rmm.rmm_kv4_read(pool, table.cuda(), ints([2, 40]), ints([2, 40]), rows=40)
    assert torch.equal(k[0, :, :2].cpu(), ref.held(x[0, :, 2:].cpu()).float().to(BF16))
    pool.copy_(before)
    rmm.rmm_kv4_append(x, x, pool, table.cuda(), ints([40, 40]), ints([4, 4]), rope=ref.table(38, D).cuda())
    assert rmm.rmm_status_read() == binding.RMM_ERR_BOUNDS                       # positions 38, 39 are outside the table
    changed = (pool != before).flatten(1).any(1).nonzero().flatten().tolist()
    assert sorted(changed) == sorted({int(table[b, 2]) for b in range(2)})
    assert rmm.rmm_status_read() == 0


def test_the_same_call_twice_gives_the_same_bits_and_leaves_its_workspace_ready():
    lengths = [1000, 333, 20]
    pool, table, K, V = filled(lengths, 2, 128, 64, seed=8)
    Q = torch.randn(3, 8, 1, 128, generator=gen(1)).to(BF16).cuda()
    ws = torch.zeros(16 << 20, dtype=torch.uint8, device="cuda")
    want = rmm.rmm_kv4_attn(Q, pool, table.cuda(), ints(lengths), ws=ws)
    for _ in range(20):
        assert torch.equal(rmm.rmm_kv4_attn(Q, pool, table.cuda(), ints(lengths), ws=ws), want)
    a = (-ws.data_ptr()) % 256
    assert torch.count_nonzero(ws[a:a + 4096]) == 0
    # other operators of the library on the same workspace, before and after
    A = torch.randn(1, 4096, dtype=BF16, device="cuda")
    W = torch.randn(4096, 4096, dtype=BF16, device="cuda")
    y, _ = rmm.rmm_product(A, W, 0.5, ws=ws)
    assert torch.equal(rmm.rmm_kv4_attn(Q, pool, table.cuda(), ints(lengths), ws=ws), want)
    assert torch.equal(rmm.rmm_product(A, W, 0.5, ws=ws)[0], y)


def test_calls_on_two_streams_with_workspaces_of_their_own():
    lengths = [3000, 2000]
    pool, table, K, V = filled(lengths, 2, 128, 64, seed=9)
    Qs = [torch.randn(2, 8, 1, 128, generator=gen(i)).to(BF16).cuda() for i in range(2)]
    wss = [torch.zeros(8 << 20, dtype=torch.uint8, device="cuda") for _ in range(2)]
    t, n = table.cuda(), ints(lengths)
    want = [rmm.rmm_kv4_attn(q, pool, t, n) for q in Qs]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(30):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(rmm.rmm_kv4_attn(Qs[i], pool, t, n, ws=wss[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o, want[i]) for o in got[i])


# ---- as they are used


class Decoder:
    """One layer's heads: norm and rotation, cache, attention."""

    def __init__(self, B, Hq, Hkv, D, most, page=16, seed=0):
        g = gen(seed)
        self.qw, self.kw = (1 + 0.2 * torch.randn(D, generator=g)).cuda(), (1 + 0.2 * torch.randn(D, generator=g)).cuda()
        self.rope = rmm.rmm_rope_table(most, D, device="cuda")
        need = -(-most // page)
        self.pages = torch.randperm(B * need, generator=g).int().view(B, need).cuda()
        self.pool = rmm.rmm_kv4_pool(B * need, Hkv, D, page)
        self.ws = torch.zeros(8 << 20, dtype=torch.uint8, device="cuda")

    def step(self, q, k, v, lengths, new=None, rho_d=1.0):
        rows = torch.arange(q.shape[2], device="cuda", dtype=torch.int32)
        at = ((lengths - (q.shape[2] if new is None else new))[:, None] + rows).int()
        q = rmm.rmm_qk_norm_rope(q, None, self.qw, None, self.rope, at.clamp(0, self.rope.shape[0] - 1), ws=self.ws)
        rmm.rmm_kv4_append(k, v, self.pool, self.pages, lengths, new, self.kw, self.rope, ws=self.ws)
        return rmm.rmm_kv4_attn(q, self.pool, self.pages, lengths, new, rho_d=rho_d, ws=self.ws)


@pytest.mark.parametrize("rho_d", [1.0, 0.5])
def test_prompt_and_decode_steps_agree_with_attention_over_the_values_held(rho_d):
    B, Hq, Hkv, D, prompt, steps = 2, 8, 2, 128, 70, 5
    most = prompt + steps
    dec = Decoder(B, Hq, Hkv, D, most)
    x = [torch.randn(B, most, h, D, generator=gen(7 + h)).to(BF16).cuda().transpose(1, 2) for h in (Hq, Hkv, Hkv + 1)]
    q, k, v = x[0], x[1], x[2][:, :Hkv]
    # the prompt's own attention runs on the values that the cache holds
    kh, vh = rmm.rmm_kv4_append(k[:, :, :prompt], v[:, :, :prompt], dec.pool, dec.pages, ints([prompt] * B), None, dec.kw, dec.rope, want_values=True)
    qr = rmm.rmm_qk_norm_rope(q[:, :, :prompt], None, dec.qw, None, dec.rope)
    O = rmm.rmm_reduced_attn(qr, kh, vh, True, rho_d)
    n = torch.full((B,), prompt, dtype=torch.int32, device="cuda")
    last = rmm.rmm_kv4_attn(qr[:, :, -16:], dec.pool, dec.pages, n) if rho_d == 1.0 else None
    if last is not None:                                     # the last rows of the prompt, asked of the cache
        assert ((last.float() - O[:, :, -16:].float()).norm() / O[:, :, -16:].float().norm()).item() <= 1e-2
    for t in range(prompt, most):
        n = n + 1
        got = dec.step(q[:, :, t:t + 1], k[:, :, t:t + 1], v[:, :, t:t + 1], n, rho_d=rho_d)
        kc, vc = rmm.rmm_kv4_read(dec.pool, dec.pages, n, n, rows=t + 1)
        qr = rmm.rmm_qk_norm_rope(q[:, :, t:t + 1], None, dec.qw, None, dec.rope, torch.full((B, 1), t, dtype=torch.int32, device="cuda"))
        want = rmm.rmm_reduced_attn(qr, kc, vc, True, rho_d)
        assert ((got.float() - want.float()).norm() / want.float().norm()).item() <= 1e-2
    assert rmm.rmm_status_read() == 0 and rmm.rmm_status_read(dec.ws) == 0


def test_captured_steps_follow_lengths_on_the_device():
    B, Hq, Hkv, D = 3, 8, 2, 64
    dec, ref_dec = Decoder(B, Hq, Hkv, D, 200, seed=3), Decoder(B, Hq, Hkv, D, 200, seed=3)
    q, k, v = (torch.zeros(B, h, 1, D, dtype=BF16, device="cuda") for h in (Hq, Hkv, Hkv))
    n = ints([1, 60, 150])
    start = n.clone()
    binding.poison_outputs(False)
    try:
        dec.step(q, k, v, n)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            n.add_(1)
            out = dec.step(q, k, v, n)
        for dst, src in ((dec, ref_dec), (ref_dec, dec)):
            dst.pool.zero_()
        n.copy_(start)
        m = start.clone()
        for t in range(40):
            for x in (q, k, v):
                x.copy_(torch.randn(x.shape, generator=gen(100 + t)).to(BF16))
            graph.replay()
            m = m + 1
            want = ref_dec.step(q, k, v, m)
            assert torch.equal(out, want) and torch.equal(dec.pool, ref_dec.pool)
    finally:
        binding.poison_outputs(True)
    assert rmm.rmm_status_read(dec.ws) == 0


def test_appending_rotated_keys_is_appending_keys_with_the_rotation():
    k = torch.randn(2, 4, 50, 128, generator=gen(1)).to(BF16).cuda()
    a, b = Decoder(2, 4, 4, 128, 64), Decoder(2, 4, 4, 128, 64)
    n = ints([50, 50])
    rmm.rmm_kv4_append(k, k, a.pool, a.pages, n, None, a.kw, a.rope)
    # fp32 rows round to bf16 inside; rows given in bf16 were rounded from fp32 and may differ by their last bit where it is a close call
    rmm.rmm_kv4_append(rmm.rmm_qk_norm_rope(k, None, a.kw, None, a.rope, out_dtype=F32), k.float(), b.pool, b.pages, n)
    assert (a.pool != b.pool).float().mean().item() < 1e-3


def test_a_wait_that_runs_out_is_reported():
    pool, table, K, V = filled([500, 300], 2, 128, 16, seed=1)
    Q = torch.randn(2, 8, 1, 128, generator=gen(1)).to(BF16).cuda()
    want = rmm.rmm_kv4_attn(Q, pool, table.cuda(), ints([500, 300]))
    torch.cuda.synchronize()
    rmm.rmm_debug_control("wait_limit_ms", 20.0)
    rmm.rmm_debug_control("withhold", 7)
    try:
        rmm.rmm_kv4_attn(Q, pool, table.cuda(), ints([500, 300]))
        assert rmm.rmm_status_read() == binding.RMM_ERR_TIMEOUT
    finally:
        rmm.rmm_debug_control("withhold", 0)
        rmm.rmm_debug_control("wait_limit_ms", 0)
    assert torch.equal(rmm.rmm_kv4_attn(Q, pool, table.cuda(), ints([500, 300])), want)
    assert rmm.rmm_status_read() == 0


def test_refusals():
    pool, table, K, V = filled([20], 2, 64, 16)
    q, k = torch.zeros(1, 4, 1, 64, dtype=BF16, device="cuda"), torch.zeros(1, 2, 1, 64, dtype=BF16, device="cuda")
    t, n = table.cuda(), ints([20])
    bad, odd = binding.RMM_ERR_INVALID_ARG, binding.RMM_ERR_UNSUPPORTED
    for f, code in [(lambda: rmm.rmm_kv4_attn(q.float(), pool, t, n), odd), (lambda: rmm.rmm_kv4_attn(q[:, :3], pool, t, n), bad),
                    (lambda: rmm.rmm_kv4_attn(q.expand(1, 4, 17, 64), pool, t, n, rho_d=0.5), odd), (lambda: rmm.rmm_kv4_attn(q, pool, t, n, rho_d=0.0), bad),
                    (lambda: rmm.rmm_kv4_attn(q, pool, t, n.long()), bad), (lambda: rmm.rmm_kv4_attn(q, pool, t[0], n), bad),
                    (lambda: rmm.rmm_kv4_attn(q, pool, t, ints([20, 20])), bad), (lambda: rmm.rmm_kv4_attn(q, pool, t.cpu(), n), bad),
                    (lambda: rmm.rmm_kv4_attn(q, pool[..., :-1], t, n), bad), (lambda: rmm.rmm_kv4_attn(q, pool.float(), t, n), bad),
                    (lambda: rmm.rmm_kv4_attn(q, pool, t, n, ints([1, 1])), bad), (lambda: rmm.rmm_kv4_attn(q[..., :32], pool, t, n), bad),
                    (lambda: rmm.rmm_kv4_append(k, k.float(), pool, t, n), odd), (lambda: rmm.rmm_kv4_append(k, k[..., :32], pool, t, n), bad),
                    (lambda: rmm.rmm_kv4_append(q, q, pool, t, n), bad), (lambda: rmm.rmm_kv4_append(k, k, pool, t, n, k_weight=torch.ones(32, device="cuda")), bad),
                    (lambda: rmm.rmm_kv4_read(pool, t, n, rows=0), bad), (lambda: rmm.rmm_kv4_read(pool, t, n, out_dtype=torch.float16), odd),
                    (lambda: rmm.rmm_kv4_attn(q, pool, t, n, ws=torch.zeros(8192, dtype=torch.uint8, device="cuda")), binding.RMM_ERR_WORKSPACE)]:
        with pytest.raises(binding.RmmError) as e:
            f()
        assert e.value.code == code, str(e.value)
    assert rmm.rmm_status_read() == 0
