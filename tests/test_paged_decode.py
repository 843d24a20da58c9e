"""One decode step of many sequences over their pages, against softmax attention in 64 bits; refusals."""
import math

import numpy as np
import pytest
import torch

import paper_2604_16734_amd as K
from tests.test_pages import BAD_PAGES, DEV, P16, P4, Pool, _pages, gpu, int32


def reference(q, pool, table, lengths, n_pages, page, scale):
    """(out, size): softmax attention in 64 bits, and the same with the values' magnitudes: what errors of the weights are relative to.
    Also the largest sum of magnitudes of a logit's products, times the scale."""
    n_seqs, hq, d = q.shape
    hkv = pool.k.shape[1]
    out, size, most = np.zeros(q.shape), np.zeros(q.shape), 0.0
    for s in range(n_seqs):
        keys = []
        for p in range(max(0, min(lengths[s], table.shape[1] * page))):
            number = int(table[s, p // page])
            if 0 <= number < n_pages:
                keys.append((number, p % page))
        if not keys:
            continue
        pages, at = np.array(keys).T
        for h in range(hkv):
            k, v = (getattr(pool, n)[pages, h, at] for n in "kv")
            if pool.e4m3:
                k, v = (x * np.exp2(getattr(pool, n + "_exp")[pages, h, at] - 127.0)[:, None] for x, n in ((k, "k"), (v, "v")))
            of = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
            logits = q[s, of] @ k.T * scale
            most = max(most, float((np.abs(q[s, of]) @ np.abs(k).T).max()) * scale)
            w = np.exp(logits - logits.max(axis=1, keepdims=True))
            w /= w.sum(axis=1, keepdims=True)
            out[s, of], size[s, of] = w @ v, w @ np.abs(v)
    return out, size, most


def check(out, ref, size, most, d):
    """Half a bf16 step for every weight and for the result; a logit is off by d fp32 roundings of its products at most and the weight
    by as much relatively, once in the sum and once in the product; and a dozen fp32 roundings of the rest."""
    half, fp32 = 2.0 ** -8, 2.0 ** -24
    tol = size * (half + 2 * d * most * fp32 + 64 * fp32) + np.abs(ref) * half + 1e-30
    got = out.double().cpu().numpy()
    assert np.isfinite(got).all()
    worst = np.max(np.abs(got - ref) / tol)
    assert worst <= 1.0, worst


def a_batch(gen, lengths, hkv, d, page, e4m3, spare=3):
    """Pages of these sequences in random order with numbers in their rows, and NaNs in all others."""
    counts = [max(1, -(-n // page)) for n in lengths]
    width, n_pages = max(counts), sum(counts) + spare
    order = torch.randperm(n_pages, generator=gen)
    table = torch.full((len(lengths), width), -1, dtype=torch.int32)
    pages = K.Pages.empty(n_pages, hkv, d, page, e4m3, DEV)
    for t in (pages.k, pages.v):
        t.view(torch.uint8).fill_(0xFF)                     # NaN in either format
    if e4m3:
        pages.k_exp.fill_(255), pages.v_exp.fill_(255)
    i = 0
    for s, c in enumerate(counts):
        table[s, :c] = order[i:i + c].int()
        i += c
    table = table.to(DEV)
    begin = int32(np.concatenate([[0], np.cumsum(lengths)]).tolist())
    n = sum(lengths)
    k, v = (torch.randn(n, hkv, d, generator=gen).to(torch.bfloat16).to(DEV) for _ in range(2))
    if n:
        pages.write(k, v, begin, table)
    return pages, table


SHAPES = [(4, 4, 64), (32, 8, 128), (7, 1, 128), (16, 1, 64), (10, 2, 128), (16, 1, 128), (6, 2, 64), (28, 4, 128)]
LENGTHS = [[1], [16, 17, 0, 31], [127, 128, 129, 130, 64], [1000], [5000, 3, 700], [0, 0]]


@gpu
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("lengths", LENGTHS)
@pytest.mark.parametrize("hq,hkv,d", SHAPES)
def test_against_64_bits(hq, hkv, d, lengths, page, e4m3):
    gen = torch.Generator().manual_seed(hq * 1000 + sum(lengths) + page)
    pages, table = a_batch(gen, lengths, hkv, d, page, e4m3)
    q = (1.5 * torch.randn(len(lengths), hq, d, generator=gen)).to(torch.bfloat16)
    print("paged decode", hq, hkv, d, lengths, page, e4m3, flush=True)
    work = pages.workspace(hq).fill_(0xFF)
    out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device=DEV)
    pages.decode(q.to(DEV), table, int32(lengths), out=out, workspace=work)
    torch.cuda.synchronize()
    ref, size, most = reference(q.double().numpy(), Pool(pages), table.cpu().numpy(), lengths, pages.n_pages, page, d ** -0.5)
    check(out, ref, size, most, d)


@gpu
@pytest.mark.parametrize("e4m3", [False, True])
def test_pages_that_are_not_there_and_lengths_out_of_range(e4m3):
    gen = torch.Generator().manual_seed(3)
    page, hq, hkv, d, lengths = 32, 8, 2, 128, [200, 96, 33, 64, 500]          # (the second one's pages are full: it is taken further)
    pages, table = a_batch(gen, lengths, hkv, d, page, e4m3)
    q = torch.randn(len(lengths), hq, d, generator=gen).to(torch.bfloat16)
    table[0, 0], table[0, 4], table[1, 1], table[2, 1], table[4, 3:11] = -1, pages.n_pages, -7, 2 ** 31 - 1, -2 ** 31
    table[3] = -1                                          # none left
    said = [200, 2 ** 31 - 1, 33, 64, 500]
    table[1, 3:] = table[0, 2]                             # (what the longer length reaches)
    for given in (said, [-5, 96, 0, -2 ** 31, 499]):
        out = pages.decode(q.to(DEV), table, int32(given))
        torch.cuda.synchronize()
        ref, size, most = reference(q.double().numpy(), Pool(pages), table.cpu().numpy(), given, pages.n_pages, page, d ** -0.5)
        check(out, ref, size, most, d)
        assert not out[3].any()


@gpu
@pytest.mark.parametrize("e4m3", [False, True])
def test_many_sequences(e4m3):
    gen = torch.Generator().manual_seed(8)
    lengths = [int(x) for x in torch.randint(0, 400, (150,), generator=gen)]
    lengths[:70] = [0] * 70
    lengths[149] = 2500
    pages, table = a_batch(gen, lengths, 2, 64, 16, e4m3)
    q = torch.randn(150, 3, 6, 64, generator=gen).to(torch.bfloat16)
    out = pages.decode(q.to(DEV)[:, 1], table, int32(lengths), softmax_scale=0.3)      # rows of another tensor
    torch.cuda.synchronize()
    ref, size, most = reference(q[:, 1].double().numpy(), Pool(pages), table.cpu().numpy(), lengths, pages.n_pages, 16, 0.3)
    check(out, ref, size, most, 64)


@gpu
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("hq,hkv,d,page,lengths", [
    (32, 32, 64, 16, [2001, 1, 0, 700, 33, 2500, 16, 129]),                   # a workgroup each, more than 64 columns of the table
    (16, 16, 128, 64, [2500] + [37 * i % 900 for i in range(17)]),
    (32, 2, 64, 64, [60001] + [11 * i for i in range(39)]),                   # many sequences, one of them in hundreds of pieces
    (8, 1, 128, 256, [30000, 0, 1, 257]),                                     # few
])
def test_every_way_to_spread_the_work(hq, hkv, d, page, lengths, e4m3):
    gen = torch.Generator().manual_seed(hq + page)
    pages, table = a_batch(gen, lengths, hkv, d, page, e4m3)
    q = (2 * torch.randn(len(lengths), hq, d, generator=gen)).to(torch.bfloat16)
    print("paged decode, ways", hq, hkv, d, page, len(lengths), e4m3, flush=True)
    out = pages.decode(q.to(DEV), table, int32(lengths), workspace=pages.workspace(hq).fill_(0xFF))
    wide = torch.full((len(lengths), 2 * table.shape[1] + 200), -1, dtype=torch.int32, device=DEV)
    wide[:, :table.shape[1]] = table                                          # the same under a table that says less
    again = pages.decode(q.to(DEV), wide, int32(lengths))
    torch.cuda.synchronize()
    ref, size, most = reference(q.double().numpy(), Pool(pages), table.cpu().numpy(), lengths, pages.n_pages, page, d ** -0.5)
    check(out, ref, size, most, d)
    check(again, ref, size, most, d)


@gpu
@pytest.mark.parametrize("e4m3", [False, True])
def test_a_long_sequence_and_the_same_bits_again(e4m3):
    """All workgroups on the pieces of one sequence; large logits, the largest of them last."""
    gen = torch.Generator().manual_seed(9)
    n, page, hq, hkv, d = 20011, 16, 8, 1, 128
    pages, table = a_batch(gen, [n], hkv, d, page, e4m3)
    q = (8 * torch.randn(1, hq, d, generator=gen)).to(torch.bfloat16).to(DEV)
    row = 30 * q[:, :1] / q[:, :1].float().norm()
    pages.write(row.to(torch.bfloat16), row.to(torch.bfloat16), int32([0, 1]), table, first=int32([n - 1]))
    out = pages.decode(q, table, int32([n]))
    again = [pages.decode(q, table, int32([n])) for _ in range(3)]
    torch.cuda.synchronize()
    ref, size, most = reference(q.double().cpu().numpy(), Pool(pages), table.cpu().numpy(), [n], pages.n_pages, page, d ** -0.5)
    check(out, ref, size, most, d)
    assert all(torch.equal(out.view(torch.int16), a.view(torch.int16)) for a in again)


@gpu
def test_numbers_that_are_not_finite_stay_with_their_sequence_and_head():
    gen = torch.Generator().manual_seed(10)
    pages, table = a_batch(gen, [300, 300], 2, 128, 64, False)
    q = torch.randn(2, 4, 128, generator=gen).to(torch.bfloat16).to(DEV)
    good = pages.decode(q, table, int32([300, 300]))
    pages.v[table[0, 1], 1, 5, 7] = float("inf")
    pages.k[table[1, 2], 0, 9] = float("nan")
    out = pages.decode(q, table, int32([300, 300]))
    torch.cuda.synchronize()
    assert torch.equal(out[0, :2], good[0, :2]) and torch.equal(out[1, 2:], good[1, 2:])
    assert torch.isinf(out[0, 2:, 7]).all() and torch.isfinite(out[0, 2:, :7]).all()
    assert torch.isnan(out[1, :2]).all()


@gpu
@pytest.mark.parametrize("e4m3", [False, True])
def test_a_graph_of_steps_goes_on_with_other_lengths(e4m3):
    """Write the token, attend, in a graph with a workspace that a second graph shares; eager work between the replays."""
    gen = torch.Generator().manual_seed(11)
    lengths, page, hq, hkv, d = [100, 0, 57], 16, 8, 2, 128
    pages, table = a_batch(gen, [n + 40 for n in lengths], hkv, d, page, e4m3)
    k, v = (torch.randn(3, hkv, d, generator=gen).to(torch.bfloat16).to(DEV) for _ in range(2))
    q = torch.randn(3, hq, d, generator=gen).to(torch.bfloat16).to(DEV)
    at, upto, begin, work = int32(lengths), int32([n + 1 for n in lengths]), int32([0, 1, 2, 3]), pages.workspace(hq)
    outs = [torch.empty_like(q) for _ in range(2)]

    def step(out):
        pages.write(k, v, begin, table, first=at)
        pages.decode(q, table, upto, out=out, workspace=work)
        at.add_(1), upto.add_(1)

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step(outs[0])                                      # token 0, eager, on another stream
    torch.cuda.synchronize()
    graphs = []
    for out in outs:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            step(out)
    for token in range(1, 13):
        for t in (k, v, q):
            t.copy_(torch.randn(t.shape, generator=gen))
        graphs[token % 2].replay()
        eager = pages.decode(q, table, int32([n + token + 1 for n in lengths]))
        torch.cuda.synchronize()
        ref, size, most = reference(q.double().cpu().numpy(), Pool(pages), table.cpu().numpy(), [n + token + 1 for n in lengths], pages.n_pages, page,
                                    d ** -0.5)
        check(outs[token % 2], ref, size, most, d)
        assert torch.equal(eager, outs[token % 2])


@gpu
def test_nothing_behind_the_result_and_the_workspace_is_written():
    gen = torch.Generator().manual_seed(12)
    pages, table = a_batch(gen, [900, 40], 1, 64, 64, False)
    q = torch.randn(2, 5, 64, generator=gen).to(torch.bfloat16).to(DEV)
    nbytes = K.kvp_paged_decode_bytes(pages.of, 5)
    room = torch.full((nbytes + 512,), 0xAB, dtype=torch.uint8, device=DEV)
    out = torch.full((4, 5, 64), 3.0, dtype=torch.bfloat16, device=DEV)
    pages.decode(q, table, int32([900, 40]), out=out[1:3], workspace=room[256:256 + nbytes])
    torch.cuda.synchronize()
    assert (out[0] == 3).all() and (out[3] == 3).all() and (out[1:3] != 3).any()
    assert (room[:256] == 0xAB).all() and (room[256 + nbytes:] == 0xAB).all()


def _decode(pages=None, **over):
    of = dict(q=P16, q_token=512, q_head=128, n_q_heads=4, table=P4, table_width=4, lengths=P4, n_seqs=2, softmax_scale=0.0, out=P16, workspace=P16,
              workspace_bytes=1 << 30)
    of.update(over)
    return K.kvp_paged_decode(pages or _pages(), *of.values())


def test_refusals():
    for bad in BAD_PAGES:
        assert _decode(_pages(**bad)) == K.KVP_EINVAL, bad
        assert K.kvp_paged_decode_bytes(_pages(**bad), 4) == 0
    for bad in [dict(q=None), dict(q=P16 + 8), dict(q_token=12), dict(q_head=-8), dict(n_q_heads=3), dict(n_q_heads=0), dict(n_q_heads=34), dict(table=None),
                dict(table_width=0), dict(table_width=1 << 25), dict(lengths=None), dict(lengths=P4 + 1), dict(n_seqs=0), dict(n_seqs=4097),
                dict(softmax_scale=-1.0), dict(softmax_scale=math.inf), dict(softmax_scale=math.nan), dict(out=None), dict(out=P16 + 2), dict(workspace=None),
                dict(workspace=P16 + 4), dict(table_width=1 << 24, n_seqs=4096)]:
        assert _decode(**bad) == K.KVP_EINVAL, bad
    need = K.kvp_paged_decode_bytes(_pages(), 4)
    assert need > 0 and _decode(workspace_bytes=need - 1) == K.KVP_ENOMEM
    assert K.kvp_paged_decode_bytes(_pages(), 3) == 0 and K.kvp_paged_decode_bytes(_pages(), 34) == 0
    assert K.kvp_paged_decode_bytes(_pages(format=K.KVP_PAGE_E4M3), 32) > 0


@gpu
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("width", [4, 40])
def test_pages_beyond_32_bits(e4m3, width):
    """The last pages of a pool of more than 4 GiB give what the first ones of a small pool give, alone and in shares."""
    gen = torch.Generator().manual_seed(width)
    page, heads, d, n = 256, 8, 128, 900
    many = (1 << 32) // (page * heads * d * (1 if e4m3 else 2)) + 5
    k, v = (torch.randn(n, heads, d, generator=gen).to(torch.bfloat16).to(DEV) for _ in range(2))
    q = torch.randn(1, 4 * heads, d, generator=gen).to(torch.bfloat16).to(DEV)
    outs = []
    for n_pages in (4, many):
        pages = K.Pages.empty(n_pages, heads, d, page, e4m3, DEV)
        table = torch.full((1, width), -1, dtype=torch.int32, device=DEV)
        table[0, :4] = torch.arange(n_pages - 1, n_pages - 5, -1)
        pages.write(k, v, int32([0, n]), table)
        outs.append(pages.decode(q, table, int32([n])))
    torch.cuda.synchronize()
    assert torch.equal(*outs) and outs[0].any()


@gpu
@pytest.mark.parametrize("e4m3,page", [(False, 16), (True, 256)])
def test_pieces_of_many_tiles(e4m3, page):
    """More than 32 tiles of 256 keys to a workgroup, behind a sequence of another length."""
    gen = torch.Generator(device=DEV).manual_seed(page)
    heads, d, lengths = 32, 128, [300, 135001 if e4m3 else 70001]
    counts = [-(-n // page) for n in lengths]
    pages = K.Pages.empty(sum(counts), heads, d, page, e4m3, DEV)
    if e4m3:
        for t, exp in ((pages.k, pages.k_exp), (pages.v, pages.v_exp)):
            t.view(torch.uint8).random_(0, 0x7F, generator=gen)          # every number that is one, not negative
            exp.random_(117, 121, generator=gen)
    else:
        pages.k.normal_(generator=gen), pages.v.normal_(generator=gen)
    order = torch.randperm(sum(counts), generator=gen, device=DEV).int()
    table = torch.full((2, counts[1]), -1, dtype=torch.int32, device=DEV)
    table[0, :counts[0]], table[1] = order[:counts[0]], order[counts[0]:]
    q = torch.randn(2, heads, d, generator=gen, device=DEV).to(torch.bfloat16)
    out = pages.decode(q, table, int32(lengths))
    torch.cuda.synchronize()
    ref, size, most = torch.zeros(2, heads, d, dtype=torch.float64), torch.zeros(2, heads, d, dtype=torch.float64), 0.0
    for s, n in enumerate(lengths):
        mine = table[s, :counts[s]].long()
        for h in range(heads):
            k, v = (x[mine, h].double().view(-1, d)[:n] for x in (pages.k, pages.v))
            if e4m3:
                k, v = (x * torch.exp2(e[mine, h].double() - 127).view(-1, 1)[:n] for x, e in ((k, pages.k_exp), (v, pages.v_exp)))
            one = q[s, h].double()
            w = torch.softmax((k * one).sum(-1) * d ** -0.5, 0)[:, None]
            ref[s, h], size[s, h] = (w * v).sum(0).cpu(), (w * v.abs()).sum(0).cpu()
            most = max(most, float((k.abs() * one.abs()).sum(-1).max()) * d ** -0.5)
    check(out, ref.numpy(), size.numpy(), most, d)


@gpu
def test_refusals_of_tensors():
    pages = K.Pages.empty(4, 2, 128, 64, False, DEV)
    row = lambda *shape: torch.zeros(shape, dtype=torch.bfloat16, device=DEV)
    good = dict(q=row(2, 4, 128), table=int32([[0], [1]]), lengths=int32([0, 0]))
    pages.decode(**good)
    for bad in [dict(q=row(2, 4, 64)), dict(q=row(3, 4, 128)), dict(q=row(2, 3, 128)), dict(q=row(2, 4, 128).float()), dict(q=row(4, 128)),
                dict(table=int32([[0]])), dict(lengths=int32([0, 0]).long()), dict(lengths=torch.zeros(2, dtype=torch.int32)), dict(out=row(2, 4, 64)),
                dict(out=row(2, 4, 256)[..., :128]), dict(workspace=torch.empty(64, dtype=torch.uint8, device=DEV))]:
        with pytest.raises(K.KvpError):
            pages.decode(**dict(good, **bad))
    torch.cuda.synchronize()


@gpu
@pytest.mark.parametrize("width", [16, 300])                                   # a workgroup for each sequence and head, and in shares
@pytest.mark.parametrize("d,hq,hkv", [(128, 8, 2), (64, 5, 1), (128, 32, 8), (64, 48, 4)])      # (the last two: joins of many sequences)
def test_logits_of_minus_infinity(d, hq, hkv, width):
    """Softmax of nothing but minus infinity is 0 / 0; beside a logit that is finite such keys weigh nothing; and without any key the result is zeros."""
    gen = torch.Generator().manual_seed(d + width)
    page, lengths = 64, [1000, 1000, 1000, 1000, 0, 40, 700]
    pages, table = a_batch(gen, lengths, hkv, d, page, False)
    table = torch.cat([table, torch.full((len(lengths), width - table.shape[1]), -1, dtype=torch.int32, device=DEV)], 1)
    q = (torch.randn(len(lengths), hq, d, generator=gen).abs() + 0.125).to(torch.bfloat16)

    def hide(seq, *keys):
        for i in keys:
            pages.k[table[seq, i // page].item(), :, i % page] = -math.inf

    hide(0, *range(1000))                                                      # all
    hide(1, *range(999))                                                       # all but the last one
    hide(2, *range(1, 1000))                                                   # all but the first one
    hide(3, *range(128, 600))
    hide(5, *range(40))
    hide(6, *range(700))
    table[6] = -1                                                              # no key of these is there
    out = pages.decode(q.to(DEV), table, int32(lengths), workspace=pages.workspace(hq).fill_(0xFF))
    torch.cuda.synchronize()
    assert torch.isnan(out[[0, 5]]).all() and not out[[4, 6]].any()
    finite = pages.k.nan_to_num(neginf=0.0)
    for s, seen in ((1, [999]), (2, [0]), (3, [*range(128), *range(600, 1000)])):
        for h in range(hq):
            at = [(table[s, i // page].item(), h // (hq // hkv), i % page) for i in seen]
            k, v = (torch.stack([t[i] for i in at]).double().cpu() for t in (finite, pages.v))
            one = q[s, h].double()
            w = torch.softmax(k @ one * d ** -0.5, 0)
            most = float((k.abs() @ one.abs()).max()) * d ** -0.5
            check(out[s, h], (w @ v).numpy(), (w @ v.abs()).numpy(), most, d)


@gpu
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 64), (16, 8, 128)])
@pytest.mark.parametrize("n,empty", [(64, 0), (65, 0), (64, 63), (128, 64), (129, 64), (129, -64), (200, 128), (300, -130)])
def test_shares_of_more_sequences_than_a_wave_has_lanes(n, empty, hq, hkv, d, e4m3):
    """Lengths are added up 64 at a time: groups of sequences that are empty before, behind and between others, under a table that says little."""
    gen = torch.Generator().manual_seed(n + empty + d)
    lengths = [int(x) for x in torch.randint(0, 700, (n,), generator=gen)]
    begin = 0 if empty >= 0 else 70 if n > 200 else 32
    lengths[begin:begin + abs(empty)] = [0] * abs(empty)
    lengths[-1], lengths[n // 2 + 40 if n > 128 else -2] = 2900, 257
    pages, table = a_batch(gen, lengths, hkv, d, 32, e4m3)
    wide = torch.full((n, table.shape[1] + 30), -1, dtype=torch.int32, device=DEV)
    wide[:, :table.shape[1]] = table
    q = torch.randn(n, hq, d, generator=gen).to(torch.bfloat16)
    print("paged decode, many in shares", n, empty, hq, hkv, d, e4m3, flush=True)
    out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device=DEV)
    pages.decode(q.to(DEV), wide, int32(lengths), out=out, workspace=pages.workspace(hq).fill_(0xFF))
    torch.cuda.synchronize()
    ref, size, most = reference(q.double().numpy(), Pool(pages), table.cpu().numpy(), lengths, pages.n_pages, 32, d ** -0.5)
    check(out, ref, size, most, d)


@gpu
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("width", [2, 200])
def test_as_many_sequences_as_a_call_takes(width, e4m3):
    gen = torch.Generator().manual_seed(width)
    n, hq, hkv, d, page = K.KVP_MAX_SEQUENCES, 2, 1, 64, 16
    lengths = [int(x) for x in torch.randint(0, 33, (n,), generator=gen)]
    lengths[100:500] = [0] * 400
    pages, table = a_batch(gen, lengths, hkv, d, page, e4m3)
    wide = torch.full((n, width), -1, dtype=torch.int32, device=DEV)
    wide[:, :table.shape[1]] = table
    q = torch.randn(n, hq, d, generator=gen).to(torch.bfloat16)
    out = pages.decode(q.to(DEV), wide, int32(lengths))
    torch.cuda.synchronize()
    ref, size, most = reference(q.double().numpy(), Pool(pages), table.cpu().numpy(), lengths, pages.n_pages, page, d ** -0.5)
    check(out, ref, size, most, d)


@pytest.mark.parametrize("scale", [2.4e38, 3.4e38])
def test_scales_that_are_too_large(scale):
    """A scale is taken times log2(e), which these are not finite with: every result would be NaN."""
    assert _decode(softmax_scale=scale) == K.KVP_EINVAL
    prompts = K.KvpPrompts(q=P16, k=P16, v=P16, out=P16, seq_begin=P4, q_token=512, q_head=128, k_token=256, k_head=128, v_token=256, v_head=128, out_token=512,
                           out_head=128, n_tokens=5, n_seqs=2, n_q_heads=4, n_kv_heads=2, head_dim=128, softmax_scale=scale)
    assert K.kvp_prompt_attention(prompts) == K.KVP_EINVAL
